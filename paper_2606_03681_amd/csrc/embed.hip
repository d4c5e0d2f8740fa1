// Embedding rows and their gradient (declarations in vocab.h).
#include "vocab.h"

#include <hip/hip_runtime.h>

namespace tfm {
namespace {

// First element of the activations' row n.
__device__ __forceinline__ int64_t row_at(const EmbedGeo& g, int64_t n) {
  const int64_t ij = n / g.n2, k = n - ij * g.n2;
  const int64_t i = ij / g.n1, j = ij - i * g.n1;
  return i * g.stride[0] + j * g.stride[1] + k * g.stride[2];
}

template <class TT, class TO, bool ADD>
__global__ __launch_bounds__(256) void k_embed_fwd(EmbedGeo g, const int32_t* __restrict__ ids,
                                                   const TT* __restrict__ table,
                                                   TO* __restrict__ out) {
  for (int64_t n = blockIdx.x; n < g.N; n += gridDim.x) {
    const int32_t id = ids[n];
    const bool here = (uint32_t)id < (uint32_t)g.V;
    if (ADD && !here) continue;
    TO* o = out + row_at(g, n);
    const TT* t = table + (int64_t)(here ? id : 0) * g.E;
    for (int c = threadIdx.x; c < g.E; c += 256) {
      float v = here ? g.scale * ld(t + c) : 0.f;
      if (ADD) v += ld(o + c);
      st(o + c, v);
    }
  }
}

// One workgroup per table row: the positions in order, those that hold the row's id added up.
template <class TO, bool ADD>
__global__ __launch_bounds__(256) void k_embed_bwd(EmbedGeo g, const int32_t* __restrict__ ids,
                                                   const TO* __restrict__ dout,
                                                   float* __restrict__ dtable) {
  __shared__ int hit[256];
  __shared__ int nhit[4];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  for (int v = blockIdx.x; v < g.V; v += gridDim.x) {
    for (int c0 = 0; c0 < g.E; c0 += 256) {
      const int c = c0 + tid;
      float acc = 0.f;
      bool any = false;
      for (int64_t n0 = 0; n0 < g.N; n0 += 256) {
        const int64_t n = n0 + tid;
        const bool mine = n < g.N && ids[n] == v;
        const uint64_t b = __ballot(mine);
        __syncthreads();
        if (lane == 0) nhit[w] = __popcll(b);
        __syncthreads();
        int at = __popcll(b & ((1ull << lane) - 1)), total = 0;
        for (int i = 0; i < 4; ++i) {
          if (i < w) at += nhit[i];
          total += nhit[i];
        }
        if (mine) hit[at] = tid;
        __syncthreads();
        for (int i = 0; i < total; ++i)
          if (c < g.E) acc += ld(dout + row_at(g, n0 + hit[i]) + c);
        any |= total > 0;
      }
      if (c < g.E) {
        float* o = dtable + (int64_t)v * g.E + c;
        if (!ADD) *o = g.scale * acc;
        else if (any) *o += g.scale * acc;
      }
    }
  }
}

}  // namespace

template <class TT, class TO>
hipError_t launch_embed_fwd(const EmbedGeo& g, const int32_t* ids, const TT* table, TO* out,
                            int accumulate, hipStream_t s) {
  const unsigned blocks = (unsigned)(g.N < 65536 ? g.N : 65536);
  if (accumulate) k_embed_fwd<TT, TO, true><<<blocks, 256, 0, s>>>(g, ids, table, out);
  else k_embed_fwd<TT, TO, false><<<blocks, 256, 0, s>>>(g, ids, table, out);
  return hipGetLastError();
}

size_t embed_bwd_bytes(const EmbedGeo&) { return 16; }

template <class TO>
hipError_t launch_embed_bwd(const EmbedGeo& g, const int32_t* ids, const TO* dout, float* dtable,
                            int accumulate, void* ws, hipStream_t s) {
  const unsigned blocks = (unsigned)(g.V < 65536 ? g.V : 65536);
  if (accumulate) k_embed_bwd<TO, true><<<blocks, 256, 0, s>>>(g, ids, dout, dtable);
  else k_embed_bwd<TO, false><<<blocks, 256, 0, s>>>(g, ids, dout, dtable);
  return hipGetLastError();
}

#define FWD(TT, TO)                                                                            \
  template hipError_t launch_embed_fwd<TT, TO>(const EmbedGeo&, const int32_t*, const TT*, TO*, \
                                               int, hipStream_t);
FWD(float, float)
FWD(float, bf16)
FWD(bf16, float)
FWD(bf16, bf16)
template hipError_t launch_embed_bwd<float>(const EmbedGeo&, const int32_t*, const float*, float*,
                                            int, void*, hipStream_t);
template hipError_t launch_embed_bwd<bf16>(const EmbedGeo&, const int32_t*, const bf16*, float*,
                                           int, void*, hipStream_t);

}  // namespace tfm
