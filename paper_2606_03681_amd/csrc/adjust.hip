// Penalties, biases and masks on logits (declarations in vocab.h).
//
// A workgroup per row and slice of its classes: counts of the slice's classes among the row's history
// and the first bias entry of each, in LDS; then one pass over the logits.
#include "vocab.h"

namespace tfm {
namespace {

constexpr int SLICE = 2048, kMaxBlocks = 1 << 20;

template <class T>
__global__ __launch_bounds__(256) void k_adjust(AdjustGeo g, const T* logits, T* out, int slices,
                                                int64_t items) {
#pragma clang fp contract(off)
  __shared__ uint32_t seen[SLICE], first[SLICE];
  const int tid = threadIdx.x;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t n = it / slices;
    const int v0 = (int)(it % slices) * SLICE, w = min(SLICE, g.V - v0);
    __syncthreads();
    for (int i = tid; i < w; i += 256) seen[i] = 0, first[i] = 0xffffffffu;
    __syncthreads();
    if (g.history) {
      const int m = g.n_history ? min(max(g.n_history[n], 0), g.n_hist) : g.n_hist;
      for (int j = tid; j < m; j += 256) {
        const uint32_t v = (uint32_t)g.history[n * g.ld_history + j] - (uint32_t)v0;
        if (v < (uint32_t)w) atomicAdd(&seen[v], 1u);
      }
    }
    for (int j = tid; j < g.n_bias; j += 256) {
      const uint32_t v = (uint32_t)g.bias_idx[n * g.ld_bias + j] - (uint32_t)v0;
      if (v < (uint32_t)w) atomicMin(&first[v], (uint32_t)j);
    }
    __syncthreads();
    float r = g.repetition ? g.repetition[n] : 1.f;
    if (!(r > 0.f)) r = 1.f;
    const float pres = g.presence ? g.presence[n] : 0.f, freq = g.frequency ? g.frequency[n] : 0.f;
    const int nc = g.ncls ? min(max(g.ncls[n], 0), g.V) : g.V;
    for (int i = tid; i < w; i += 256) {
      const int v = v0 + i;
      float x = ld(logits + n * g.ld + v);
      if (seen[i]) {
        x = x > 0.f ? x / r : x * r;
        x = x - (pres + freq * (float)seen[i]);
      }
      if (first[i] != 0xffffffffu) x = x + g.bias[n * g.ld_bias + first[i]];
      const bool ok = v < nc && (!g.allowed || (g.allowed[n * g.ld_allowed + v / 32] >> (v % 32)) & 1);
      st(out + n * g.ld_out + v, ok ? x : -INFINITY);
    }
  }
}

}  // namespace

template <class T>
hipError_t launch_adjust(const AdjustGeo& g, const T* logits, T* out, hipStream_t s) {
  const int slices = (g.V + SLICE - 1) / SLICE;
  const int64_t items = g.N * slices;
  k_adjust<T><<<(unsigned)(items < kMaxBlocks ? items : kMaxBlocks), 256, 0, s>>>(g, logits, out,
                                                                                 slices, items);
  return hipGetLastError();
}
template hipError_t launch_adjust(const AdjustGeo&, const float*, float*, hipStream_t);
template hipError_t launch_adjust(const AdjustGeo&, const bf16*, bf16*, hipStream_t);

}  // namespace tfm
