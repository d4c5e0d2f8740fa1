// Attention of query rows over a pool of e4m3 codes (declarations in cache8.h).
//
// One wave per (sequence, row, head): a lane has a key of each 64, then a few channels of the sum.
#include "cache8.h"
#include "mfma.h"
#include "wave.h"

namespace tfm {
namespace {

constexpr int kMaxBlocks = 1 << 20;

template <class T>
__global__ __launch_bounds__(64) void k_cache8_attend(Cache8Attend a, const T* __restrict__ q,
                                                      T* __restrict__ out, int64_t items) {
  __shared__ float qs[128], ps[64];
  __shared__ int64_t blocks[64];
  __shared__ float vs[64];
  const Cache8Geo& g = a.g;
  const int d = g.d, lane = threadIdx.x;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int h = (int)(it % a.heads), kh = h / (a.heads / g.heads);
    const int64_t bi = it / a.heads, b = bi / a.L;
    const int i = (int)(bi % a.L);
    const int rows = a.n_rows ? min(max(a.n_rows[b], 0), a.L) : a.L;
    if (i >= rows) continue;
    const int len = min(max(a.lens[b], 0), a.max_rows);
    const int64_t upto64 = a.causal ? (int64_t)len - rows + i + 1 : len;
    const int upto = (int)max((int64_t)0, min(upto64, (int64_t)len));
    const T* qr = q + b * a.sq[0] + i * a.sq[1] + h * a.sq[2];
    __syncthreads();
    for (int c = lane; c < d; c += 64) qs[c] = ld(qr + c) ;
    __syncthreads();
    float m = -3e38f, l = 0.f, o0 = 0.f, o1 = 0.f;
    for (int j0 = 0; j0 < upto; j0 += 64) {
      const int j = j0 + lane;
      float s = -INFINITY;
      int pid = -1;
      if (j < upto) pid = cache8_page(g, b, j >> g.shift);
      if (pid >= 0) {
        const int64_t block = (int64_t)pid * g.heads + kh;
        const uint8_t* kr = g.keys + (block * g.page + (j & (g.page - 1))) * d;
        s = 0.f;
        for (int c = 0; c < d; ++c) s += qs[c] * __builtin_amdgcn_cvt_f32_fp8(kr[c], 0);
        const int ek = min(max((int)g.powers[2 * block], CACHE8_E_MIN), CACHE8_E_MAX);
        const int ev = min(max((int)g.powers[2 * block + 1], CACHE8_E_MIN), CACHE8_E_MAX);
        s *= __uint_as_float((uint32_t)ek << 23) * a.scale_log2;
        vs[lane] = __uint_as_float((uint32_t)ev << 23);
        blocks[lane] = block * g.page * d + (j & (g.page - 1));
      } else {
        blocks[lane] = -1;
      }
      const float top = fmaxf(m, wave_max(s));
      const float p = pid >= 0 ? exp2f(s - top) : 0.f, keep = exp2f(m - top);
      m = top;
      l = l * keep + wave_sum(p);
      o0 *= keep;
      o1 *= keep;
      __syncthreads();
      ps[lane] = p;
      __syncthreads();
      for (int t = 0; t < 64; ++t) {
        if (blocks[t] < 0) continue;
        const uint8_t* vr = g.values + blocks[t];
        const float w = ps[t] * vs[t];
        if (lane < d) o0 += w * __builtin_amdgcn_cvt_f32_fp8(vr[lane * g.page], 0);
        if (lane + 64 < d) o1 += w * __builtin_amdgcn_cvt_f32_fp8(vr[(lane + 64) * g.page], 0);
      }
      __syncthreads();
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T* orow = out + b * a.so[0] + i * a.so[1] + h * a.so[2];
    if (lane < d) st(orow + lane, l == 0.f ? 0.f : o0 * inv);
    if (lane + 64 < d) st(orow + lane + 64, l == 0.f ? 0.f : o1 * inv);
    if (a.lse && lane == 0)
      a.lse[bi * a.heads + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
  }
}

}  // namespace

size_t cache8_attend_bytes(const Cache8Attend&) { return 0; }

template <class T>
hipError_t launch_cache8_attend(const Cache8Attend& a, const T* q, T* out, hipStream_t s) {
  const int64_t items = (int64_t)a.B * a.L * a.heads;
  k_cache8_attend<T><<<(unsigned)(items < kMaxBlocks ? items : kMaxBlocks), 64, 0, s>>>(a, q, out,
                                                                                       items);
  return hipGetLastError();
}
template hipError_t launch_cache8_attend(const Cache8Attend&, const float*, float*, hipStream_t);
template hipError_t launch_cache8_attend(const Cache8Attend&, const bf16*, bf16*, hipStream_t);

}  // namespace tfm
