// Rows of keys and values into a pool of e4m3 codes (declarations in cache8.h).
//
// A workgroup per block (page, head) that gets rows.  Every step is exact but the rounding to a code,
// so that the bytes do not depend on how the work is split: the power of two comes from the bits of
// the block's largest magnitude, and products with powers of two do not round.
#include "cache8.h"

namespace tfm {
namespace {

constexpr int kMaxBlocks = 1 << 20;

// The byte of the least power with m <= 448 2^(e - 127): 448 = 1.75 2^8.
__device__ __forceinline__ int power_of(float m) {
  const uint32_t u = __float_as_uint(m);
  const int e = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u);
  return min(max(e, CACHE8_E_MIN), CACHE8_E_MAX);
}
__device__ __forceinline__ float two_to(int e) {  // 2^e, -126 <= e <= 127
  return __uint_as_float((uint32_t)(e + 127) << 23);
}
__device__ __forceinline__ bool fits(float x) { return fabsf(x) <= 0x1.cp56f; }  // 448 2^48
__device__ __forceinline__ uint8_t code_of(float x) {
  return (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, 0.f, 0, false);
}

template <class T>
__global__ __launch_bounds__(256) void k_cache8_append(Cache8Append a, const T* __restrict__ k,
                                                       const T* __restrict__ v, int slots,
                                                       int64_t items) {
  __shared__ uint32_t top[2];
  const Cache8Geo& g = a.g;
  const int d = g.d, page = g.page, tid = threadIdx.x;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int h = (int)(it % g.heads);
    const int64_t bs = it / g.heads;
    const int64_t b = bs / slots;
    const int64_t cap = (int64_t)g.max_pages << g.shift;
    const int64_t first = a.lens ? min(max((int64_t)a.lens[b], (int64_t)0), cap) : 0;
    const int64_t n = a.n_new ? min(max(a.n_new[b], 0), a.L) : a.L;
    const int64_t e = (first >> g.shift) + bs % slots;
    const int64_t lo = max(first, e << g.shift), hi = min(min(first + n, (e + 1) << g.shift), cap);
    if (lo >= hi) continue;
    const int pid = cache8_page(g, b, (int)e);
    if (pid < 0) continue;
    const int had = (int)(lo - (e << g.shift)), m = (int)(hi - lo);
    const int64_t block = (int64_t)pid * g.heads + h;
    const T* kr = k + b * a.sk[0] + (lo - first) * a.sk[1] + h * a.sk[2];
    const T* vr = v + b * a.sv[0] + (lo - first) * a.sv[1] + h * a.sv[2];
    __syncthreads();
    if (tid < 2) top[tid] = 0;
    __syncthreads();
    float mk = 0.f, mv = 0.f;
    for (int i = tid; i < m * d; i += 256) {
      const float x = fabsf(ld(kr + (i / d) * a.sk[1] + i % d));
      const float y = fabsf(ld(vr + (i / d) * a.sv[1] + i % d));
      if (fits(x)) mk = fmaxf(mk, x);
      if (fits(y)) mv = fmaxf(mv, y);
    }
    atomicMax(&top[0], __float_as_uint(mk));
    atomicMax(&top[1], __float_as_uint(mv));
    __syncthreads();
    uint8_t* pw = g.powers + block * 2;
    int ek = power_of(__uint_as_float(top[0])), ev = power_of(__uint_as_float(top[1]));
    int ok = ek, ov = ev;
    if (had) {
      ok = min(max((int)pw[0], CACHE8_E_MIN), CACHE8_E_MAX);
      ov = min(max((int)pw[1], CACHE8_E_MIN), CACHE8_E_MAX);
      ek = max(ek, ok);
      ev = max(ev, ov);
    }
    __syncthreads();
    if (tid == 0) pw[0] = (uint8_t)ek, pw[1] = (uint8_t)ev;
    uint8_t* kc = g.keys + block * page * d;
    uint8_t* vc = g.values + block * page * d;
    if (ok != ek || ov != ev) {
      for (int i = tid; i < had * d; i += 256) {
        uint8_t* p = kc + i;
        uint8_t* r = vc + (i % d) * page + i / d;
        if (ok != ek && (*p & 0x7f) != 0x7f)
          *p = code_of(__builtin_amdgcn_cvt_f32_fp8(*p, 0) * two_to(ok - ek));
        if (ov != ev && (*r & 0x7f) != 0x7f)
          *r = code_of(__builtin_amdgcn_cvt_f32_fp8(*r, 0) * two_to(ov - ev));
      }
    }
    const float fk = two_to(127 - ek), fv = two_to(127 - ev);
    for (int i = tid; i < m * d; i += 256) {
      const float x = ld(kr + (i / d) * a.sk[1] + i % d);
      const float y = ld(vr + (i / d) * a.sv[1] + i % d);
      kc[had * d + i] = fits(x) ? code_of(x * fk) : CACHE8_NAN;
      vc[(i % d) * page + had + i / d] = fits(y) ? code_of(y * fv) : CACHE8_NAN;
    }
  }
}

}  // namespace

template <class T>
hipError_t launch_cache8_append(const Cache8Append& a, const T* k, const T* v, hipStream_t s) {
  const int slots = (int)(((int64_t)a.L + a.g.page - 2) / a.g.page + 1);
  const int64_t items = (int64_t)a.B * slots * a.g.heads;
  k_cache8_append<T><<<(unsigned)(items < kMaxBlocks ? items : kMaxBlocks), 256, 0, s>>>(
      a, k, v, slots, items);
  return hipGetLastError();
}
template hipError_t launch_cache8_append(const Cache8Append&, const float*, const float*, hipStream_t);
template hipError_t launch_cache8_append(const Cache8Append&, const bf16*, const bf16*, hipStream_t);

}  // namespace tfm
