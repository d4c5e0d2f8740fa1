// Rows of keys and values into a pool of e4m3 codes (declarations in cache8.h).
//
// A block (page, head) that gets rows goes to one wave, or to a workgroup where it may get more than a
// wave's registers hold.  A lane has 8 channels of 4 rows in a row: it reads them once (again, from the
// caches, where there are more than one such piece for a lane), the lanes' largest magnitudes give the
// block's power, and the codes of the keys go out as they are, those of the values through LDS, where
// 4 rows of a channel are one word and 16 leave together.
//
// Every step is exact but the rounding to a code, so that the bytes do not depend on how the work is
// split: the power of two comes from the bits of the largest magnitude, and products with powers of two
// do not round.
//
// Bound: HBM.  1616 sequences of 768 rows, 6 heads, d = 32, bfloat16: 259 us, 5.5 TB/s (element by
// element, values scattered to their channels, it was 1259); one row of 64 sequences, 8 heads, d = 128:
// 8 us, one wave's chain of loads (length, page, power, row).  Where a block's power grows its old codes
// go one byte a lane at a time: the same step with all 512 blocks growing at their last row takes 20, 86
// and 357 us at pages of 16, 64 and 256.
#include "cache8.h"
#include "mfma.h"
#include "wave.h"

namespace tfm {
namespace {

constexpr int kMaxBlocks = 1 << 23;

// The byte of the least power with m <= 448 2^(e - 127): 448 = 1.75 2^8.
__device__ __forceinline__ int power_of(float m) {
  const uint32_t u = __float_as_uint(m);
  const int e = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u);
  return min(max(e, CACHE8_E_MIN), CACHE8_E_MAX);
}
__device__ __forceinline__ bool fits(float x) { return fabsf(x) <= 0x1.cp56f; }  // 448 2^48

// Four codes of x f, NaN where x does not fit.
__device__ __forceinline__ uint32_t codes(const float* x, float f) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = fits(x[i]) ? x[i] * f : __builtin_nanf("");
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
}
__device__ __forceinline__ uint8_t again(uint8_t c, float f) {  // a code under another power
  if ((c & 0x7f) == 0x7f) return c;
  return (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_cvt_f32_fp8(c, 0) * f, 0.f, 0, false);
}

// 8 channels of a row, as they lie.
template <class T>
struct Piece {
  uint32_t w[2 * sizeof(T)];
  __device__ __forceinline__ void load(const T* p, bool wide, bool on) {
#pragma unroll
    for (int i = 0; i < (int)(2 * sizeof(T)); ++i) w[i] = 0;
    if (!on) return;
    if (wide) {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
        const uint4 u = reinterpret_cast<const uint4*>(p)[i];
        w[4 * i] = u.x; w[4 * i + 1] = u.y; w[4 * i + 2] = u.z; w[4 * i + 3] = u.w;
      }
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(p[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = p[2 * i] | (uint32_t)p[2 * i + 1] << 16;
    }
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
};

template <class T>
__device__ __forceinline__ float largest(const Piece<T>* x, float m) {
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float a = fabsf(x[r].get(i));
      m = fits(a) ? fmaxf(m, a) : m;
    }
  return m;
}

// W: waves to a block; HOLD: its rows are read once; ls: bytes between channels in LDS.
template <class T, int W, bool HOLD>
__global__ __launch_bounds__(256) void k_cache8_append(Cache8Append a, const T* __restrict__ k,
                                                       const T* __restrict__ v, int slots,
                                                       int64_t items, int ls, int wide) {
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
  __shared__ float tops[4][2];
  const Cache8Geo& g = a.g;
  const int d = g.d, page = g.page, wave = wave_id(), lane = threadIdx.x & 63;
  const int tid = W == 1 ? lane : (int)threadIdx.x;
  constexpr int N = 64 * W;
  uint8_t* img = lds + (W == 1 ? wave * ls * d : 0);
  const int64_t u0 = (int64_t)blockIdx.x * (4 / W) + (W == 1 ? wave : 0);
  const int64_t cap = (int64_t)g.max_pages << g.shift;
  const int dp = d / 8;  // pieces of a row
  for (int64_t it = u0; it < items; it += (int64_t)gridDim.x * (4 / W)) {
    const int h = (int)(it % g.heads);
    const int64_t bs = it / g.heads, b = bs / slots;
    const int64_t first = a.lens ? min(max((int64_t)a.lens[b], (int64_t)0), cap) : 0;
    const int64_t n = a.n_new ? min(max(a.n_new[b], 0), a.L) : a.L;
    const int64_t e = (first >> g.shift) + (bs - b * slots);
    const int64_t lo = max(first, e << g.shift), hi = min(min(first + n, (e + 1) << g.shift), cap);
    if (lo >= hi) continue;
    const int pid = cache8_page(g, b, (int)e);
    if (pid < 0) continue;
    const int had = (int)(lo - (e << g.shift)), end = had + (int)(hi - lo);
    const int64_t block = (int64_t)pid * g.heads + h;
    const int g0 = had / 16, ng = (end + 15) / 16 - g0;  // the image: slots from 16 g0 on
    // slot s of the block is row lo - first + s - had
    const T* kr = k + b * a.sk[0] + (lo - first - had) * a.sk[1] + h * a.sk[2];
    const T* vr = v + b * a.sv[0] + (lo - first - had) * a.sv[1] + h * a.sv[2];
    uint8_t* pw = g.powers + block * 2;
    const uint8_t pk = pw[0], pv = pw[1];
    const int q0 = had / 4, nq = ((end + 3) / 4 - q0) * dp;  // pieces of four rows
    Piece<T> x[4], y[4];
    auto load = [&](int i) {
      const int s0 = 4 * (q0 + i / dp), c0 = i % dp * 8;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const bool on = i < nq && s0 + r >= had && s0 + r < end;
        x[r].load(kr + (s0 + r) * a.sk[1] + c0, wide, on);
        y[r].load(vr + (s0 + r) * a.sv[1] + c0, wide, on);
      }
    };
    float mk = 0.f, mv = 0.f;
    if constexpr (HOLD) {
      load(tid);
      mk = largest(x, mk);
      mv = largest(y, mv);
    } else {
      for (int i = tid; i < nq; i += N) {
        load(i);
        mk = largest(x, mk);
        mv = largest(y, mv);
      }
    }
    mk = wave_max(mk);
    mv = wave_max(mv);
    if constexpr (W > 1) {
      __syncthreads();  // the last block's image has left
      if (lane == 0) tops[wave][0] = mk, tops[wave][1] = mv;
      __syncthreads();
      mk = fmaxf(fmaxf(tops[0][0], tops[1][0]), fmaxf(tops[2][0], tops[3][0]));
      mv = fmaxf(fmaxf(tops[0][1], tops[1][1]), fmaxf(tops[2][1], tops[3][1]));
    }
    int ek = power_of(mk), ev = power_of(mv);
    uint8_t* kc = g.keys + block * page * d;
    uint8_t* vc = g.values + block * page * d;
    if (had) {
      const int ok = power_byte(pk), ov = power_byte(pv);
      ek = max(ek, ok);
      ev = max(ev, ov);
      if (ok != ek) {
        for (int i = tid; i < had * d; i += N) kc[i] = again(kc[i], two_to(ok - ek));
      }
      if (ov != ev) {
        for (int i = tid; i < had * d; i += N) {
          uint8_t* p = vc + (i % d) * page + i / d;
          *p = again(*p, two_to(ov - ev));
        }
      }
    }
    if (tid == 0) *reinterpret_cast<uint16_t*>(pw) = (uint16_t)(ek | ev << 8);
    const float fk = two_to(127 - ek), fv = two_to(127 - ev);
    for (int i = tid; i < nq; i += N) {
      if constexpr (!HOLD) load(i);
      const int s0 = 4 * (q0 + i / dp), c0 = i % dp * 8;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float z[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = x[r].get(j);
        if (s0 + r >= had && s0 + r < end)
          *reinterpret_cast<uint2*>(kc + (s0 + r) * d + c0) = make_uint2(codes(z, fk), codes(z + 4, fk));
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float z[4] = {y[0].get(j), y[1].get(j), y[2].get(j), y[3].get(j)};
        *reinterpret_cast<uint32_t*>(img + (c0 + j) * ls + s0 - 16 * g0) = codes(z, fv);
      }
    }
    if constexpr (W > 1)
      __syncthreads();
    else
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    // 16 slots of a channel at a time
    for (int i = tid; i < ng * d; i += N) {
      const int ch = i / ng, s0 = 16 * (g0 + i - ch * ng);
      const uint8_t* from = img + ch * ls + s0 - 16 * g0;
      uint8_t* to = vc + ch * page + s0;
      if (s0 >= had && s0 + 16 <= end) {
        *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(from);
      } else {
        for (int j = max(had - s0, 0); j < min(end - s0, 16); ++j) to[j] = from[j];
      }
    }
    if constexpr (W == 1) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
}

}  // namespace

template <class T>
hipError_t launch_cache8_append(const Cache8Append& a, const T* k, const T* v, hipStream_t s) {
  const Cache8Geo& g = a.g;
  // Pages that a sequence's rows may touch, of those that it has.
  const int64_t touched = ((int64_t)a.L + g.page - 2) / g.page + 1;
  const int slots = (int)(touched < g.max_pages ? touched : g.max_pages);
  const int64_t items = (int64_t)a.B * slots * g.heads;
  bool wide = (uintptr_t)k % 16 == 0 && (uintptr_t)v % 16 == 0;
  for (int i = 0; i < 3; ++i)
    wide = wide && a.sk[i] * sizeof(T) % 16 == 0 && a.sv[i] * sizeof(T) % 16 == 0;
  // pieces of 4 rows x 8 channels that a block may get
  const int rows = a.L < g.page ? a.L : g.page;
  const int most = ((rows + 2) / 4 + 1 < g.page / 4 ? (rows + 2) / 4 + 1 : g.page / 4) * (g.d / 8);
  const int W = most <= 64 ? 1 : 4;  // (a wave holds 64 pieces in registers, a workgroup 256)
  const int64_t groups = (items + 4 / W - 1) / (4 / W);
  const unsigned blocks = (unsigned)(groups < kMaxBlocks ? groups : kMaxBlocks);
  const int span = (rows + 30) / 16 * 16, ls = (span < g.page ? span : g.page) + 16;
  const size_t lds = (size_t)(4 / W) * g.d * ls;  // at most 34 KB
  if (W == 1)
    k_cache8_append<T, 1, true><<<blocks, 256, lds, s>>>(a, k, v, slots, items, ls, wide);
  else if (most <= 256)
    k_cache8_append<T, 4, true><<<blocks, 256, lds, s>>>(a, k, v, slots, items, ls, wide);
  else
    k_cache8_append<T, 4, false><<<blocks, 256, lds, s>>>(a, k, v, slots, items, ls, wide);
  return hipGetLastError();
}
template hipError_t launch_cache8_append(const Cache8Append&, const float*, const float*, hipStream_t);
template hipError_t launch_cache8_append(const Cache8Append&, const bf16*, const bf16*, hipStream_t);

}  // namespace tfm
