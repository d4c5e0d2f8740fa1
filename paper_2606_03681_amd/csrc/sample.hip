// Sampling (declarations in vocab.h).
#include "vocab.h"

#include <hip/hip_runtime.h>

namespace tfm {
namespace {

typedef unsigned long long u64;

// Logits as integers in the same order: 0 for what is never drawn (-inf and NaN).
__device__ __forceinline__ uint32_t key_of(float x) {
  if (!(x > -INFINITY)) return 0;
  const uint32_t u = __float_as_uint(x + 0.f);  // -0 and 0 are equal
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

template <class V, class F>
__device__ __forceinline__ V block_all(V v, V* buf, F op) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = op(v, __shfl_xor(v, o));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
  __syncthreads();
  return op(op(buf[0], buf[1]), op(buf[2], buf[3]));
}

// One workgroup per row.
template <class T>
__global__ __launch_bounds__(256) void k_sample(SampleGeo g, const T* __restrict__ logits,
                                                double one) {
  __shared__ u64 buf[4];
  __shared__ u64 scan_w[4];
  __shared__ uint32_t scan_t[4];
  __shared__ int found;
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  auto add = [](u64 a, u64 b) { return a + b; };
  auto mx = [](u64 a, u64 b) { return a > b ? a : b; };
  auto mn = [](u64 a, u64 b) { return a < b ? a : b; };
  for (int64_t n = blockIdx.x; n < g.N; n += gridDim.x) {
    const T* s = logits + n * g.ld;
    int V = g.V;
    if (g.ncls) V = min(max(g.ncls[n], 0), g.V);
    // the largest key and its lowest index in one number
    u64 best = 0;
    for (int v = tid; v < V; v += 256) {
      const uint32_t k = key_of(ld(s + v));
      if (k) best = mx(best, (u64)k << 32 | (uint32_t)~v);
    }
    best = block_all(best, buf, mx);
    const uint32_t kmax = (uint32_t)(best >> 32);
    const float tau = g.temperature ? g.temperature[n] : 1.f;
    const int topk = g.top_k ? g.top_k[n] : 0;
    const float topp = g.top_p ? g.top_p[n] : 1.f;
    const float minp = g.min_p ? g.min_p[n] : 0.f;
    if (kmax == 0 || !(tau > 0.f) || topk == 1 || topp <= 0.f || minp > 1.f) {
      if (tid == 0) {
        g.token[n] = kmax ? (int32_t)~(uint32_t)best : -1;
        if (g.logprob) g.logprob[n] = kmax ? 0.f : -INFINITY;
      }
      __syncthreads();
      continue;
    }
    const double top = (double)of_key(kmax), itau = 1.0 / (double)tau;
    auto xof = [&](uint32_t k) { return k == kmax ? 0.0 : ((double)of_key(k) - top) * itau; };
    auto weight = [&](uint32_t k) { return k ? (u64)(exp(xof(k)) * one + 0.5) : 0ull; };
    // kept so far: keys above kt, and the first rt classes whose key is kt
    uint32_t kt = 0x007fffffu;  // the key that -inf would have: below every logit's
    u64 rt = ~0ull;
    auto count_from = [&](uint32_t lo) {
      u64 c = 0;
      for (int v = tid; v < V; v += 256) c += key_of(ld(s + v)) >= lo;
      return block_all(c, buf, add);
    };
    auto mass_from = [&](uint32_t lo) {
      u64 c = 0;
      for (int v = tid; v < V; v += 256) {
        const uint32_t k = key_of(ld(s + v));
        if (k >= lo) c += weight(k);
      }
      return block_all(c, buf, add);
    };
    if (topk > 0 && count_from(1) > (u64)topk) {
      uint32_t lo = 1, hi = kmax;  // the largest key from which on at least topk classes lie
      while (lo < hi) {
        const uint32_t mid = lo + (hi - lo + 1) / 2;
        if (count_from(mid) >= (u64)topk) lo = mid;
        else hi = mid - 1;
      }
      kt = lo;
      rt = (u64)topk - (kt == kmax ? 0 : count_from(kt + 1));
    }
    if (topp < 1.f) {
      const u64 above = kt == 0xffffffffu ? 0 : mass_from(kt + 1);
      u64 ties = count_from(kt) - (kt == 0xffffffffu ? 0 : count_from(kt + 1));
      if (ties > rt) ties = rt;
      const double target = (double)topp * (double)(above + ties * weight(kt));
      uint32_t lo = kt, hi = kmax;  // the smallest key above which less than the target lies
      while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2;
        if ((double)mass_from(mid + 1) < target) hi = mid;
        else lo = mid + 1;
      }
      const u64 before = lo == 0xffffffffu ? 0 : mass_from(lo + 1);
      const u64 w = weight(lo);
      u64 r = ~0ull;
      if (w) {
        const double q = (target - (double)before) / (double)w;
        if (q < 2.0 * VOCAB_VMAX) {  // else every class with this key is kept
          r = (u64)q;
          while (r > 0 && !((double)(before + (r - 1) * w) < target)) --r;
          while ((double)(before + r * w) < target) ++r;
        }
      }
      if (lo > kt) { kt = lo; rt = r; }
      else if (r < rt) rt = r;
      if (rt == 0) rt = 1;
    }
    const double least = minp > 0.f ? log((double)minp) : -INFINITY;
    // total of the kept classes
    u64 mass = 0, ties = 0;
    for (int v = tid; v < V; v += 256) {
      const uint32_t k = key_of(ld(s + v));
      if (k > kt && xof(k) >= least) mass += weight(k);
      ties += k == kt;
    }
    mass = block_all(mass, buf, add);
    ties = block_all(ties, buf, add);
    if (ties > rt) ties = rt;
    if (xof(kt) >= least) mass += ties * weight(kt);
    float u = g.u[n];
    u = u > 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f;
    const double goal = (double)u * (double)mass;
    // walk in order of the classes
    u64 run = 0, seen = 0;
    if (tid == 0) found = -1;
    int token = -1;
    for (int v0 = 0; v0 < V && token < 0; v0 += 256) {
      const int v = v0 + tid;
      const uint32_t k = v < V ? key_of(ld(s + v)) : 0;
      const bool tie = k == kt && k != 0;
      const uint64_t tb = __ballot(tie);
      __syncthreads();
      if (lane == 0) scan_t[wv] = (uint32_t)__popcll(tb);
      __syncthreads();
      u64 rank = seen + __popcll(tb & ((1ull << lane) - 1));
      for (int i = 0; i < wv; ++i) rank += scan_t[i];
      const bool kept = k != 0 && xof(k) >= least && (k > kt || (tie && rank < rt));
      const u64 w = kept ? weight(k) : 0;
      u64 pre = w;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const u64 q = __shfl_up(pre, o);
        if (lane >= o) pre += q;
      }
      if (lane == 63) scan_w[wv] = pre;
      __syncthreads();
      u64 all = 0;
      for (int i = 0; i < 4; ++i) {
        if (i < wv) pre += scan_w[i];
        all += scan_w[i];
        seen += scan_t[i];
      }
      if (kept && (double)(run + pre) > goal && !((double)(run + pre - w) > goal)) found = v;
      __syncthreads();
      token = found;
      run += all;
    }
    if (tid == 0) {
      g.token[n] = token;
      if (g.logprob)
        g.logprob[n] = (float)(xof(key_of(ld(s + token))) - log((double)mass / one));
    }
    __syncthreads();
  }
}

}  // namespace

template <class T>
hipError_t launch_sample(const SampleGeo& g, const T* logits, hipStream_t s) {
  int bits = 0;
  while ((1 << bits) < g.V) ++bits;
  const double one = ldexp(1.0, 62 - bits < 51 ? 62 - bits : 51);
  const unsigned blocks = (unsigned)(g.N < 65536 ? g.N : 65536);
  k_sample<T><<<blocks, 256, 0, s>>>(g, logits, one);
  return hipGetLastError();
}
template hipError_t launch_sample<float>(const SampleGeo&, const float*, hipStream_t);
template hipError_t launch_sample<bf16>(const SampleGeo&, const bf16*, hipStream_t);

}  // namespace tfm
