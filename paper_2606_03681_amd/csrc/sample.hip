// Sampling (declarations in vocab.h).
//
// A class's weight exp(x), x = (s - max) / tau <= 0, is an integer, exp(x) 2^S rounded, with S such
// that a row's sum stays below 2^63: sums of integers have no order, so that neither the shape of a
// reduction nor atomics can move a border between two classes.  The exponential is evaluated in 64
// bits; at the full rate of 64-bit products that is about what reading the logits costs.
//
// Classes in falling order of (logit, -index) are kept from the front, so what is kept is told by
// the last kept class alone.  top_k and top_p look for that class by histograms of counts or
// weights, first over equal steps of x and then, inside the step that holds the border, over ever
// finer ranges of the logit's bits, until the few classes left (they are gathered in a list) can be
// ranked against each other.  Classes too light to hold the border together stay out of the first
// histogram, and where few classes can be kept at all they go straight into the list: an atomic on
// LDS costs a wave some 115 cycles.  The draw then needs one sum over the kept classes in order of
// their indices, of which chunks are kept so that only the drawn class's chunk is read again.
//
// Rows of up to 64 classes go to groups of 8 to 64 lanes that rank all classes against each other;
// longer ones to a workgroup each.  Its passes read the row again, from the caches: a pass has some
// hundred cycles of arithmetic per 16 bytes, and few registers leave room for the waves that hide
// the loads (the row held in registers took 250 of them at 32 classes per thread).
//
// What bounds it: a weight is 19 instructions in 64 bits, some 80 cycles of a SIMD for 64 classes, and
// every class has one in the draw and another in the search for top_p: 21 us each of this chip over
// 8,192 x 5,000.  Reading that row set from HBM takes 34 us and finding the largest class 42.  The
// rest of a top-p call is reading the row four times through the caches, the histogram's atomics and,
// with 256 threads, spilled registers.  Few rows leave CUs idle: a row stays in one workgroup.
// us by mode (largest class / temperature alone / top-k / top-p / both / min-p):
//    64 x 131,072 bfloat16    13   49   55  141   68   54     (the row on one of 64 CUs)
//     1 x  32,000 float32    5.4   17   22   41   31   13
//  8,192 x  5,000 float32     42   80  123  155  149   76     (164 MB, a copy's rate: 34)
//  4,096 x    300 float32      8   17   33   35   45   20
// Rows without a class that stands out (logits within 1/16) put all classes into few bins of the
// histogram, whose atomics then wait for each other: top-p 286 us over 8,192 x 5,000 and 213 over
// 64 x 131,072, the other modes as above.
// A series of the seventh degree behind a table of 32 roots of two in LDS has 14 instructions: 7 %
// less for 1,024 threads, but 15 % more for 256 threads and bfloat16, which then spill; both have to
// round alike, so that a row's draw does not depend on its batch.
#include "math64.h"
#include "mfma.h"
#include "order.h"
#include "vocab.h"
#include "wave.h"

#include <hip/hip_runtime.h>

namespace tfm {
namespace {

// 2^f, |f| <= 1 / 2, by powers up to f^11: the Taylor series (ln 2)^k / k! to f^13, whose last two
// powers are replaced by the Chebyshev polynomials' lower terms (T13 without its first is within
// 2^-12 of x^13, T12 within 2^-11 of x^12, x = 2 f).  Off by less than 2^-55.6, of which the degree is
// 2^-56.9 and the rest the rounding of the coefficients.  In scalar registers,
// where literals would each take two moves.
struct PowerTable {
  double c[12];
};
__constant__ PowerTable POWER = {
    {1.0, 0x1.62e42fefa39efp-1, 0x1.ebfbdff82c5aep-3,
     0x1.c6b08d704a0d1p-5, 0x1.3b2ab6fb9f1d3p-7, 0x1.5d87fe78a22b2p-10,
     0x1.4309131120d4p-13, 0x1.ffcbfc75e5fb2p-17, 0x1.62bfc2f06930fp-20,
     0x1.b524db5f98239p-24, 0x1.e6221f6484be9p-28, 0x1.ea03e67c9deafp-32}};
constexpr double INV_LN2 = 0x1.71547652b82fep+0;

// A row's largest logit and scale.
struct Row {
  float max;
  double iu;    // 1 / (tau ln 2): u = x / ln 2 = (s - max) iu
  double least; // u that stands for those below it: weight 0, or (largest logit +inf, where no
                // other class can be drawn) u = 0
  int S;
  // exp(x) 2^S rounded: 2^n 2^f, n = round(u), f = u - n.  Both roundings to integers are
  // additions of large numbers.  Against the exact value the result is off by less than 0.75 of its
  // steps of 2^-51 (20 million random x, tau = 1).
  __device__ __forceinline__ uint64_t weight(float s) const {
    const double u = __builtin_fmax(((double)s - (double)max) * iu, least);
    const double t = u + 0x1.8p52, f = u - (t - 0x1.8p52);
    double p = POWER.c[11];
#pragma unroll
    for (int i = 10; i >= 0; --i) p = __builtin_fma(p, f, POWER.c[i]);
    const int32_t e = (int32_t)(uint32_t)(uint64_t)__double_as_longlong(t) + S + 1023;
    const double scale = __longlong_as_double((long long)((uint64_t)(uint32_t)(e << 20) << 32));
    return (uint64_t)__double_as_longlong(__builtin_fma(p, scale, 0x1p52)) & 0xfffffffffffffull;
  }
};

struct Settings {
  float tau, top_p, min_p, u;
  int top_k;
  bool greedy;  // the first class of the order is drawn whatever u says
};
__device__ __forceinline__ Settings settings_of(const SampleGeo& g, int64_t n) {
  Settings o;
  o.tau = g.temperature ? g.temperature[n] : 1.f;
  o.top_k = g.top_k ? g.top_k[n] : 0;
  o.top_p = g.top_p ? g.top_p[n] : 1.f;
  o.min_p = g.min_p ? g.min_p[n] : 0.f;
  o.u = g.u[n];
  o.u = o.u > 0.f ? fminf(o.u, 0x1.fffffep-1f) : 0.f;
  o.greedy = !(o.tau > 0.f) || o.top_k == 1 || o.top_p <= 0.f || o.min_p > 1.f;
  return o;
}
__device__ __forceinline__ Row row_of(const Settings& o, float max, int S) {
  return {max, INV_LN2 / (double)o.tau, max == INFINITY ? 0.0 : -86.0, S};
}
// Key of the smallest logit whose x reaches log(min_p), min_p in (0, 1].
__device__ __forceinline__ uint32_t least_key(const Settings& o, float top) {
  return min_p_key(log64((double)o.min_p), o.tau, top);
}
__device__ __forceinline__ float logprob_of(const Row& r, float s, uint64_t mass) {
  const double x = s == r.max ? 0.0 : ((double)s - (double)r.max) * r.iu * (LN2_HI + LN2_LO);
  return (float)(x - log64((double)mass * __builtin_amdgcn_ldexp(1.0, -r.S)));
}

// ---- rows of up to 64 classes -------------------------------------------------------------------
template <int W, class V, class F>
__device__ __forceinline__ V group_all(V v, F op) {
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) v = op(v, (V)__shfl_xor(v, o, W));
  return v;
}

// W lanes per row, a class each.
template <class T, int W>
__global__ __launch_bounds__(256) void k_sample_small(SampleGeo g, int64_t first, int S,
                                                      const T* __restrict__ logits) {
  const int lane = threadIdx.x % W;
  const int64_t at = first + (int64_t)blockIdx.x * (256 / W) + threadIdx.x / W;
  const bool mine = at < g.N;
  const int64_t n = mine ? at : g.N - 1;
  const int V = g.ncls ? min(max(g.ncls[n], 0), g.V) : g.V;
  const float s = lane < V ? ld(logits + n * g.ld + lane) : -INFINITY;
  const uint32_t key = key_of(s);
  const Settings o = settings_of(g, n);
  const uint32_t kmax = group_all<W>(key, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
  const Row r = row_of(o, of_key(kmax), S);
  // (next to a largest logit of +inf no other class weighs anything)
  const uint64_t w = key && !o.greedy && (r.max < INFINITY || key == kmax) ? r.weight(s) : 0;
  auto add = [](uint64_t a, uint64_t b) { return a + b; };
  // classes before this one, and their weight
  int ahead = 0;
  uint64_t before = 0;
  if (__any(o.greedy || o.top_k > 0 || o.top_p < 1.f || o.min_p > 0.f)) {
    for (int j = 0; j < W; ++j) {
      const uint32_t kj = __shfl(key, j, W);
      const uint64_t wj = __shfl((unsigned long long)w, j, W);
      const bool a = kj > key || (kj == key && j < lane);
      ahead += a;
      before += a ? wj : 0;
    }
  }
  bool kept = key != 0;
  if (o.greedy) {
    kept = kept && ahead == 0;
  } else {
    if (o.top_k > 0) kept = kept && ahead < o.top_k;
    if (o.top_p < 1.f) {
      const uint64_t mass = group_all<W>((unsigned long long)(kept ? w : 0), add);
      kept = kept && (ahead == 0 || (double)before < (double)o.top_p * (double)mass);
    }
    if (o.min_p > 0.f) kept = kept && key >= least_key(o, r.max);
  }
  const uint64_t share = kept ? (o.greedy ? 1 : w) : 0;
  uint64_t run = share;
#pragma unroll
  for (int d = 1; d < W; d <<= 1) {
    const uint64_t q = __shfl_up((unsigned long long)run, d, W);
    if (lane >= d) run += q;
  }
  const uint64_t mass = __shfl((unsigned long long)run, W - 1, W);
  const uint64_t hits = __ballot((double)run > (double)o.u * (double)mass);
  const int base = (threadIdx.x & 63) - lane;
  const uint64_t own = W == 64 ? hits : hits >> base & ((1ull << (W & 63)) - 1);
  const int token = mass ? __ffsll((unsigned long long)own) - 1 : -1;
  if (mine && lane == max(token, 0)) {
    g.token[n] = token;
    if (g.logprob)
      g.logprob[n] = token < 0 ? -INFINITY : o.greedy ? 0.f : logprob_of(r, s, mass);
  }
}

// ---- longer rows ---------------------------------------------------------------------------------
constexpr int LIST = 512;   // classes that are ranked against each other
constexpr int GROUPS = 256; // groups of threads whose maxima bound the top_k-th logit from below
                            // (four to a lane of one wave)
constexpr float STEPS_OVER = 32.f;  // x that the histogram's equal steps cover

constexpr int CHUNKS = 128;        // most stretches of a row whose weights are summed
constexpr int STRETCH = 8;         // pieces that a lane has of a stretch, at most

// One workgroup of TH threads per row.  With many rows per CU (TH = 256) more waves are worth some
// spilled registers off the loops (8,192 x 5,000 float32, top_k and top_p: 187 us unbounded, 171 at
// 6 waves per SIMD, 151 at 8; 1,024 x 50,021 bf16, top_p: 282, 280, 341).
template <class T, int TH>
__global__ __launch_bounds__(TH, TH == 256 ? (sizeof(T) == 4 ? 8 : 6) : 1) void k_sample(
    SampleGeo g, int64_t first, int S, const T* __restrict__ logits) {
  constexpr int E = 16 / sizeof(T), NW = TH / 64;
  constexpr int LOG_BINS = TH == 256 ? 9 : 11, BINS = 1 << LOG_BINS;
  __shared__ uint64_t hist[BINS];
  // classes as (key, ~index): larger is earlier in the order; and a part of them
  __shared__ uint64_t list[LIST];
  __shared__ alignas(16) uint64_t part_of[LIST];
  __shared__ uint32_t part_count;
  __shared__ uint64_t wbuf[NW];
  __shared__ uint64_t chunk[CHUNKS];
  __shared__ uint32_t count, key_lo, key_hi;
  __shared__ int32_t found_bin;
  __shared__ uint64_t found_before, found;
  const int tid = threadIdx.x, lane = tid & 63, w = wave_id();
  const int64_t n = first + blockIdx.x;
  const T* s = logits + n * g.ld;
  const int V = g.ncls ? min(max(g.ncls[n], 0), g.V) : g.V;
  // classes before the first piece; pieces; the class beside them that this thread looks after
  const int lead = min((int)(-(uintptr_t)s % 16 / sizeof(T)), V);
  const int np = (V - lead) / E;
  const char* s0 = reinterpret_cast<const char*>(s + lead);
  const int odd = tid < lead ? tid : min(tid + np * E, V);
  constexpr uint32_t NONE = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;  // -inf
  const float xo = odd < V ? ld(s + odd) : -INFINITY;
  const Settings o = settings_of(g, n);
  // The pieces in rounds of the workgroup, each wave a stretch of 64 C pieces of a round: C such
  // that the rounds come out even.
  const int rounds = (np + TH * STRETCH - 1) / (TH * STRETCH);
  const int C = rounds ? (np + TH * rounds - 1) / (TH * rounds) : 0;
  auto get = [](const uint4& u, int j) __attribute__((always_inline)) -> float {
    const uint32_t v[4] = {u.x, u.y, u.z, u.w};
    if constexpr (sizeof(T) == 4) return __uint_as_float(v[j]);
    else return __uint_as_float(j & 1 ? v[j >> 1] & 0xffff0000u : v[j >> 1] << 16);
  };
  auto load = [&](int v) __attribute__((always_inline)) {
    return *reinterpret_cast<const uint4*>(s0 + (uint32_t)v * 16u);
  };
  // f(E logits, class of the first) for all of this wave's pieces, every lane active; -inf where
  // there are no classes.  The classes beside the pieces come as one more piece.
  auto each = [&](auto f) __attribute__((always_inline)) {
    float v[E];
    for (int r = 0; r < rounds; ++r) {
      const int first_piece = (r * NW + w) * 64 * C;
      for (int c = 0; c < C && first_piece + c * 64 < np; ++c) {
        const int at = first_piece + c * 64 + lane;
        uint4 p = make_uint4(NONE, NONE, NONE, NONE);
        if (at < np) p = load(at);
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = get(p, j);
        f(v, lead + at * E);
      }
    }
    if (w == 0) {
      v[0] = xo;
#pragma unroll
      for (int j = 1; j < E; ++j) v[j] = -INFINITY;
      f(v, odd);
    }
  };
  // the sum over the workgroup, for every thread
  auto block_sum = [&](uint64_t v) __attribute__((always_inline)) -> uint64_t {
    v = wave_sum(v);
    __syncthreads();
    if (lane == 0) wbuf[w] = v;
    __syncthreads();
    return wave_sum(lane < NW ? wbuf[lane] : (uint64_t)0);
  };

  float top = -INFINITY;
  // (the row comes from HBM here: four loads in flight)
  for (int r = 0; r < rounds; ++r) {
    const int first_piece = (r * NW + w) * 64 * C + lane;
    for (int c = 0; c < C; c += 4) {
      uint4 p[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        p[q] = make_uint4(NONE, NONE, NONE, NONE);
        const int at = first_piece + (c + q) * 64;
        if (c + q < C && at < np) p[q] = load(at);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int j = 0; j < E; ++j) top = fmaxf(top, get(p[q], j));
    }
  }
  if (w == 0) top = fmaxf(top, xo);
  const float own_max = top;
  top = wave_max(top);
  if (lane == 0) wbuf[w] = __float_as_uint(top);
  __syncthreads();
  top = wave_max(lane < NW ? __uint_as_float((uint32_t)wbuf[lane]) : -INFINITY);
  if (top == -INFINITY) {
    if (tid == 0) {
      g.token[n] = -1;
      if (g.logprob) g.logprob[n] = -INFINITY;
    }
    return;
  }
  if (o.greedy) {
    uint32_t at = 0;  // the lowest class with the largest logit, complemented
    each([&](const float (&v)[E], int c) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < E; ++j)
        if (v[j] == top) at = max(at, ~(uint32_t)(c + j));
    });
    at = wave_max(at);
    __syncthreads();
    if (lane == 0) wbuf[w] = at;
    __syncthreads();
    at = wave_max(lane < NW ? (uint32_t)wbuf[lane] : 0u);
    if (tid == 0) {
      g.token[n] = (int32_t)~at;
      if (g.logprob) g.logprob[n] = 0.f;
    }
    return;
  }
  const Row r = row_of(o, top, S);
  // the last kept class: its logit and index; every one that can be drawn at first
  float last = top == INFINITY ? INFINITY : -3.402823466e38f;
  int32_t last_idx = 0x7fffffff;
  auto kept = [&](float v, int c) __attribute__((always_inline)) {
    return v > last || (v == last && c <= last_idx);
  };

  // How far the border is searched: `want` classes (MASS = false), or the classes before which less
  // than `goal` of weight lies.
  uint64_t want = 0;
  double goal = 0.0;
  // bin of the histogram in which `carry` plus the bins up to it reach the border; -1: none does
  auto cross = [&](auto mass, uint64_t carry) __attribute__((always_inline)) -> int {
    constexpr bool MASS = decltype(mass)::value;
    constexpr int PER = BINS / TH;
    uint64_t v[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      v[i] = hist[tid * PER + i];
      sum += v[i];
    }
    uint64_t run = wave_scan(sum, (uint64_t)0, [](uint64_t a, uint64_t b) { return a + b; });
    if (lane == 63) wbuf[w] = run;
    if (tid == 0) found_bin = -1;
    __syncthreads();
    run += carry - sum;
    for (int i = 0; i < w; ++i) run += wbuf[i];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const uint64_t next = run + v[i];
      const bool here = MASS ? (double)run < goal && !((double)next < goal)
                             : run < want && next >= want;
      if (here) {
        found_bin = tid * PER + i;
        found_before = run;
      }
      run = next;
    }
    __syncthreads();
    return found_bin;
  };
  auto clear = [&]() __attribute__((always_inline)) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < BINS / TH; ++i) hist[i * TH + tid] = 0;
    __syncthreads();
  };
  // classes for which in(logit, class), into the list as far as it goes; their number
  auto gather = [&](auto in) __attribute__((always_inline)) -> uint32_t {
    __syncthreads();
    if (tid == 0) {
      count = 0;
      key_lo = 0xffffffffu;
      key_hi = 0;
    }
    __syncthreads();
    uint32_t lo = 0xffffffffu, hi = 0;
    each([&](const float (&v)[E], int c) __attribute__((always_inline)) {
      uint32_t bits = 0;
#pragma unroll
      for (int j = 0; j < E; ++j) bits |= in(v[j], c + j) ? 1u << j : 0u;
      if (__ballot(bits != 0) == 0) return;
      // one place in the list per class, taken by the wave at once
      const uint32_t mine = __popc(bits);
      const uint32_t to = wave_scan(mine, 0u, [](uint32_t a, uint32_t b) { return a + b; });
      uint32_t at = 0;
      if (lane == 63) at = atomicAdd(&count, to);
      at = from_lane(at, 63) + to - mine;
#pragma unroll
      for (int j = 0; j < E; ++j)
        if (bits >> j & 1) {
          const uint32_t k = key_of(v[j]);
          lo = min(lo, k);
          hi = max(hi, k);
          if (at < LIST) list[at] = (uint64_t)k << 32 | (uint32_t)~(c + j);
          ++at;
        }
    });
    lo = ~wave_max(~lo);
    hi = wave_max(hi);
    if (lane == 0) {
      atomicMin(&key_lo, lo);
      atomicMax(&key_hi, hi);
    }
    __syncthreads();
    return count;
  };
  // The border among the m classes of the list, `carry` lying before them (goal < 0: the list is all
  // that is kept); false: it does not reach the border.  By histograms over ever finer ranges of
  // (key, ~index), which no two classes share, until a wave can rank what is left.
  auto rank = [&](auto mass, uint32_t m, uint64_t carry) __attribute__((always_inline)) -> bool {
    constexpr bool MASS = decltype(mass)::value;
    uint64_t lo = (uint64_t)key_lo << 32, hi = (uint64_t)key_hi << 32 | 0xffffffffu;
    if (MASS && goal < 0.0) {
      uint64_t sum = 0;
      for (uint32_t j = tid; j < m; j += TH) sum += r.weight(of_key((uint32_t)(list[j] >> 32)));
      goal = (double)o.top_p * (double)block_sum(sum);
    }
    uint64_t* from = list;
    uint64_t* to = part_of;
    while (m > 64) {
      const int shift = max(0, 64 - __clzll((long long)(hi - lo)) - LOG_BINS);
      clear();
      for (uint32_t j = tid; j < m; j += TH) {
        const uint64_t e = from[j];
        atomicAdd((unsigned long long*)&hist[(hi - e) >> shift],
                  MASS ? (unsigned long long)r.weight(of_key((uint32_t)(e >> 32))) : 1ull);
      }
      if (tid == 0) part_count = 0;
      __syncthreads();
      const int b = cross(mass, carry);
      if (b < 0) return false;
      carry = found_before;
      for (uint32_t j = tid; j < m; j += TH) {
        const uint64_t e = from[j];
        if ((int)((hi - e) >> shift) == b) to[atomicAdd(&part_count, 1u)] = e;
      }
      __syncthreads();
      m = part_count;
      hi -= (uint64_t)b << shift;
      lo = hi - min((1ull << shift) - 1, (unsigned long long)hi);
      uint64_t* const swap = from;
      from = to;
      to = swap;
    }
    if (tid == 0) found = 0;
    __syncthreads();
    if (w == 0) {
      const uint64_t mine = lane < (int)m ? from[lane] : 0;
      const uint64_t q = lane < (int)m ? (MASS ? r.weight(of_key((uint32_t)(mine >> 32))) : 1) : 0;
      uint64_t before = carry;
      for (uint32_t j = 0; j < m; ++j)
        if (from_lane(mine, (int)j) > mine) before += from_lane(q, (int)j);
      if (lane < (int)m && (MASS ? (double)before < goal && !((double)(before + q) < goal)
                                 : before + 1 == want))
        found = mine;
    }
    __syncthreads();
    const uint64_t f = found;
    if (f == 0) return false;
    last = of_key((uint32_t)(f >> 32));
    last_idx = (int32_t)~(uint32_t)f;
    return true;
  };
  // hist[bin(logit, class)] gets the weights, or numbers, of the kept classes for which in(); the
  // weight of the other kept classes that this thread meets is returned
  auto tally = [&](auto mass, auto in, auto bin) __attribute__((always_inline)) -> uint64_t {
    constexpr bool MASS = decltype(mass)::value;
    uint64_t rest = 0;
    clear();
    each([&](const float (&v)[E], int c) __attribute__((always_inline)) {
      bool keep[E], any = false;
#pragma unroll
      for (int j = 0; j < E; ++j) {
        keep[j] = kept(v[j], c + j);
        any |= keep[j];
      }
      if (__ballot(any) == 0) return;
      uint64_t q[E];
#pragma unroll
      for (int j = 0; j < E; ++j) q[j] = MASS ? r.weight(v[j]) : 1;
#pragma unroll
      for (int j = 0; j < E; ++j) {
        const bool on = keep[j] && in(v[j], c + j);
        if (on) atomicAdd((unsigned long long*)&hist[bin(v[j], c + j)], (unsigned long long)q[j]);
        if (MASS) rest += keep[j] && !on ? q[j] : 0;
      }
    });
    __syncthreads();
    return rest;
  };
  // the border among the kept classes with keys in [lo, hi], `carry` lying before them
  auto refine = [&](auto mass, uint32_t lo, uint32_t hi, uint32_t m, uint64_t carry)
      __attribute__((always_inline)) {
    constexpr bool MASS = decltype(mass)::value;
    while (m > LIST && lo != hi) {
      const int shift = max(0, 32 - __clz(hi - lo) - LOG_BINS);
      const float f_lo = of_key(lo), f_hi = of_key(hi);
      tally(mass, [&](float v, int) { return v >= f_lo && v <= f_hi; },
            [&](float v, int) { return (hi - key_of(v)) >> shift; });
      const int b = cross(mass, carry);
      carry = found_before;
      const uint32_t upper = hi - ((uint32_t)b << shift), wide = (1u << shift) - 1;
      const uint32_t lower = max(lo, upper - min(wide, upper));
      const float g_lo = of_key(lower), g_hi = of_key(upper);
      m = gather([&](float v, int c) { return v >= g_lo && v <= g_hi && kept(v, c); });
      lo = key_lo;
      hi = key_hi;
    }
    if (m > LIST) {
      // one key more often than the list goes: how many of them, then the last one's index
      if (MASS) {
        const uint64_t each_w = r.weight(of_key(lo));
        uint64_t more = (uint64_t)((goal - (double)carry) / (double)each_w);
        while (more > 0 && !((double)(carry + (more - 1) * each_w) < goal)) --more;
        while ((double)(carry + more * each_w) < goal) ++more;
        want = more;
      } else {
        want -= carry;
      }
      constexpr int SHIFT = 18 - LOG_BINS;  // (2^SHIFT <= LIST)
      const float tie = of_key(lo);
      tally(std::false_type(), [&](float v, int) { return v == tie; },
            [&](float, int c) { return c >> SHIFT; });
      const int b = cross(std::false_type(), 0);
      carry = found_before;
      m = gather([&](float v, int c) { return v == tie && c >> SHIFT == b && kept(v, c); });
      rank(std::false_type(), m, carry);
      return;
    }
    rank(mass, m, carry);
  };
  // step of x in which a logit lies
  const float steps = fminf((float)BINS / STEPS_OVER * (float)(r.iu * (LN2_HI + LN2_LO)), 3e38f);
  auto step_of = [&](float v) __attribute__((always_inline)) {
    return (int)fminf((top - v) * steps, (float)(BINS - 1));
  };
  // by the histogram over x
  auto search = [&](auto mass) __attribute__((always_inline)) {
    constexpr bool MASS = decltype(mass)::value;
    float from = -INFINITY;
    if (MASS) {
      // Classes lighter than (1 - top_p) / V of the total hold less than 1 - top_p of it together:
      // the border lies above them, and they only count for the total (an addition to LDS costs
      // more than the weight).  The total is at least the threads' largest kept weights together.
      // That share is 4 steps of the weights or more (V <= 2^18, 1 - top_p >= 2^-24), which roundings
      // raise by 0.75: below exp(-0.21) of it none passes it.
      const uint64_t some = block_sum(kept(own_max, 0x7fffffff) ? r.weight(own_max) : 0);
      const float part = (float)((1.0 - (double)o.top_p) * (double)some / V *
                                 __builtin_amdgcn_ldexp(1.0, -S));
      const double cut = (double)top + (double)o.tau * ((double)__logf(part) - 0.22);
      from = (float)(cut - fabs(cut) * 0x1p-22);
      if (!(from <= top)) from = -INFINITY;
      __syncthreads();
    }
    const uint64_t rest = tally(mass, [&](float v, int) { return v >= from; },
                                [&](float v, int) { return step_of(v); });
    if (MASS) {
      uint64_t sum = rest;
#pragma unroll
      for (int i = 0; i < BINS / TH; ++i) sum += hist[i * TH + tid];
      goal = (double)o.top_p * (double)block_sum(sum);
      __syncthreads();
    }
    const int b = cross(mass, 0);
    if (b < 0) return;  // (nothing is cut off)
    const uint64_t carry = found_before;
    const uint32_t m = gather([&](float v, int c) { return step_of(v) == b && kept(v, c) && v >= from; });
    refine(mass, key_lo, key_hi, m, carry);
  };
  // The kept classes that reach about the q-th largest of the groups' maxima, into the list: at
  // least q and few more, unless there are fewer than q in all.
  auto gather_top = [&](int q) __attribute__((always_inline)) -> uint32_t {
    constexpr int PER = TH / GROUPS;
    static_assert(__alignof__(part_of) >= alignof(uint4) && sizeof(part_of) >= 4 * GROUPS,
                  "the keys are read as uint4");
    uint32_t* keys = reinterpret_cast<uint32_t*>(part_of);
    uint32_t k = key_of(own_max);
#pragma unroll
    for (int d = 1; d < PER; d <<= 1) k = max(k, (uint32_t)__shfl_xor(k, d));
    __syncthreads();
    if (tid % PER == 0) keys[tid / PER] = k;
    __syncthreads();
    if (w == 0) {
      // the upper 16 bits of the q-th largest, bit by bit
      const uint4 four = reinterpret_cast<const uint4*>(keys)[lane];
      uint32_t bound = 0;
      for (uint32_t bit = 0x80000000u; bit >= 0x10000u; bit >>= 1) {
        const uint32_t c = bound | bit;
        const int reach = __popcll(__ballot(four.x >= c)) + __popcll(__ballot(four.y >= c)) +
                          __popcll(__ballot(four.z >= c)) + __popcll(__ballot(four.w >= c));
        if (reach >= q) bound = c;
      }
      if (lane == 0) found = bound;
    }
    __syncthreads();
    const uint32_t f = (uint32_t)found;
    const float bound = f >= 0x00800000u ? of_key(f) : -3.402823466e38f;
    return gather([&](float v, int c) { return v >= bound && kept(v, c); });
  };
  // weights of the kept classes: of each stretch, and of the class beside the pieces
  uint64_t odd_share = 0;
  auto share = [&](float v, int c) __attribute__((always_inline)) -> uint64_t {
    const uint64_t q = r.weight(v);
    return kept(v, c) ? q : 0;
  };
  auto weigh = [&]() __attribute__((always_inline)) -> uint64_t {  // their sum, in this wave
    uint64_t all = 0;
    for (int q = 0; q < rounds; ++q) {
      const int first_piece = (q * NW + w) * 64 * C;
      uint64_t sum = 0;
      for (int c = 0; c < C && first_piece + c * 64 < np; ++c) {
        const int v = first_piece + c * 64 + lane;
        uint4 p = make_uint4(NONE, NONE, NONE, NONE);
        if (v < np) p = load(v);
        bool any = false;
#pragma unroll
        for (int j = 0; j < E; ++j) any |= kept(get(p, j), lead + v * E + j);
        if (__ballot(any) == 0) continue;
#pragma unroll
        for (int j = 0; j < E; ++j) sum += share(get(p, j), lead + v * E + j);
      }
      sum = wave_sum(sum);
      if (lane == 0) chunk[q * NW + w] = sum;
      all += sum;
    }
    if (w == 0) {
      odd_share = odd < V ? share(xo, odd) : 0;
      all += wave_sum(odd_share);
    }
    return all;
  };

  bool few = false;  // the kept classes fit the list
  if (o.top_k > 0) {
    want = (uint64_t)o.top_k;
    if (o.top_k <= GROUPS) {
      const uint32_t m = gather_top(o.top_k);
      if (m <= LIST) {
        few = true;
        if (m >= (uint32_t)o.top_k) rank(std::false_type(), m, 0);  // (else all that can be drawn)
      }
    }
    if (!few) search(std::false_type());
  }
  if (o.top_p < 1.f) {
    if (few) {
      goal = -1.0;
      const uint32_t m = gather(kept);
      rank(std::true_type(), m, 0);
    } else {
      search(std::true_type());
    }
  }
  if (o.min_p > 0.f) {
    const float bound = of_key(least_key(o, top));
    if (bound > last) {
      last = bound;
      last_idx = 0x7fffffff;
    }
  }

  // The draw: the kept classes' weights in order of their indices, which is the classes before the
  // first piece, the stretches, the classes behind the last piece.
  weigh();
  auto add = [](uint64_t a, uint64_t b) { return a + b; };
  __syncthreads();
  if (w != 0) return;
  // one wave draws: where the running sum passes u times the total, first among the stretches
  const uint64_t beside = wave_scan(odd_share, (uint64_t)0, add);
  const uint64_t lead_sum = wave_sum(tid < lead ? odd_share : (uint64_t)0);
  const int chunks = rounds * NW;
  const uint64_t c0 = 2 * lane < chunks ? chunk[2 * lane] : 0;
  const uint64_t c1 = 2 * lane + 1 < chunks ? chunk[2 * lane + 1] : 0;
  const uint64_t upto = wave_scan(c0 + c1, (uint64_t)0, add);
  const uint64_t pieces = from_lane(upto, 63), mass = pieces + from_lane(beside, 63);
  const double aim = (double)o.u * (double)mass;
  auto passes = [&](uint64_t before, uint64_t own) __attribute__((always_inline)) {
    return !((double)before > aim) && (double)(before + own) > aim;
  };
  int token = -1;
  float logit = 0.f;
  auto drawn = [&](bool hit, int c, float v) __attribute__((always_inline)) {
    const uint64_t b = __ballot(hit);
    if (b) {
      const int l = __ffsll((unsigned long long)b) - 1;
      token = (int)from_lane((uint32_t)c, l);
      logit = from_lane(v, l);
    }
  };
  drawn(odd < V && passes(beside - odd_share + (tid < lead ? (uint64_t)0 : pieces), odd_share), odd, xo);
  uint64_t run = lead_sum + upto - c0 - c1;  // before this lane's first stretch
  const bool in0 = passes(run, c0), in1 = passes(run + c0, c1);
  const uint64_t hits = __ballot(in0 || in1);
  if (hits) {
    const int l = __ffsll((unsigned long long)hits) - 1;
    const int at = (int)from_lane((uint32_t)(2 * lane + (in0 ? 0 : 1)), l);
    run = from_lane(in0 ? run : run + c0, l);
    for (int c = 0; c < C && token < 0; ++c) {
      const int v = at * 64 * C + c * 64 + lane;
      uint64_t q[E], sum = 0;
      uint4 p = make_uint4(0, 0, 0, 0);
      if (v < np) p = load(v);
#pragma unroll
      for (int j = 0; j < E; ++j) {
        q[j] = v < np ? share(get(p, j), lead + v * E + j) : 0;
        sum += q[j];
      }
      const uint64_t to = wave_scan(sum, (uint64_t)0, add);
      uint64_t before = run + to - sum;
      bool hit = false;
      int which = 0;
      float z = 0.f;
#pragma unroll
      for (int j = 0; j < E; ++j) {
        if (passes(before, q[j])) {
          hit = true;
          which = lead + v * E + j;
          z = get(p, j);
        }
        before += q[j];
      }
      drawn(hit, which, z);
      run += from_lane(to, 63);
    }
  }
  if (lane == 0) {
    g.token[n] = token;
    if (g.logprob) g.logprob[n] = logprob_of(r, logit, mass);
  }
}

template <class T, int W>
hipError_t run_small(const SampleGeo& g, int S, const T* logits, hipStream_t s) {
  constexpr int64_t most = MAX_THREADS / 256;
  for (int64_t first = 0; first < g.N; first += most * (256 / W)) {
    const int64_t blocks = (g.N - first + 256 / W - 1) / (256 / W);
    k_sample_small<T, W><<<(unsigned)(blocks < most ? blocks : most), 256, 0, s>>>(g, first, S, logits);
  }
  return hipGetLastError();
}
template <class T, int TH>
hipError_t run_rows(const SampleGeo& g, int S, const T* logits, hipStream_t s) {
  constexpr int64_t most = MAX_THREADS / TH;
  for (int64_t first = 0; first < g.N; first += most)
    k_sample<T, TH><<<(unsigned)(g.N - first < most ? g.N - first : most), TH, 0, s>>>(g, first, S, logits);
  return hipGetLastError();
}

}  // namespace

template <class T>
hipError_t launch_sample(const SampleGeo& g, const T* logits, hipStream_t s) {
  int bits = 0;
  while ((1 << bits) < g.V) ++bits;
  const int S = 62 - bits < 51 ? 62 - bits : 51;
  if (g.V <= 8) return run_small<T, 8>(g, S, logits, s);
  if (g.V <= 16) return run_small<T, 16>(g, S, logits, s);
  if (g.V <= 32) return run_small<T, 32>(g, S, logits, s);
  if (g.V <= 64) return run_small<T, 64>(g, S, logits, s);
  // many threads to a row that has pieces for them, while there are CUs without a row, or with one
  // more turn where rows are long.  us with 1,024 threads / with 256, temperature alone and top-p:
  //   1 x 5,000 float32   7.7 / 9.2, 16 / 20       64 x 131,072 bfloat16   50 / 83, 122 / 238
  //   256 x 5,000         8.3 / 11,  17 / 22       512 x 131,072           113 / 127, 264 / 330
  //   384 x 5,000         13 / 13,   29 / 26       512 x 12,000 float32    17 / 21, 42 / 50
  //   1,024 x 5,000       22 / 17,   56 / 34       1,024 x 50,021 bf16     112 / 88, 260 / 206
  const int np = g.V / (16 / (int)sizeof(T));
  if (np > 512 && g.N <= (np > 2048 ? 512 : 256)) return run_rows<T, 1024>(g, S, logits, s);
  return run_rows<T, 256>(g, S, logits, s);
}
template hipError_t launch_sample<float>(const SampleGeo&, const float*, hipStream_t);
template hipError_t launch_sample<bf16>(const SampleGeo&, const bf16*, hipStream_t);

}  // namespace tfm
