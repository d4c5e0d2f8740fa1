// Embedding rows and their gradient (declarations in vocab.h).
//
// Forward: a copy with a factor, in pieces of 16 bytes where the rows allow it.
// Backward: dtable[v] = scale sum_{n: id_n = v} dout_n.  The positions are sorted by id (stable
// radix sort, so equal ids keep their order), and the sorted positions are cut into pieces of equal
// length whatever the ids are: every group of lanes adds up the rows of its piece in registers and
// writes a sum where the id changes.  Sums that cross a piece's border are joined in LDS within a
// workgroup and through float32 rows in the workspace between workgroups, in order, so the result
// does not depend on timing.  Each gradient row is written once, by the one group that completes
// it; rows of ids that do not occur are zeroed by further workgroups of the same launch.
//
// Both are bound by HBM where the rows are many: 327,680 ids into rows of 192 bfloat16 elements take
// 26 us forward (as a copy of the 127 MB; the 0.4 MB table is read from the caches) and 54 us
// backward (floor 26.6), of which the sums are 29 (4.4 TB/s), the sort 20 and the join 5: the sort
// moves little, but is three launches of a few dependent steps each.  40,000 ids into 50,021 rows of
// 1,024 elements backward: 92 us (floor 60), the sums 64 of it (4.5 TB/s).  16 rows of 2,048 forward:
// 3 us in the kernel, 11 with the host's call.  Sums by floating-point atomics would not be
// reproducible and would read and write the gradient once per id.
// Adding to those 327,680 rows takes 43 us, writing float32 rows 51 and adding to them 97, at the
// copy's rate too; float32 rows from a bfloat16 table take 102 to write (floor 53: a lane's eight
// elements are two stores, each of which leaves gaps).
#include "mfma.h"
#include "vocab.h"

#include <hip/hip_runtime.h>

#include <algorithm>

namespace tfm {
namespace {

// ---- rows as vectors --------------------------------------------------------------------------
// VEC elements of type T at p as floats; p is aligned to min(16, VEC sizeof(T)) bytes.
template <int VEC>
__device__ __forceinline__ void ldv(const float* p, float* v) {
  if constexpr (VEC >= 4) {
#pragma unroll
    for (int i = 0; i < VEC / 4; ++i) {
      const float4 a = reinterpret_cast<const float4*>(p)[i];
      v[4 * i] = a.x; v[4 * i + 1] = a.y; v[4 * i + 2] = a.z; v[4 * i + 3] = a.w;
    }
  } else if constexpr (VEC == 2) {
    const float2 a = *reinterpret_cast<const float2*>(p);
    v[0] = a.x; v[1] = a.y;
  } else {
    v[0] = *p;
  }
}
__device__ __forceinline__ void halves(uint32_t u, float* v) {
  v[0] = __uint_as_float(u << 16);
  v[1] = __uint_as_float(u & 0xffff0000u);
}
template <int VEC>
__device__ __forceinline__ void ldv(const bf16* p, float* v) {
  if constexpr (VEC == 8) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    halves(u.x, v); halves(u.y, v + 2); halves(u.z, v + 4); halves(u.w, v + 6);
  } else if constexpr (VEC == 4) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    halves(u.x, v); halves(u.y, v + 2);
  } else if constexpr (VEC == 2) {
    halves(*reinterpret_cast<const uint32_t*>(p), v);
  } else {
    v[0] = ld(p);
  }
}
template <int VEC>
__device__ __forceinline__ void stv(float* p, const float* v) {
  if constexpr (VEC >= 4) {
#pragma unroll
    for (int i = 0; i < VEC / 4; ++i)
      reinterpret_cast<float4*>(p)[i] =
          make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
  } else if constexpr (VEC == 2) {
    *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
  } else {
    *p = v[0];
  }
}
__device__ __forceinline__ uint32_t pair_of(const float* v) { return pack2(v[0], v[1]); }
template <int VEC>
__device__ __forceinline__ void stv(bf16* p, const float* v) {
  if constexpr (VEC == 8)
    *reinterpret_cast<uint4*>(p) = make_uint4(pair_of(v), pair_of(v + 2), pair_of(v + 4), pair_of(v + 6));
  else if constexpr (VEC == 4)
    *reinterpret_cast<uint2*>(p) = make_uint2(pair_of(v), pair_of(v + 2));
  else if constexpr (VEC == 2)
    *reinterpret_cast<uint32_t*>(p) = pair_of(v);
  else
    st(p, v[0]);
}

// The same past the caches, for outputs too large for them to hold until they are read.
template <int VEC, bool PAST, class T>
__device__ __forceinline__ void put(T* p, const float* v) {
  if constexpr (PAST && VEC * sizeof(T) >= 16) {
    if constexpr (sizeof(T) == 2) {
      const u32x4 q = {pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])};
      __builtin_nontemporal_store(q, reinterpret_cast<u32x4*>(p));
    } else {
#pragma unroll
      for (int i = 0; i < VEC / 4; ++i) {
        const f32x4 q = {v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
        __builtin_nontemporal_store(q, reinterpret_cast<f32x4*>(p) + i);
      }
    }
  } else {
    stv<VEC>(p, v);
  }
}

// Vectors that start at any element, which global loads and stores take as they come.
template <int VEC>
__device__ __forceinline__ void ld_any(const float* p, float* v) {
  __builtin_memcpy(v, p, 4 * VEC);
}
template <int VEC>
__device__ __forceinline__ void ld_any(const bf16* p, float* v) {
  if constexpr (VEC == 1) {
    v[0] = ld(p);
  } else {
    uint32_t u[VEC / 2];
    __builtin_memcpy(u, p, 2 * VEC);
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) halves(u[i], v + 2 * i);
  }
}
template <int VEC, bool PAST>
__device__ __forceinline__ void st_any(float* p, const float* v) {
  if constexpr (PAST && VEC == 4) {
    typedef f32x4 f32x4_any __attribute__((aligned(4)));
    __builtin_nontemporal_store(f32x4{v[0], v[1], v[2], v[3]}, reinterpret_cast<f32x4_any*>(p));
  } else {
    __builtin_memcpy(p, v, 4 * VEC);
  }
}

// First element of the activations' row n.  n < 2^27, so n / d is the upper half of n (2^64 / d + 1)
// for every d > 1.
__device__ __forceinline__ uint32_t div_by(uint32_t n, uint64_t m) {
  return m ? (uint32_t)__umul64hi(n, m) : n;
}
__device__ __forceinline__ int64_t row_at(const EmbedGeo& g, uint32_t n) {
  const uint32_t ij = div_by(n, g.m2), k = n - ij * (uint32_t)g.n2;
  const uint32_t i = div_by(ij, g.m1), j = ij - i * (uint32_t)g.n1;
  return i * g.stride[0] + j * g.stride[1] + k * g.stride[2];
}

// ---- forward -----------------------------------------------------------------------------------
// The rows' vectors one after another, L to a row, R of them in flight per thread.  A workgroup
// first looks up the ids and places of its rows, once per row and not once per vector: that is some
// 60 cycles of integer products, as much as moving a vector.  ml: as EmbedGeo's m1 for L (exact
// here too: fewer than 2^43 vectors, L <= 2^16); ms: 2^32 / L + 1 (exact below 2^11 for L <= 2^10).
template <class TT, class TO, int VEC, int R, bool ADD, bool PAST>
__global__ __launch_bounds__(256) void k_embed_fwd(EmbedGeo g, uint32_t L, uint64_t ml, uint32_t ms,
                                                   const int32_t* __restrict__ ids,
                                                   const TT* __restrict__ table,
                                                   TO* __restrict__ out) {
  constexpr int SPAN = 256 * R;  // vectors of a workgroup
  __shared__ int64_t place[SPAN + 1];
  __shared__ int32_t rid[SPAN + 1];
  const int64_t total = g.N * L;
  for (int64_t i0 = (int64_t)blockIdx.x * SPAN; i0 < total; i0 += (int64_t)gridDim.x * SPAN) {
    const int64_t nb = ml ? (int64_t)__umul64hi((uint64_t)i0, ml) : i0;
    const uint32_t cb = (uint32_t)(i0 - nb * L);
    const uint32_t rows = (cb + SPAN - 1) / L + 1;  // that the span touches
    __syncthreads();
    for (uint32_t r = threadIdx.x; r < rows; r += 256) {
      const int64_t n = nb + r;
      rid[r] = n < g.N ? ids[n] : -1;
      place[r] = n < g.N ? row_at(g, (uint32_t)n) : -1;
    }
    __syncthreads();
    int32_t id[R];
    float v[R][VEC], o[R][VEC];
    int64_t p[R];
    uint32_t c[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const uint32_t at = cb + r * 256 + threadIdx.x;
      const uint32_t dn = L == 1 ? at : L > 1024 ? at >= L : __umulhi(at, ms);
      c[r] = (at - dn * L) * VEC;
      id[r] = rid[dn];
      p[r] = place[dn];
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const bool here = (uint32_t)id[r] < (uint32_t)g.V;
      ldv<VEC>(table + (int64_t)(here ? id[r] : 0) * g.E + c[r], v[r]);
      if (ADD && here) ldv<VEC>(out + p[r] + c[r], o[r]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const bool here = (uint32_t)id[r] < (uint32_t)g.V;
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        v[r][i] = here ? g.scale * v[r][i] : 0.f;
        if (ADD) v[r][i] += o[r][i];
      }
      if (p[r] >= 0 && (here || !ADD)) put<VEC, PAST>(out + p[r] + c[r], v[r]);
    }
  }
}

// ---- sort by id ---------------------------------------------------------------------------------
// Keys: the id, V for an absent one (they end up behind every id); .x of a pair, .y being the
// position, so that a pass moves each with one 8-byte store.  Radix passes from the lowest digit up,
// of at most 10 bits: the counts of a digit fit in LDS once per wave.  A workgroup ranks a tile of
// keys, each wave a contiguous part of it, 64 at a time, by ballots over the digit's bits.  Bound by
// latency: 327,680 keys of one digit 5.5 us to count, 3.6 to scan, 11 to place.
constexpr int SORT_T = 512;   // threads
constexpr int SORT_R = 4;     // keys of a thread: a tile's rounds are ranked one after another
constexpr int SORT_TILE = SORT_T * SORT_R;
constexpr int SMALL_R = 8;    // of the sort in one workgroup
constexpr int SMALL_TILE = SORT_T * SMALL_R;
constexpr int SORT_W = SORT_T / 64;
constexpr int SORT_BITS = 10;               // widest digit
constexpr int SORT_FUSE = 24;               // workgroups up to which each sums the counts before it
                                            // itself: one launch less (2^10 counts from 24 others
                                            // are read in about the time of a launch)

struct SortGeo {
  int32_t N, V, nblk;
  int32_t shift, bits;     // digit of the pass
};

// Key and position at place n: of the ids in the first pass, of the last one's pairs then.
__device__ __forceinline__ int2 pair_at(const SortGeo& s, const int32_t* ids, int n) {
  const int32_t k = ids[n];
  return make_int2((uint32_t)k >= (uint32_t)s.V ? s.V : k, n);
}
__device__ __forceinline__ int2 pair_at(const SortGeo&, const int2* pairs, int n) { return pairs[n]; }

// Counts of the digits of every tile: cnt[workgroup][digit], or cnt[digit][workgroup] for the scan.
template <class S>
__global__ __launch_bounds__(SORT_T) void k_sort_count(SortGeo s, const S* __restrict__ src,
                                                       uint32_t* __restrict__ cnt) {
  __shared__ uint32_t h[1 << SORT_BITS];
  const int bins = 1 << s.bits;
  for (int d = threadIdx.x; d < bins; d += SORT_T) h[d] = 0;
  __syncthreads();
  const int n0 = blockIdx.x * SORT_TILE;
#pragma unroll
  for (int r = 0; r < SORT_R; ++r) {
    const int n = n0 + r * SORT_T + threadIdx.x;
    if (n < s.N) atomicAdd(&h[pair_at(s, src, n).x >> s.shift & (bins - 1)], 1u);
  }
  __syncthreads();
  for (int d = threadIdx.x; d < bins; d += SORT_T)
    cnt[s.nblk > SORT_FUSE ? (int64_t)d * s.nblk + blockIdx.x : (int64_t)blockIdx.x * bins + d] = h[d];
}

// One wave per digit: its counts become the number of earlier equal digits, its total goes behind.
__global__ __launch_bounds__(256) void k_sort_scan(SortGeo s, uint32_t* __restrict__ cnt) {
  const int bins = 1 << s.bits, lane = threadIdx.x & 63;
  const int d = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (d >= bins) return;
  uint32_t* c = cnt + (int64_t)d * s.nblk;
  uint32_t run = 0;
  for (int b = 0; b < s.nblk; b += 64) {
    const uint32_t mine = b + lane < s.nblk ? c[b + lane] : 0;
    uint32_t inc = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t q = __shfl_up(inc, o);
      if (lane >= o) inc += q;
    }
    if (b + lane < s.nblk) c[b + lane] = run + inc - mine;
    run += __shfl(inc, 63);
  }
  if (lane == 0) cnt[(int64_t)bins * s.nblk + d] = run;
}

// Exclusive scan of v[0 .. 2^bits) by the workgroup; v and buf in LDS.
__device__ __forceinline__ void scan_bins(uint32_t* v, int bins, uint32_t* buf) {
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  constexpr int PER = (1 << SORT_BITS) / SORT_T;
  uint32_t x[PER], sum = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    x[i] = t * PER + i < bins ? v[t * PER + i] : 0;
    sum += x[i];
  }
  uint32_t inc = sum;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t q = __shfl_up(inc, o);
    if (lane >= o) inc += q;
  }
  if (lane == 63) buf[w] = inc;
  __syncthreads();
  uint32_t run = inc - sum;
  for (int i = 0; i < w; ++i) run += buf[i];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (t * PER + i < bins) v[t * PER + i] = run;
    run += x[i];
  }
  __syncthreads();
}

// Ranks of the workgroup's keys among its keys of the same digit, in order: wave w holds keys
// w R 64 + r 64 + lane.  wcnt[w][digit] ends as the number of such keys of earlier waves.
// digit < 0: no key.
template <int R>
__device__ __forceinline__ void rank_tile(const int (&digit)[R], int bits,
                                          uint32_t (*wcnt)[1 << SORT_BITS],
                                          uint32_t (&rank)[R], uint32_t* total) {
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, bins = 1 << bits;
  for (int d = t; d < bins; d += SORT_T)
#pragma unroll
    for (int i = 0; i < SORT_W; ++i) wcnt[i][d] = 0;
  __syncthreads();
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const bool on = digit[r] >= 0;
    uint64_t same = __ballot(on);  // lanes that hold the same digit
    for (int b = 0; b < bits; ++b) {
      const bool bit = digit[r] >> b & 1;
      const uint64_t m = __ballot(bit);
      same &= bit ? m : ~m;
    }
    const uint64_t below = same & ((1ull << lane) - 1);
    volatile uint32_t* c = &wcnt[w][on ? digit[r] : 0];
    const uint32_t at = *c;
    rank[r] = at + __popcll(below);
    __builtin_amdgcn_wave_barrier();
    if (on && below == 0) *c = at + __popcll(same);
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
  for (int d = t; d < bins; d += SORT_T) {
    uint32_t run = 0;
#pragma unroll
    for (int i = 0; i < SORT_W; ++i) {
      const uint32_t q = wcnt[i][d];
      wcnt[i][d] = run;
      run += q;
    }
    if (total) total[d] = run;
  }
  __syncthreads();
}

// One pass: the pairs to their places.
template <class S>
__global__ __launch_bounds__(SORT_T) void k_sort_place(SortGeo s, const S* __restrict__ src,
                                                       const uint32_t* __restrict__ cnt,
                                                       int2* __restrict__ dst) {
  __shared__ uint32_t wcnt[SORT_W][1 << SORT_BITS];
  __shared__ uint32_t base[1 << SORT_BITS];
  __shared__ uint32_t before[1 << SORT_BITS];
  __shared__ uint32_t buf[SORT_W];
  const int t = threadIdx.x, lane = t & 63, w = t >> 6, bins = 1 << s.bits;
  // first place of every digit, and how many of its keys earlier workgroups hold
  for (int d = t; d < bins; d += SORT_T) {
    if (s.nblk > SORT_FUSE) {
      base[d] = cnt[(int64_t)bins * s.nblk + d];
      before[d] = cnt[(int64_t)d * s.nblk + blockIdx.x];
    } else {
      uint32_t all = 0, mine = 0;
      for (int b0 = 0; b0 < s.nblk; b0 += 8) {
        uint32_t q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = cnt[(b0 + i < s.nblk ? b0 + i : b0) * bins + d];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (b0 + i < (int)blockIdx.x) mine += q[i];
          if (b0 + i < s.nblk) all += q[i];
        }
      }
      base[d] = all;
      before[d] = mine;
    }
  }
  scan_bins(base, bins, buf);
  const int n0 = blockIdx.x * SORT_TILE + w * SORT_R * 64 + lane;
  int2 pair[SORT_R];
  int digit[SORT_R];
#pragma unroll
  for (int r = 0; r < SORT_R; ++r) {
    const int n = n0 + r * 64;
    pair[r] = n < s.N ? pair_at(s, src, n) : make_int2(0, 0);
    digit[r] = n < s.N ? pair[r].x >> s.shift & (bins - 1) : -1;
  }
  uint32_t rank[SORT_R];
  rank_tile(digit, s.bits, wcnt, rank, nullptr);
#pragma unroll
  for (int r = 0; r < SORT_R; ++r)
    if (digit[r] >= 0)
      dst[base[digit[r]] + before[digit[r]] + wcnt[w][digit[r]] + rank[r]] = pair[r];
}

// The whole sort of at most one tile in one workgroup.
__global__ __launch_bounds__(SORT_T) void k_sort_small(SortGeo s, int passes,
                                                       const int32_t* __restrict__ ids,
                                                       int2* __restrict__ dst) {
  __shared__ uint32_t wcnt[SORT_W][1 << SORT_BITS];
  __shared__ uint32_t base[1 << SORT_BITS];
  __shared__ uint32_t buf[SORT_W];
  __shared__ int32_t keys[SMALL_TILE];
  __shared__ uint16_t from[SMALL_TILE];
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  const int n0 = w * SMALL_R * 64 + lane;
  int32_t key[SMALL_R];
  int digit[SMALL_R], pos[SMALL_R];
#pragma unroll
  for (int r = 0; r < SMALL_R; ++r) {
    const int n = n0 + r * 64;
    key[r] = n < s.N ? pair_at(s, ids, n).x : 0;
    pos[r] = n;
  }
  for (int p = 0; p < passes; ++p) {
    const int shift = p * s.bits, bins = 1 << s.bits;
#pragma unroll
    for (int r = 0; r < SMALL_R; ++r)
      digit[r] = n0 + r * 64 < s.N ? key[r] >> shift & (bins - 1) : -1;
    uint32_t rank[SMALL_R];
    rank_tile(digit, s.bits, wcnt, rank, base);
    scan_bins(base, bins, buf);
#pragma unroll
    for (int r = 0; r < SMALL_R; ++r) {
      if (digit[r] < 0) continue;
      const uint32_t at = base[digit[r]] + wcnt[w][digit[r]] + rank[r];
      keys[at] = key[r];
      from[at] = (uint16_t)pos[r];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < SMALL_R; ++r) {
      const int n = n0 + r * 64;
      if (n < s.N) {
        key[r] = keys[n];
        pos[r] = from[n];
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int r = 0; r < SMALL_R; ++r) {
    const int n = n0 + r * 64;
    if (n < s.N) dst[n] = make_int2(key[r], pos[r]);
  }
}

// ---- sums ----------------------------------------------------------------------------------------
constexpr int SUM_T = 256;
constexpr int SUM_U = 8;       // rows in flight per group
constexpr int FILL_ROWS = 64;  // gradient rows that a zeroing workgroup looks after

struct SumGeo {
  int64_t N;
  int32_t piece;   // sorted positions of a group, a multiple of SUM_U
  int32_t nblk;    // workgroups that add; the others zero
  int32_t W;       // lanes of a group
  int32_t slices;  // grid.y
  int32_t past;    // zeroed rows go past the caches
};

// Sorted positions [a, b) of group k of workgroup blk.
__device__ __forceinline__ int64_t piece_at(const SumGeo& s, int64_t blk, int k, int groups) {
  const int64_t a = (blk * groups + k) * (int64_t)s.piece;
  return a < s.N ? a : s.N;
}

template <int VEC, bool ADD>
__device__ __forceinline__ void write_row(const EmbedGeo& g, float* dtable, int32_t v, int c,
                                          const float* acc) {
  float* o = dtable + (int64_t)v * g.E + c;
  float x[VEC];
  if (ADD) ld_any<VEC>(o, x);
#pragma unroll
  for (int i = 0; i < VEC; ++i) x[i] = ADD ? x[i] + g.scale * acc[i] : g.scale * acc[i];
  st_any<VEC, false>(o, x);
}

// Lane i's value within each group of W lanes.
template <int W>
__device__ __forceinline__ int32_t from_lane(int32_t v, int i) {
  if constexpr (W == 64) return __builtin_amdgcn_readlane(v, i);
  else return __shfl(v, i, W);
}
template <int W>
__device__ __forceinline__ int64_t from_lane(int64_t v, int i) {
  const uint32_t lo = (uint32_t)from_lane<W>((int32_t)(uint32_t)v, i);
  const uint32_t hi = (uint32_t)from_lane<W>((int32_t)(v >> 32), i);
  return (int64_t)((uint64_t)hi << 32 | lo);
}

// Zeroes the rows whose ids do not occur, FILL_ROWS at a time, of the workgroup's slice.
template <int VEC, int W>
__device__ __forceinline__ void zero_rows(const EmbedGeo& g, const SumGeo& s,
                                          const int2* sorted, float* dtable, int* present) {
  constexpr int Z = VEC < 4 ? VEC : 4;  // a store instruction covers its stretch without gaps
  const float zero[Z] = {};
  const int64_t step = (int64_t)((int)gridDim.x - s.nblk) * FILL_ROWS;
  for (int64_t v0 = (int64_t)((int)blockIdx.x - s.nblk) * FILL_ROWS; v0 < g.V; v0 += step) {
    __syncthreads();
    if (threadIdx.x < FILL_ROWS) {
      const int64_t v = v0 + threadIdx.x;
      int64_t lo = 0, hi = s.N;  // first sorted position with a key >= v
      while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (sorted[mid].x < v) lo = mid + 1;
        else hi = mid;
      }
      present[threadIdx.x] = v >= g.V || (lo < s.N && sorted[lo].x == v);
    }
    __syncthreads();
    for (int r = threadIdx.x / W; r < FILL_ROWS; r += SUM_T / W) {
      if (present[r]) continue;
      float* o = dtable + (v0 + r) * g.E;
#pragma unroll
      for (int q = 0; q < VEC / Z; ++q) {
        const int c = (int)blockIdx.y * W * VEC + (q * W + threadIdx.x % W) * Z;
        if (c >= g.E) continue;
        if (s.past) st_any<Z, true>(o + c, zero);
        else st_any<Z, false>(o + c, zero);
      }
    }
  }
}

// Each group of W lanes adds the rows of its piece of the sorted positions, SUM_U loads ahead, in
// float32.  Bound by HBM: reads every row of dout once and writes every row of dtable once.
// part: [nblk][2][E]: what a workgroup's positions add to a run that began in an earlier one, and
// to a run that begins here and goes on in the next.
template <class TO, int VEC, int W, bool ADD>
__global__ __launch_bounds__(SUM_T) void k_embed_sum(EmbedGeo g, SumGeo s,
                                                     const int2* __restrict__ sorted,
                                                     const TO* __restrict__ dout,
                                                     float* __restrict__ dtable,
                                                     float* __restrict__ part) {
  constexpr int K = SUM_T / W;  // groups
  // per group: its share of a run that came in, and of one that goes out
  __shared__ float edge[K][2][W * VEC];
  __shared__ int32_t okey[K];   // key that goes out of the group, -1: none
  __shared__ int32_t through[K];  // the key that came in goes out as well
  __shared__ int present[FILL_ROWS];
  if ((int)blockIdx.x >= s.nblk) {
    zero_rows<VEC, W>(g, s, sorted, dtable, present);
    return;
  }
  const int k = threadIdx.x / W, lane = threadIdx.x % W;
  const int c = ((int)blockIdx.y * W + lane) * VEC;
  const bool live = c < g.E;
  const int64_t a = piece_at(s, blockIdx.x, k, K), b = piece_at(s, blockIdx.x, k + 1, K);
  float acc[VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) acc[i] = 0.f;
  int32_t cur = -1;
  const bool head = a > 0 && a < b && sorted[a - 1].x == sorted[a].x;
  bool came_in = head;  // the current run began in an earlier piece
  const TO* d = dout + (live ? c : 0);
  // a lane per position for its key and its row's place, the next W positions a step ahead
  int2 next = make_int2(g.V, 0);
  if (a + lane < b) next = sorted[a + lane];
  bool end = a >= b;
  for (int64_t t0 = a; !end; t0 += W) {
    const int32_t key_w = next.x;
    const int64_t row_w = row_at(g, (uint32_t)next.y);
    next = make_int2(g.V, 0);
    if (t0 + W + lane < b) next = sorted[t0 + W + lane];
    const int left = b - t0 < W ? (int)(b - t0) : W;
    for (int t = 0; t < left && !end; t += SUM_U) {
      int32_t key[SUM_U];
      float x[SUM_U][VEC];
#pragma unroll
      for (int i = 0; i < SUM_U; ++i) {
        key[i] = from_lane<W>(key_w, t + i);
        const int64_t at = from_lane<W>(row_w, t + i < left ? t + i : 0);
        ld_any<VEC>(d + at, x[i]);
      }
#pragma unroll
      for (int i = 0; i < SUM_U; ++i) {
        if (key[i] != cur) {
          if (cur >= 0) {
            if (came_in) {
#pragma unroll
              for (int j = 0; j < VEC; ++j) edge[k][0][lane * VEC + j] = acc[j];
            } else if (live) {
              write_row<VEC, ADD>(g, dtable, cur, c, acc);
            }
            came_in = false;
          }
#pragma unroll
          for (int j = 0; j < VEC; ++j) acc[j] = 0.f;
          cur = key[i] < g.V ? key[i] : -1;
        }
        if (cur >= 0) {
#pragma unroll
          for (int j = 0; j < VEC; ++j) acc[j] += x[i][j];
        } else {
          end = true;  // only absent ids follow
          break;
        }
      }
    }
    end |= t0 + W >= b;
  }
  // the last run: complete, or going on in the next piece
  const bool goes_on = cur >= 0 && b < s.N && sorted[b].x == cur;
  if (cur >= 0) {
    if (came_in || goes_on) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) edge[k][came_in ? 0 : 1][lane * VEC + j] = acc[j];
    } else if (live) {
      write_row<VEC, ADD>(g, dtable, cur, c, acc);
    }
  }
  if (lane == 0) {
    okey[k] = goes_on && !came_in ? cur : -1;
    through[k] = goes_on && came_in;
  }
  __syncthreads();
  // join inside the workgroup: each group the run that leaves it first, group 0 also the run that
  // came into the workgroup
  for (int from = k == 0 ? -1 : k; from <= k; ++from) {
    int32_t run;
    int at;
    if (from < 0) {
      if (!head || sorted[a].x >= g.V) continue;
      run = sorted[a].x;
      at = 0;
#pragma unroll
      for (int j = 0; j < VEC; ++j) acc[j] = edge[0][0][lane * VEC + j];
    } else {
      if (okey[k] < 0) continue;
      run = okey[k];
      at = k + 1;
#pragma unroll
      for (int j = 0; j < VEC; ++j) acc[j] = edge[k][1][lane * VEC + j];
      if (at < K) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) acc[j] += edge[at][0][lane * VEC + j];
      }
    }
    while (at < K && through[at]) {
      if (++at < K) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) acc[j] += edge[at][0][lane * VEC + j];
      }
    }
    if (!live) continue;
    if (from < 0) stv<VEC>(part + ((int64_t)blockIdx.x * 2 + 0) * g.E + c, acc);
    else if (at == K) stv<VEC>(part + ((int64_t)blockIdx.x * 2 + 1) * g.E + c, acc);
    else write_row<VEC, ADD>(g, dtable, run, c, acc);
  }
}

// Runs that cross workgroups: the workgroup in which one begins adds the later ones' shares, its
// groups every K-th of them, and then the groups' sums in order.
template <int VEC, int W, bool ADD>
__global__ __launch_bounds__(SUM_T) void k_embed_join(EmbedGeo g, SumGeo s,
                                                      const int2* __restrict__ sorted,
                                                      const float* __restrict__ part,
                                                      float* __restrict__ dtable) {
  constexpr int K = SUM_T / W;
  __shared__ float sums[K][W * VEC];
  const int64_t a = piece_at(s, blockIdx.x, 0, K), b = piece_at(s, blockIdx.x, K, K);
  if (b >= s.N) return;
  const int32_t run = sorted[b - 1].x;
  if (run >= g.V || sorted[b].x != run || (a > 0 && sorted[a - 1].x == run)) return;
  const int k = threadIdx.x / W, lane = threadIdx.x % W;
  const int c = ((int)blockIdx.y * W + lane) * VEC;
  const bool live = c < g.E;
  float acc[VEC], x[4][VEC];
#pragma unroll
  for (int i = 0; i < VEC; ++i) acc[i] = 0.f;
  bool more = true;
  for (int64_t j0 = blockIdx.x + 1 + k; more && j0 < s.nblk; j0 += 4 * K) {
    bool in[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t j = j0 + q * K, jj = j < s.nblk ? j : s.nblk - 1;
      in[q] = j < s.nblk && sorted[piece_at(s, jj, 0, K)].x == run;
      ldv<VEC>(part + (jj * 2) * g.E + (live ? c : 0), x[q]);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (in[q]) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[i] += x[q][i];
      }
    }
    more = in[3];
  }
#pragma unroll
  for (int i = 0; i < VEC; ++i) sums[k][lane * VEC + i] = acc[i];
  __syncthreads();
  if (k != 0 || !live) return;
  ldv<VEC>(part + ((int64_t)blockIdx.x * 2 + 1) * g.E + c, acc);
  for (int q = 0; q < K; ++q)
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc[i] += sums[q][lane * VEC + i];
  write_row<VEC, ADD>(g, dtable, run, c, acc);
}

// ---- host side -----------------------------------------------------------------------------------

int sort_passes(int32_t V, int* bits) {
  int total = 0;
  while (total < 31 && (V >> total) != 0) ++total;
  const int passes = (total + SORT_BITS - 1) / SORT_BITS;
  *bits = (total + passes - 1) / passes;
  return passes;
}

// Lanes of a group: the row in vectors of VEC elements, at most a wave; a power of two >= 8.
int group_width(int32_t E, int vec) {
  int W = 8;
  while (W < 64 && W * vec < E) W *= 2;
  return W;
}

// Widest vector that rows of E elements divide into, of at most `most` elements.
int row_vec(int32_t E, int most) {
  while (E % most) most /= 2;
  return most;
}

// How the sorted positions are cut into groups and workgroups, and so the order of every sum, goes by
// N, E and the type of the rows (`most` elements to 16 bytes) alone: rows and gradients that start on
// smaller boundaries are read and written in the same vectors.
// Sorted positions per group: enough groups for 16 waves on each of 256 CUs, which hide the row
// loads' latency; at least 16, so that the edges' share of the traffic stays small.
SumGeo sum_geo(const EmbedGeo& g, int most) {
  SumGeo s;
  s.N = g.N;
  const int vec = row_vec(g.E, most);
  s.W = group_width(g.E, vec);
  s.slices = (g.E + s.W * vec - 1) / (s.W * vec);
  const double groups = 4096.0 * (64 / s.W) / s.slices;
  int64_t piece = (int64_t)((double)g.N / (groups > 1.0 ? groups : 1.0)) + 1;
  if (piece < 16) piece = 16;
  piece = (piece + SUM_U - 1) / SUM_U * SUM_U;
  s.piece = (int32_t)piece;
  const int64_t per = piece * (SUM_T / s.W);
  s.nblk = (int32_t)((g.N + per - 1) / per);
  // (as for the forward: 50,021 rows of 1,024, most of them zeros, 96 -> 92 us)
  s.past = (int64_t)g.V * g.E * 4 > (32 << 20);
  return s;
}

struct EmbedWs {
  size_t pair[2], cnt, part, total;
};
EmbedWs embed_ws(const EmbedGeo& g) {
  EmbedWs w;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += (bytes + 255) / 256 * 256;
    return at;
  };
  int bits;
  const int passes = sort_passes(g.V, &bits);
  const size_t nblk = g.N <= SMALL_TILE ? 1 : (size_t)((g.N + SORT_TILE - 1) / SORT_TILE);
  w.pair[0] = take((size_t)g.N * 8);
  w.pair[1] = take(nblk > 1 && passes > 1 ? (size_t)g.N * 8 : 0);
  w.cnt = take(nblk > 1 ? ((nblk + 1) << bits) * 4 : 0);
  // rows of either type
  const size_t blocks = (size_t)std::max(sum_geo(g, 4).nblk, sum_geo(g, 8).nblk);
  w.part = take(blocks * 2 * (size_t)g.E * 4);
  w.total = off > 0 ? off : 256;
  return w;
}

bool fits(const void* p, size_t bytes) { return (uintptr_t)p % bytes == 0; }

// Widest vector, in elements of at most 16 bytes of T, at which every row starts.
template <class T>
int vec_of(const EmbedGeo& g, const T* rows) {
  int vec = 16 / (int)sizeof(T);
  auto ok = [&](int v) {
    if (g.E % v || !fits(rows, v * sizeof(T))) return false;
    for (int i = 0; i < 3; ++i)
      if (g.stride[i] % v) return false;
    return true;
  };
  while (vec > 1 && !ok(vec)) vec /= 2;
  return vec;
}

template <class TT, class TO, int VEC, bool ADD>
hipError_t fwd_vec(const EmbedGeo& g, const int32_t* ids, const TT* table, TO* out, hipStream_t s) {
  const uint32_t L = (uint32_t)(g.E / VEC);
  const uint64_t ml = L > 1 ? ~uint64_t(0) / L + 1 : 0;
  const uint32_t ms = L > 1 ? (uint32_t)((uint64_t(1) << 32) / L + 1) : 0;
  const int64_t total = g.N * L;
  // an output that the 8 L2 caches of 4 MB cannot hold goes past them: 16 x 1,024 x 20 rows of 192
  // (126 MB) take 25.7 us against 32.8
  const bool past = g.N * g.E * (int64_t)sizeof(TO) > (32 << 20);
  // four vectors in flight per thread once that leaves every CU its eight workgroups
  const bool many = total >= 4 * 256 * 8 * 256 || past;
  int64_t blocks = (total + (many ? 1023 : 255)) / (many ? 1024 : 256);
  if (blocks > (1 << 23)) blocks = 1 << 23;
#define RUN(R, P) \
  k_embed_fwd<TT, TO, VEC, R, ADD, P><<<(unsigned)blocks, 256, 0, s>>>(g, L, ml, ms, ids, table, out)
  if (past) RUN(4, true);
  else if (many) RUN(4, false);
  else RUN(1, false);
#undef RUN
  return hipGetLastError();
}

template <class TO, int VEC, int W, bool ADD>
hipError_t bwd_run(const EmbedGeo& g, const SumGeo& s, const int2* sorted, const TO* dout, float* dtable, float* part, hipStream_t st) {
  // (a launch holds fewer than 2^32 threads)
  const int64_t most = MAX_THREADS / SUM_T / s.slices - s.nblk, want = (g.V + FILL_ROWS - 1) / FILL_ROWS;
  const unsigned fill = ADD ? 0u : (unsigned)(want < most ? want : most);
  const dim3 grid((unsigned)s.nblk + fill, (unsigned)s.slices);
  k_embed_sum<TO, VEC, W, ADD><<<grid, SUM_T, 0, st>>>(g, s, sorted, dout, dtable, part);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || s.nblk < 2) return e;
  k_embed_join<VEC, W, ADD><<<dim3((unsigned)s.nblk, (unsigned)s.slices), SUM_T, 0, st>>>(
      g, s, sorted, part, dtable);
  return hipGetLastError();
}

template <class TO, int VEC>
hipError_t bwd_vec(const EmbedGeo& g, const int2* sorted, const TO* dout,
                   float* dtable, float* part, int add, hipStream_t st) {
  const SumGeo s = sum_geo(g, 16 / (int)sizeof(TO));
#define RUN(X)                                                                               \
  case X:                                                                                    \
    return add ? bwd_run<TO, VEC, X, true>(g, s, sorted, dout, dtable, part, st)         \
               : bwd_run<TO, VEC, X, false>(g, s, sorted, dout, dtable, part, st);
  switch (s.W) { RUN(8) RUN(16) RUN(32) RUN(64) }
#undef RUN
  return hipErrorInvalidValue;
}

}  // namespace

template <class TT, class TO>
hipError_t launch_embed_fwd(const EmbedGeo& g, const int32_t* ids, const TT* table, TO* out,
                            int accumulate, hipStream_t s) {
  // vectors of 4 or 8 elements: 16 bytes of the narrower type where both sides start on them
  int vec = vec_of(g, out);
  constexpr int most = sizeof(TT) < sizeof(TO) ? 16 / sizeof(TT) : 16 / sizeof(TO);
  if (vec == 4 && most == 8 && sizeof(TO) == 4) {
    bool ok = g.E % 8 == 0 && fits(table, 16);
    if (ok) vec = 8;
  }
  while (vec > 1 && !fits(table, vec * sizeof(TT) < 16 ? vec * sizeof(TT) : 16)) vec /= 2;
#define RUN(X)                                                                               \
  case X:                                                                                    \
    return accumulate ? fwd_vec<TT, TO, X, true>(g, ids, table, out, s)                        \
                      : fwd_vec<TT, TO, X, false>(g, ids, table, out, s);
  switch (vec) { RUN(1) RUN(2) RUN(4) RUN(8) }
#undef RUN
  return hipErrorInvalidValue;
}

size_t embed_bwd_bytes(const EmbedGeo& g) { return embed_ws(g).total; }

template <class TO>
hipError_t launch_embed_bwd(const EmbedGeo& g, const int32_t* ids, const TO* dout, float* dtable,
                            int accumulate, void* ws, hipStream_t st) {
  const EmbedWs W = embed_ws(g);
  char* w = (char*)ws;
  SortGeo s;
  s.N = (int32_t)g.N;
  s.V = g.V;
  s.nblk = g.N <= SMALL_TILE ? 1 : (int32_t)((g.N + SORT_TILE - 1) / SORT_TILE);
  const int passes = sort_passes(g.V, &s.bits);
  hipError_t e = hipSuccess;
  int2* sorted = (int2*)(w + W.pair[0]);
  uint32_t* cnt = (uint32_t*)(w + W.cnt);
  s.shift = 0;
  if (s.nblk == 1 && g.N > 0) {
    k_sort_small<<<1, SORT_T, 0, st>>>(s, passes, ids, sorted);
    e = hipGetLastError();
  }
  for (int p = 0; s.nblk > 1 && p < passes && e == hipSuccess; ++p) {
    s.shift = p * s.bits;
    const int2* from = sorted;
    sorted = (int2*)(w + W.pair[p & 1]);
    if (p == 0) k_sort_count<<<s.nblk, SORT_T, 0, st>>>(s, ids, cnt);
    else k_sort_count<<<s.nblk, SORT_T, 0, st>>>(s, from, cnt);
    if (s.nblk > SORT_FUSE) k_sort_scan<<<((1 << s.bits) + 3) / 4, 256, 0, st>>>(s, cnt);
    if (p == 0) k_sort_place<<<s.nblk, SORT_T, 0, st>>>(s, ids, cnt, sorted);
    else k_sort_place<<<s.nblk, SORT_T, 0, st>>>(s, from, cnt, sorted);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return e;
  float* part = (float*)(w + W.part);
  switch (row_vec(g.E, 16 / (int)sizeof(TO))) {
    case 1: return bwd_vec<TO, 1>(g, sorted, dout, dtable, part, accumulate, st);
    case 2: return bwd_vec<TO, 2>(g, sorted, dout, dtable, part, accumulate, st);
    case 4: return bwd_vec<TO, 4>(g, sorted, dout, dtable, part, accumulate, st);
    case 8:
      if constexpr (sizeof(TO) == 2)
        return bwd_vec<TO, 8>(g, sorted, dout, dtable, part, accumulate, st);
  }
  return hipErrorInvalidValue;
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
