// Attention of query rows over a pool of e4m3 codes (declarations in cache8.h).
//
// The query rows of all heads that share a key/value head of a sequence are the columns of one
// problem, row i and head j of G at column i G + j: one row of a group of heads and many rows of one
// head are the same work.  A wave takes 16 QB columns and tiles of 64 rows of the cache (keys, below):
//
//   S^T = K Q^T     v_mfma_f32_16x16x32_bf16: codes are exact as bfloat16, the block's power goes into
//                   the scores' factor
//   p = 2^(S c - ref), online, ref a running reference of the exponent per column
//   O^T += V^T P^T  v_mfma_f32_16x16x32_f16: codes times 2^(power - unit) are exact as half, unit the
//                   largest power that the wave's columns have seen so far
//
// The weights' sum is of the unrounded ones, in float32 (as one more product, 1 P^T, it would cost fewer
// cycles, but the rounded weights put lse off by up to 2^-11).
// Row m of the t-th of the tile's four 16-row products is key 16 (m / 4) + 4 t + m % 4, so that a lane's
// 16 scores are those of 16 keys in a row: one block's, since pages are multiples of 16, and in the
// order in which the lane reads 16 bytes of V^T.  Nothing moves between lanes, and codes go from memory
// to registers without LDS (but see staged()).
//
// p is held as half with 2^8 in front: 2^-11 of each weight, and 2^-33 of the largest where half has no
// more bits (bfloat16 would have doubled the output's own rounding error).  The reference is looked at
// only where a lane's weights sum to more than half can hold, the first tile's among them, whose
// reference is the lowest float: then it becomes its column's largest score, the column's sums are
// rescaled and the tile weighed again.  With the largest score as reference 16 weights sum to at most
// 2^12, and a later one may be up to 2^7 of it, so that this is rare, and other tiles need no maximum.
// Values are held with 2^7 in front: exact unless their block is 2^22 below the largest, 2^-40 of that
// one's largest code then.  Float32 queries are three bfloat16 parts (24 bits) and their weights two
// halves.
//
// Few columns (SPLIT): the four waves of a workgroup share the columns and take turns over the tiles;
// many: each wave has columns of its own.  A tile's keys are read while the one before it is weighed
// and summed, its values from then on.  Where the workgroups are too few the keys are split over more
// of them, and a second launch joins their sums.
//
// Bounds and figures.  Few columns: the codes' bytes; 64 sequences of 1 to 16,384 rows, one row of 32
// heads on 8, d = 128: 207 us, 5.2 TB/s.  Many columns: vector instructions, 436 of a wave and tile at
// d = 32 and 64 columns (64 exponentials at two issue slots each, scores to weights, codes to
// bfloat16 and half), 32 matrix instructions beside them; 1616 sequences of 768 rows, 256 rows of 6
// heads, d = 32: 439 us, 560 TFLOP/s, the vector units 83 to 96 % busy.  (Of the 436, 64 are the sum
// and 64 the scores' factor and reference: attn_item.hip, which sums on the matrix cores and starts its
// accumulators at the reference, needs neither and is the faster on bfloat16 keys.)
#include <float.h>

#include "cache8.h"
#include "mfma.h"

namespace tfm {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int KT = 64;              // keys per tile
constexpr int P_BIAS = 8, V_BIAS = 7;  // weights and values are held times 2 to these
constexpr float P_MOST = 61440.f;       // a lane's 16 weights may sum to this, and half holds each
constexpr int V_GAP = 20;               // powers of two by which blocks of a product may differ

// 8 codes (two dwords) as bfloat16 and, times a power of two, as half.
__device__ __forceinline__ bf16x8 codes_bf16(uint32_t lo, uint32_t hi) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
  bf16x8 r = {a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
  return r;
}
__device__ __forceinline__ f16x8 codes_f16(uint32_t lo, uint32_t hi, float two) {  // times two
  const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, two, false);
  const f16x2 b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, two, true);
  const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, two, false);
  const f16x2 d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, two, true);
  f16x8 r = {a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
  return r;
}
// Bytes of w that are NaN codes, as 0x80.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
  return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
}

// A float as three bfloat16 whose sum it is.
__device__ __forceinline__ void three_parts(float x, uint16_t* p) {
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    p[i] = f2bf(x);
    x -= bf2f(p[i]);
  }
}

// Operand of S^T: CH products over 32 channels (one over 16 at D = 16).
template <int D>
struct KQ {
  static constexpr int CH = D / 32;
  typedef bf16x8 frag;
  static __device__ __forceinline__ f32x4 mma(const frag& k, const frag& q, const f32x4& s) {
    return mfma16(k, q, s);
  }
};
template <>
struct KQ<16> {
  static constexpr int CH = 1;
  typedef s16x4 frag;
  static __device__ __forceinline__ f32x4 mma(const frag& k, const frag& q, const f32x4& s) {
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(k, q, s, 0, 0, 0);
  }
};

// What a lane reads of a tile: keys' codes; values' codes, the bytes of both powers of its 16 keys'
// block, and whether there is one.
template <int D>
struct Keys {
  uint32_t k[4][D / 16];
  uint32_t power;
  bool here;
};
template <int D>
struct Values {
  uint4 v[D / 16];
};

// Whether tiles go through LDS, for all four waves: where registers hold no tile beside 32 columns' sums.
// Many columns at d = 128, bf16, pages of 64 and more (8 sequences of 1000 rows, 2000 keys, 16 heads):
// 349 us with 16 columns and the tile in registers, 190 us staged with 32.  With keys in two pieces, the
// tile in registers was the faster one at d = 64 (122 us, 139 us staged; now, in one piece, 107), as with
// pages under 64 (218 us, 246 us).
template <int D, bool F32, int QB, bool SPLIT>
constexpr bool staged() { return !SPLIT && D == 128 && !F32 && QB == 2; }
// Waves per SIMD that the registers of a kernel leave room for.  (Three at D <= 32: 476 us for the 1616
// sequences above with two, 442 with three, queries in LDS for it; with pages under 64 two registers do
// not fit and go through scratch.)
template <int D, bool F32, int QB, bool SPLIT>
constexpr int waves() { return D <= 32 && QB == 4 ? 3 : D == 128 && QB == 2 && SPLIT ? 1 : 2; }

template <int D, class T, int QB, bool SPLIT, bool UNI>
__global__ __launch_bounds__(256, (waves<D, sizeof(T) == 4, QB, SPLIT>())) void k_cache8_attend(
    Cache8Attend a, const T* q, T* out /* may be q */, float* __restrict__ part,
    float* __restrict__ part_ml, uint32_t prob0, uint32_t nprob, int coltiles, int splits, int chunk,
    int wide) {
  constexpr int DB = D / 16, CH = KQ<D>::CH, KW = D / 16;  // KW: dwords of a key per lane
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int NQ = F32 ? 3 : 1, NP = F32 ? 2 : 1;
  constexpr bool STAGE = staged<D, F32, QB, SPLIT>();  // tiles go through LDS, for all four waves
  typedef typename KQ<D>::frag QF;
  const Cache8Geo& g = a.g;
  const int lane = threadIdx.x & 63, wave = wave_id(), c = lane & 15, lg = lane >> 4;
  // Workgroups in order of (split, problem, columns): with the splits of a problem side by side those
  // behind the last keys fell on the same XCDs, as their number is often a power of two (64 sequences
  // of 1 to 16,384 rows: 244 us instead of 211).
  const uint32_t rest = blockIdx.x / (uint32_t)coltiles, sp = rest / nprob;
  const int ct = blockIdx.x - rest * coltiles;
  const uint32_t prob = prob0 + rest - sp * nprob;  // below 2^31, as B L heads is
  const uint32_t bq = prob / (uint32_t)g.heads;
  const int64_t b = bq;
  const int kh = prob - bq * g.heads, G = a.heads / g.heads;
  const int rows = a.n_rows ? min(max(a.n_rows[b], 0), a.L) : a.L;
  const int ncols = rows * G;
  const int col0 = (SPLIT ? ct : ct * 4 + wave) * 16 * QB;
  if ((STAGE ? ct * 64 * QB : col0) >= ncols) return;  // (a wave without columns reads tiles for others)
  const int k0 = (int)sp * chunk, shift = g.shift;
  // The table's entries from ebase (a multiple of 64) on, one a lane, and the 64 after them: a tile's
  // pages come from these registers, so that none waits for its page's number.  (Read before the
  // sequence's length is there.)
  auto entries = [&](int e0) {
    return g.max_pages > 0 ? cache8_page(g, b, min(e0 + lane, g.max_pages - 1)) : -1;
  };
  int ebase = ((k0 + (SPLIT ? wave * KT : 0)) >> shift) & ~63;
  int near = entries(ebase), far = entries(ebase + 64);
  const int len = min(max(a.lens[b], 0), a.max_rows);
  if (splits > 1 && k0 >= len) return;

  // the keys that each column sees
  auto row_of = [&](int col) { return (int)((uint32_t)col / (uint32_t)G); };
  int upto[QB], lo = len, hi = len, hi_all = len;  // hi_all: of the workgroup's columns
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) upto[qb] = len;
  if (a.causal) {
    lo = 0x7fffffff;
    hi = 0;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      upto[qb] = min(max(len - rows + row_of(min(col0 + qb * 16 + c, ncols - 1)) + 1, 0), len);
      lo = min(lo, upto[qb]);
      hi = max(hi, upto[qb]);
    }
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {
      lo = min(lo, __shfl_xor(lo, o, 64));
      hi = max(hi, __shfl_xor(hi, o, 64));
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    hi = __builtin_amdgcn_readfirstlane(hi);
    hi_all = min(max(len - rows + row_of(min((ct + 1) * 64 * QB, ncols) - 1) + 1, 0), len);
  }

  // the queries' operands, in LDS at D >= 64, where registers are short
  constexpr bool QLDS = D >= 64 || (D == 32 && QB == 4);
  constexpr int QBYTES = QLDS ? NQ * QB * CH * 1024 : 0;  // of a wave
  constexpr int OBYTES = SPLIT ? 4 * 16 * QB * (D + 4) * 4 : 0;
  constexpr int TBYTES = 128 * D;  // of a tile: 64 rows of keys, then D rows of values
  constexpr int LBYTES = STAGE ? 4 * QBYTES + 2 * TBYTES : 4 * QBYTES > OBYTES ? 4 * QBYTES : OBYTES;
  __shared__ __attribute__((aligned(16))) uint8_t lds[LBYTES > 0 ? LBYTES : 16];
  QF qf[NQ][QB][CH];  // (dead behind the stores below where it is in LDS)
  uint8_t* ql = lds + wave * QBYTES + lane * 16;
  const bool neg = a.scale_log2 < 0;
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    if (STAGE && col0 >= ncols) break;  // (the last column is another wave's, which may write it in place)
    const int col = min(col0 + qb * 16 + c, ncols - 1), i = row_of(col), h = kh * G + col - i * G;
    const T* p = q + b * a.sq[0] + i * a.sq[1] + h * a.sq[2] + lg * (D / 4);
    uint16_t e[NQ][D / 4];
    if (wide) {
      constexpr int V = D / 4 * sizeof(T) / 8;  // 8-byte pieces
      uint2 u[V];
#pragma unroll
      for (int j = 0; j < V; ++j) u[j] = reinterpret_cast<const uint2*>(p)[j];
      const T* x = reinterpret_cast<const T*>(u);
#pragma unroll
      for (int j = 0; j < D / 4; ++j) {
        if constexpr (F32) {
          uint16_t t[3];
          three_parts(x[j], t);
#pragma unroll
          for (int n = 0; n < 3; ++n) e[n][j] = t[n];
        } else {
          e[0][j] = x[j];
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < D / 4; ++j) {
        if constexpr (F32) {
          uint16_t t[3];
          three_parts(p[j], t);
#pragma unroll
          for (int n = 0; n < 3; ++n) e[n][j] = t[n];
        } else {
          e[0][j] = p[j];
        }
      }
    }
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
      for (int ch = 0; ch < CH; ++ch) {
        uint16_t f[sizeof(QF) / 2];
#pragma unroll
        for (int j = 0; j < (int)sizeof(QF) / 2; ++j)
          f[j] = (uint16_t)(e[n][ch * 8 + j] ^ (neg ? 0x8000u : 0u));
        __builtin_memcpy(&qf[n][qb][ch], f, sizeof(QF));
        if constexpr (QLDS)
          *reinterpret_cast<QF*>(ql + ((n * QB + qb) * CH + ch) * 1024) = qf[n][qb][ch];
      }
  }
  auto query_frag = [&](int n, int qb, int ch) {
    if constexpr (QLDS) return *reinterpret_cast<const QF*>(ql + ((n * QB + qb) * CH + ch) * 1024);
    return qf[n][qb][ch];
  };
  const float scale = fabsf(a.scale_log2);

  const int kend = STAGE && col0 >= ncols ? k0 : min(splits > 1 ? k0 + chunk : len, hi);
  constexpr int STEP = SPLIT ? 4 * KT : KT;
  const int page = g.page;
  const int64_t hd = (int64_t)g.heads * page * D;  // bytes of a page
  // the pages of the keys 16 (c / 4) .. and 16 lg .. of a tile (UNI: one page, the same in every lane)
  const int gk = UNI ? 0 : c >> 2, gv = UNI ? 0 : lg;
  auto look = [&](int t0) {  // before pid_of of tile t0
    if ((t0 >> shift) - ebase < 64) return;  // (a step is 16 entries at most)
    ebase += 64;
    near = far;
    far = entries(ebase + 64);
  };
  auto pid_of = [&](int t0, int grp) {
    const int e = ((t0 + 16 * grp) >> shift) - ebase;
    return UNI ? __builtin_amdgcn_readlane(near, e) : __shfl(near, e, 64);
  };
  auto load_k = [&](Keys<D>& x, int t0, int pk, int pv) {
    x.here = pv >= 0;
    pk = max(pk, 0);
    pv = max(pv, 0);
    const int ck = c >> 2;
    const uint8_t* kb;
    if constexpr (UNI)
      kb = g.keys + pk * hd + ((int64_t)kh * page + (t0 & (page - 1))) * D +
           (16 * ck + (c & 3)) * D + lg * (D / 4);
    else
      kb = g.keys + pk * hd + ((int64_t)kh * page + ((t0 + 16 * ck) & (page - 1)) + (c & 3)) * D +
           lg * (D / 4);
    x.power = *reinterpret_cast<const uint16_t*>(g.powers + ((int64_t)pv * g.heads + kh) * 2);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      if constexpr (D == 16) {
        x.k[t][0] = *reinterpret_cast<const uint32_t*>(kb + 4 * t * D);
      } else if constexpr (D == 32) {
        const uint2 u = *reinterpret_cast<const uint2*>(kb + 4 * t * D);
        x.k[t][0] = u.x; x.k[t][1] = u.y;
      } else {
#pragma unroll
        for (int w = 0; w < KW; w += 4) {
          const uint4 u = *reinterpret_cast<const uint4*>(kb + 4 * t * D + 4 * w);
          x.k[t][w] = u.x; x.k[t][w + 1] = u.y; x.k[t][w + 2] = u.z; x.k[t][w + 3] = u.w;
        }
      }
    }
  };
  auto load_v = [&](Values<D>& x, int t0, int pv) {
    pv = max(pv, 0);
    const uint8_t* vb = g.values + pv * hd + (int64_t)kh * page * D +
                        (UNI ? (t0 & (page - 1)) + 16 * lg : (t0 + 16 * lg) & (page - 1)) + c * page;
#pragma unroll
    for (int db = 0; db < DB; ++db)
      x.v[db] = *reinterpret_cast<const uint4*>(vb + (int64_t)db * 16 * page);
  };

  float ref[QB], lsum[QB];  // lsum: of the lane's own keys
  f32x4 oacc[DB][QB];
  int unit = CACHE8_E_MIN;
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    ref[qb] = -FLT_MAX;
    lsum[qb] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) oacc[db][qb] = zero4();
  }
  // A staged tile: each thread brings two 16-byte pieces of keys and two of values.  Pieces are swapped
  // within their row by bits of the row's number, so that the eight rows of which eight lanes read a
  // piece lie in different banks.
  int cur = 0;  // the buffer that is read
  auto swap_k = [](int row) { return (row & 3) | (row >> 2 & 4); };
  uint4 kp0, kp1, vp0, vp1;
  uint32_t gpower = 0;
  bool ghere = false;
  auto bring = [&](int t0) {
    look(t0);
    const int p = pid_of(t0, 0);
    const int64_t pg = max(p, 0);
    const int row = threadIdx.x >> 3, j = threadIdx.x & 7, d = threadIdx.x >> 2, u = threadIdx.x & 3;
    const uint8_t* kt = g.keys + pg * hd + ((int64_t)kh * page + (t0 & (page - 1)) + row) * D + 16 * j;
    const uint8_t* vt = g.values + pg * hd + ((int64_t)kh * D + d) * page + (t0 & (page - 1)) + 16 * u;
    kp0 = *reinterpret_cast<const uint4*>(kt);
    vp0 = *reinterpret_cast<const uint4*>(vt);
    kp1 = *reinterpret_cast<const uint4*>(kt + 32 * D);
    vp1 = *reinterpret_cast<const uint4*>(vt + 64 * (int64_t)page);
    ghere = p >= 0;
    gpower = *reinterpret_cast<const uint16_t*>(g.powers + (pg * g.heads + kh) * 2);
  };
  auto put = [&](int buf) {
    uint8_t* at = lds + 4 * QBYTES + buf * TBYTES;
    const int row = threadIdx.x >> 3, j = threadIdx.x & 7, d = threadIdx.x >> 2, u = threadIdx.x & 3;
    uint8_t* vt = at + 64 * D + d * 64 + 16 * (u ^ (d >> 1 & 3));  // (row 64 on swaps alike)
    *reinterpret_cast<uint4*>(at + row * D + 16 * (j ^ swap_k(row))) = kp0;
    *reinterpret_cast<uint4*>(vt) = vp0;
    *reinterpret_cast<uint4*>(at + (row + 32) * D + 16 * (j ^ swap_k(row))) = kp1;
    *reinterpret_cast<uint4*>(vt + 64 * 64) = vp1;
  };
  // 16 codes of key t of the lane's four (piece w of its channels), and of values' row block db.
  const int krow = 16 * (c >> 2) + (c & 3);
  auto staged_keys = [&](int t, int w) {
    return *reinterpret_cast<const uint4*>(lds + 4 * QBYTES + cur * TBYTES + (krow + 4 * t) * D +
                                           16 * ((lg * (D / 64) + w) ^ swap_k(krow)));
  };
  auto staged_values = [&](int db) {
    return *reinterpret_cast<const uint4*>(lds + 4 * QBYTES + cur * TBYTES + 64 * D +
                                           (16 * db + c) * 64 + 16 * (lg ^ (c >> 1 & 3)));
  };
  auto key_frag = [&](const Keys<D>& x, int t, int ch) {
    QF kf;
    if constexpr (D == 16) {
      const bf16x8 w = codes_bf16(x.k[t][0], 0);
      __builtin_memcpy(&kf, &w, 8);
    } else {
      kf = codes_bf16(x.k[t][2 * ch], x.k[t][2 * ch + 1]);
    }
    return kf;
  };
  // Scores of block qb (in place) to its weights.
  bool first = true;  // (then the reference says nothing yet)
  auto weigh = [&](f32x4* s, int qb, float cs, int t0, bool partial, bool here, f16x8 (*pf)[2]) {
    if (partial) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (t0 + 16 * lg + 4 * t + i >= upto[qb] || !here) s[t][i] = -INFINITY;
    }
    auto weights = [&]() {
      const float off = (float)P_BIAS - ref[qb];
      float sum[2];
#pragma unroll
      for (int kc = 0; kc < 2; ++kc)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float p = exp2_hw(fmaf(s[2 * kc + j / 4][j % 4], cs, off));
          sum[kc] = j ? sum[kc] + p : p;
          const _Float16 h = (_Float16)p;
          pf[0][kc][j] = h;
          if constexpr (NP == 2) pf[1][kc][j] = (_Float16)(p - (float)h);
        }
      return sum[0] + sum[1];
    };
    float sum = INFINITY;
    if (!first) sum = weights();
    if (__any(!(sum <= P_MOST))) {
      float mx = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3]));
#pragma unroll
      for (int t = 1; t < 4; ++t)
        mx = fmaxf(mx, fmaxf(fmaxf(s[t][0], s[t][1]), fmaxf(s[t][2], s[t][3])));
      // (of the columns that need it alone: a row's bits do not depend on the rows beside it)
      const bool more = rows4_max(sum <= P_MOST ? 0.f : 1.f) > 0.f;
      mx = rows4_max(mx * cs);
      const float now = more ? fmaxf(ref[qb], mx) : ref[qb];
      if (!first) {
        const float corr = exp2_hw(ref[qb] - now);
        lsum[qb] *= corr;
#pragma unroll
        for (int db = 0; db < DB; ++db) oacc[db][qb] *= corr;
      }
      ref[qb] = now;
      sum = weights();
    }
    lsum[qb] += sum;
  };
  // Scores of a tile, weights, sums, of the keys of one group of lanes (only) or of all (-1).
  // codes_read: called once the registers of the keys (and, at D <= 32, of the values) are free.
  auto compute = [&](Keys<D>& x, Values<D>& y, int t0, int only, auto codes_read) {
    const int ek = power_byte(x.power & 0xff), ev = power_byte(x.power >> 8);
    const bool here = x.here && (UNI || only < 0 || lg == only);
    // (not 0, by which a masked score, -inf, could not be multiplied; a score of queries below 2^112 is
    // below 2^128 before it, so that the least factor adds at most 2^-21 to an exponent)
    const float cs = fmaxf(scale * two_to(ek - 127), 0x1p-149f);
    const bool partial = t0 + KT > lo || __any(!here);
    int top = ev;
    bool dirty = false;  // a staged tile has NaN codes that its readers leave out
    auto clean = [](uint32_t* w) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t m = nan_bytes(w[j]);
        w[j] &= ~(m | (m - (m >> 7)));  // 0x80 to 0xff
      }
    };
    auto values_of = [&](int db) {
      if constexpr (STAGE)
        return staged_values(db);
      else
        return y.v[db];
    };
    // What values say before the weights are there: the largest power among the blocks that any column
    // sees (others' bytes may be anything), and where the NaN codes are.
    auto look_at_values = [&]() {
      if (partial) {
        const bool seen = here && t0 + 16 * lg < hi;
        top = seen ? ev : 0;
        uint32_t nans = 0;
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const uint4 u = values_of(db);
          nans |= nan_bytes(u.x) | nan_bytes(u.y) | nan_bytes(u.z) | nan_bytes(u.w);
        }
        if (__any(nans != 0)) {
          // NaN codes (or what lies behind the last key): out of the products, whose weight for them
          // may be 0, and NaN in the sums of the columns that see them
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            uint4 u = values_of(db);
            uint32_t* w = STAGE ? reinterpret_cast<uint32_t*>(&u) : reinterpret_cast<uint32_t*>(&y.v[db]);
            f32x4 cnt[QB];
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) cnt[qb] = zero4();
#pragma unroll
            for (int kc = 0; kc < 2; ++kc) {
              f16x8 is;
#pragma unroll
              for (int j = 0; j < 8; ++j)
                is[j] = (_Float16)(float)(nan_bytes(w[2 * kc + j / 4]) >> (8 * (j % 4) + 7) & 1);
#pragma unroll
              for (int qb = 0; qb < QB; ++qb) {
                f16x8 sees;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                  sees[j] = (_Float16)(here && t0 + 16 * lg + 8 * kc + j < upto[qb] ? 1.f : 0.f);
                cnt[qb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(is, sees, cnt[qb], 0, 0, 0);
              }
            }
#pragma unroll
            for (int qb = 0; qb < QB; ++qb)
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (cnt[qb][i] > 0.f) oacc[db][qb][i] = __builtin_nanf("");
            if constexpr (!STAGE) clean(w);
          }
          dirty = true;
        }
      }
    };
    // The unit for this tile, and the factor of this lane's values.
    auto raise = [&]() {
      int now = top;
      if constexpr (UNI) {
        now = __builtin_amdgcn_readfirstlane(now);
      } else {
        now = max(now, __shfl_xor(now, 16, 64));
        now = __builtin_amdgcn_readfirstlane(max(now, __shfl_xor(now, 32, 64)));
      }
      if (now > unit) {
        const float f = two_to(unit - now);
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int qb = 0; qb < QB; ++qb) oacc[db][qb] *= f;
        unit = now;
      }
      // (a block that no column sees: any power will do)
      return two_to(min(ev - unit, 0) + V_BIAS);
    };
    auto value_frag = [&](const uint4& u, int kc, float two) {
      return kc ? codes_f16(u.z, u.w, two) : codes_f16(u.x, u.y, two);
    };
    auto add = [&](const f16x8& vf, const f16x8 (*pf)[2], int db, int kc, int qb) {
#pragma unroll
      for (int n = NP - 1; n >= 0; --n)
        oacc[db][qb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pf[n][kc], oacc[db][qb], 0, 0, 0);
    };
    if constexpr (D <= 32) {
      // one block of columns after another, the next one's products under way
      look_at_values();
      if constexpr (QLDS) asm volatile("" ::: "memory");  // the queries stay in LDS
      QF kf[4][CH];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int ch = 0; ch < CH; ++ch) kf[t][ch] = key_frag(x, t, ch);
      auto products = [&](f32x4* r, int qb) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          r[t] = zero4();
#pragma unroll
          for (int ch = 0; ch < CH; ++ch)
#pragma unroll
            for (int n = NQ - 1; n >= 0; --n) r[t] = KQ<D>::mma(kf[t][ch], query_frag(n, qb, ch), r[t]);
        }
      };
      const float two = raise();
      f16x8 vf[DB][2];
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int kc = 0; kc < 2; ++kc) vf[db][kc] = value_frag(y.v[db], kc, two);
      codes_read();
      f32x4 s[4];
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        f16x8 pf[NP][2];
        products(s, qb);
        weigh(s, qb, cs, t0, partial, here, pf);
#pragma unroll
        for (int kc = 0; kc < 2; ++kc)
#pragma unroll
          for (int db = 0; db < DB; ++db) add(vf[db][kc], pf, db, kc, qb);
      }
    } else {
      f16x8 pf[QB][NP][2];
      f32x4 s[QB][4];
      asm volatile("" ::: "memory");  // the queries stay in LDS
#pragma unroll
      for (int qb = 0; qb < QB; ++qb)
#pragma unroll
        for (int t = 0; t < 4; ++t) s[qb][t] = zero4();
#pragma unroll
      for (int ch = 0; ch < CH; ++ch) {
        if constexpr (STAGE) {  // two products' keys at a time
          if (ch % 2 == 0) {
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              const uint4 u = staged_keys(t, ch / 2);
              x.k[t][0] = u.x; x.k[t][1] = u.y; x.k[t][2] = u.z; x.k[t][3] = u.w;
            }
          }
        }
        QF f[NQ][QB];
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
          for (int qb = 0; qb < QB; ++qb) f[n][qb] = query_frag(n, qb, ch);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const QF kf = key_frag(x, t, STAGE ? ch % 2 : ch);
#pragma unroll
          for (int n = NQ - 1; n >= 0; --n)
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) s[qb][t] = KQ<D>::mma(kf, f[n][qb], s[qb][t]);
        }
      }
      codes_read();
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) weigh(s[qb], qb, cs, t0, partial, here, pf[qb]);
      look_at_values();
      const float two = raise();
      constexpr int AT = STAGE ? 2 : DB;  // blocks of values between two products into one sum
      auto sums = [&](auto fetch) {
#pragma unroll
        for (int d0 = 0; d0 < DB; d0 += AT) {
          uint4 u[AT];
#pragma unroll
          for (int i = 0; i < AT; ++i) u[i] = fetch(d0 + i);
#pragma unroll
          for (int kc = 0; kc < 2; ++kc)
#pragma unroll
            for (int i = 0; i < AT; ++i) {
              const f16x8 vf = value_frag(u[i], kc, two);
#pragma unroll
              for (int qb = 0; qb < QB; ++qb) add(vf, pf[qb], d0 + i, kc, qb);
            }
        }
      };
      if (STAGE && dirty) {
        sums([&](int db) {
          uint4 u = values_of(db);
          clean(reinterpret_cast<uint32_t*>(&u));
          return u;
        });
      } else {
        sums(values_of);
      }
    }
    first = false;
  };
  // Whether a tile has blocks far apart and columns that may see the smaller one alone.
  auto apart = [&](const Keys<D>& x, int t0) {
    if (UNI || t0 + KT <= lo) return false;
    const bool seen = x.here && t0 + 16 * lg < hi;
    const int ev = power_byte(x.power >> 8);
    int low = seen ? ev : 255, high = seen ? ev : 0;
#pragma unroll
    for (int o = 16; o < 64; o <<= 1) {
      low = min(low, __shfl_xor(low, o, 64));
      high = max(high, __shfl_xor(high, o, 64));
    }
    return __builtin_amdgcn_readfirstlane(high - low) > V_GAP;
  };

  int t0 = k0 + (SPLIT ? wave * KT : 0);
  if constexpr (STAGE) {
    const int kall = min(splits > 1 ? k0 + chunk : len, hi_all);
    if (k0 < kall) {
      Keys<D> x;
      Values<D> none;
      auto turn = [&] { x.power = gpower, x.here = ghere; };
      bring(k0);
      put(0);
      turn();
      lds_barrier();
      for (; t0 < kall; t0 += KT) {
        const bool more = t0 + KT < kall;
        if (more) bring(t0 + KT);
        if (t0 < kend) compute(x, none, t0, -1, [] {});
        if (more) {
          put(cur ^ 1);
          turn();
        }
        lds_barrier();
        cur ^= 1;
      }
    }
  } else if (t0 < kend) {
    Keys<D> x;
    Values<D> y;
    look(t0);
    int pk = pid_of(t0, gk), pv = UNI ? pk : pid_of(t0, gv);
    load_k(x, t0, pk, pv);
    // (in this order, as in the loop: a wait for the keys must not be one for the values)
    __builtin_amdgcn_sched_barrier(0);
    load_v(y, t0, pv);
    __builtin_amdgcn_sched_barrier(0);
    for (; t0 < kend; t0 += STEP) {
      const bool more = t0 + STEP < kend;
      int only = -1, last = -1;
      if (apart(x, t0)) only = 0, last = 3;
      for (;; ++only) {
        if (only >= 0) {  // one block of the tile at a time, without the others' values
          load_v(y, t0, pv);
          if (lg != only) y = Values<D>{};
        }
        compute(x, y, t0, only, [&] {
          if (!more || only != last) return;
          look(t0 + STEP);
          pk = pid_of(t0 + STEP, gk);
          pv = UNI ? pk : pid_of(t0 + STEP, gv);
          load_k(x, t0 + STEP, pk, pv);
          if constexpr (D <= 32) load_v(y, t0 + STEP, pv);
        });
        if (UNI || only == last) break;
      }
      if constexpr (D > 32) {
        if (more) load_v(y, t0 + STEP, pv);
      }
    }
  }

  // the sums in units of 1, over all lanes of a column
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
    const float one = two_to(unit - 127 - V_BIAS - P_BIAS);
    lsum[qb] = rows4_sum(lsum[qb]) * two_to(-P_BIAS);
#pragma unroll
    for (int db = 0; db < DB; ++db) oacc[db][qb] *= one;
  }
  if constexpr (SPLIT) {
    // the four waves' sums, in LDS: wave w's of column k
    __shared__ float ml[4][16 * QB][2];
    float(*ow)[16 * QB][D + 4] = reinterpret_cast<float(*)[16 * QB][D + 4]>(lds);
    if constexpr (QLDS) __syncthreads();  // every wave has done with its queries
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const int k = qb * 16 + c;
      if (lg == 0) ml[wave][k][0] = ref[qb], ml[wave][k][1] = lsum[qb];
#pragma unroll
      for (int db = 0; db < DB; ++db)
        *reinterpret_cast<f32x4*>(&ow[wave][k][db * 16 + lg * 4]) = oacc[db][qb];
    }
    __syncthreads();
    // 4 channels of a column per thread
    for (int it = threadIdx.x; it < 16 * QB * (D / 4); it += 256) {
      const int k = it / (D / 4), d0 = it % (D / 4) * 4, col = col0 + k;
      if (col >= ncols) continue;
      const float m = fmaxf(fmaxf(ml[0][k][0], ml[1][k][0]), fmaxf(ml[2][k][0], ml[3][k][0]));
      float l = 0.f;
      f32x4 o = zero4();
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float f = exp2_hw(ml[w][k][0] - m);
        l = fmaf(ml[w][k][1], f, l);
        o += *reinterpret_cast<const f32x4*>(&ow[w][k][d0]) * f;
      }
      const int i = col / G, h = kh * G + col - i * G;
      if (splits > 1) {
        const int64_t at = ((int64_t)prob * a.L * G + col) * splits + sp;
        *reinterpret_cast<f32x4*>(part + at * D + d0) = o;
        if (d0 == 0) part_ml[at * 2] = m, part_ml[at * 2 + 1] = l;
      } else {
        T* p = out + b * a.so[0] + i * a.so[1] + h * a.so[2] + d0;
        const float inv = l == 0.f ? 0.f : __builtin_amdgcn_rcpf(l);
#pragma unroll
        for (int j = 0; j < 4; ++j) st(p + j, l == 0.f ? 0.f : o[j] * inv);
        if (a.lse && d0 == 0)
          a.lse[(b * a.L + i) * a.heads + h] =
              l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
      }
    }
  } else {
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const int col = col0 + qb * 16 + c;
      if (col >= ncols) continue;
      const int i = row_of(col), h = kh * G + col - i * G;
      const float l = lsum[qb];
      if (splits > 1) {
        const int64_t at = ((int64_t)prob * a.L * G + col) * splits + sp;
#pragma unroll
        for (int db = 0; db < DB; ++db)
          *reinterpret_cast<f32x4*>(part + at * D + db * 16 + lg * 4) = oacc[db][qb];
        if (lg == 0) part_ml[at * 2] = ref[qb], part_ml[at * 2 + 1] = l;
        continue;
      }
      T* p = out + b * a.so[0] + i * a.so[1] + h * a.so[2] + lg * 4;
      const float inv = l == 0.f ? 0.f : __builtin_amdgcn_rcpf(l);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        float y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = l == 0.f ? 0.f : oacc[db][qb][j] * inv;
        if (wide) {
          if constexpr (F32)
            *reinterpret_cast<float4*>(p + db * 16) = make_float4(y[0], y[1], y[2], y[3]);
          else
            *reinterpret_cast<uint2*>(p + db * 16) = make_uint2(pack2(y[0], y[1]), pack2(y[2], y[3]));
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) st(p + db * 16 + j, y[j]);
        }
      }
      if (a.lse && lg == 0)
        a.lse[(b * a.L + i) * a.heads + h] =
            l == 0.f ? -INFINITY : (ref[qb] + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
    }
  }
}

// The sums of the splits of each column: `share` groups of D / 4 lanes take them in turns, then the
// groups' sums are added in their order.
template <int D, class T>
__global__ __launch_bounds__(256) void k_cache8_join(Cache8Attend a, T* __restrict__ out,
                                                     const float* __restrict__ part,
                                                     const float* __restrict__ part_ml,
                                                     int64_t columns, int splits, int chunk,
                                                     int share) {
  __shared__ float gm[256], gl[256];
  __shared__ f32x4 go[256];
  const Cache8Geo& g = a.g;
  constexpr int W = D / 4;
  const int lanes = W * share, tid = threadIdx.x, sub = tid % lanes / W, d0 = tid % W * 4;
  const int64_t at = (int64_t)blockIdx.x * (256 / lanes) + tid / lanes;
  const int G = a.heads / g.heads;
  const int64_t per = (int64_t)a.L * G, prob = at / per, b = prob / g.heads;
  const int col = (int)(at - prob * per), i = col / G;
  const int h = (int)(prob - b * g.heads) * G + col - i * G;
  const bool on = at < columns && !(a.n_rows && i >= a.n_rows[b]);
  float m = -FLT_MAX, l = 0.f;
  f32x4 o = zero4();
  if (on) {  // splits behind the last key were not written
    const int len = min(max(a.lens[b], 0), a.max_rows), live = min(splits, (len + chunk - 1) / chunk);
    // Splits whose sums are under way at a time (references first, then sums, one after another: 12.5 us
    // instead of 8.5 for 128 columns of 256 splits, 16.1 instead of 17.4 for 64,000 of 3).
    constexpr int N = 8;
    for (int s0 = sub; s0 < live; s0 += N * share) {
      float2 ml[N];
      f32x4 x[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int64_t k = at * splits + min(s0 + i * share, live - 1);
        ml[i] = *reinterpret_cast<const float2*>(part_ml + k * 2);
        x[i] = *reinterpret_cast<const f32x4*>(part + k * D + d0);
      }
      float now = m;
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (s0 + i * share < live) now = fmaxf(now, ml[i].x);
      const float old = exp2_hw(m - now);
      l *= old;
      o *= old;
      m = now;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (s0 + i * share >= live) break;
        const float f = exp2_hw(ml[i].x - m);
        l = fmaf(ml[i].y, f, l);
        o += x[i] * f;
      }
    }
  }
  if (share > 1) {
    gm[tid] = m;
    gl[tid] = l;
    go[tid] = o;
    __syncthreads();
    if (sub) return;
    const float mine = m;
    for (int s = 1; s < share; ++s) m = fmaxf(m, gm[tid + s * W]);
    const float f0 = exp2_hw(mine - m);
    l *= f0;
    o *= f0;
    for (int s = 1; s < share; ++s) {
      const float f = exp2_hw(gm[tid + s * W] - m);
      l = fmaf(gl[tid + s * W], f, l);
      o += go[tid + s * W] * f;
    }
  }
  if (!on) return;
  T* p = out + b * a.so[0] + i * a.so[1] + h * a.so[2] + d0;
  const float inv = l == 0.f ? 0.f : __builtin_amdgcn_rcpf(l);
#pragma unroll
  for (int j = 0; j < 4; ++j) st(p + j, l == 0.f ? 0.f : o[j] * inv);
  if (a.lse && d0 == 0)
    a.lse[(b * a.L + i) * a.heads + h] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
}

// How a call is cut: 16 QB columns per wave, the waves of a workgroup on the same columns or not, and
// the keys in `splits` pieces of `chunk`.
struct Cut {
  int qb, coltiles, splits, chunk;
  bool split;
};

Cut cut_of(const Cache8Attend& a, bool f32) {
  Cut c;
  const int64_t cols = (int64_t)a.L * (a.heads / a.g.heads), probs = (int64_t)a.plan_B * a.g.heads;
  const int64_t keys = a.max_rows;
  c.split = cols <= 32;
  // (Columns of a wave: as many as its registers hold.  d = 128, 16 heads on 4, 4 sequences of up to
  // 1000 rows: 288 us with 32, spilled or one wave a SIMD, 207 with 16 and two.  From 33 columns on
  // every wave has its own, and waves without any wait: one head of one sequence on 16,000 keys, 16 / 32
  // / 33 / 64 / 128 columns: 10 / 11 / 29 / 29 / 30 us at d = 32, 12 / 14 / 25 / 30 / 30 at d = 128.)
  c.qb = c.split ? (cols <= 16 ? 1 : 2) : f32 ? 1 : a.g.d <= 32 ? 4 : 2;
  if (!c.split && c.qb == 2 && a.g.d == 128) {
    // Staged tiles, whose workgroups take 128 columns instead of 64, need one for every CU: 8 heads,
    // 1024 rows on 1100 keys, 1 / 2 / 4 sequences (128 / 256 / 512 workgroups): 36 / 39 / 48 us staged,
    // 28 / 37 / 70 us not; 128 rows on 8000 keys, 2 / 8 sequences: 45 / 66 us and 35 / 109 us.
    const int64_t wgs = (cols + 127) / 128 * probs * ((keys + 1023) / 1024);
    if (a.g.page < KT || cols <= 64 || wgs < 256) c.qb = 1;  // (33 to 64 leave half of it idle)
  }
  const int per = 16 * c.qb * (c.split ? 1 : 4);
  c.coltiles = (int)((cols + per - 1) / per);
  const int64_t blocks = probs * c.coltiles, want = 2048;
  // Keys worth a workgroup of their own, whose sums go through memory.  With 512 workgroups and more the
  // CUs are full and a split only evens them out: 8 sequences of 1000 rows on 2000 keys, 16 heads, d = 64:
  // 100 us in one piece, 127 in two; 4 of up to 1000 rows on 3000 to 5000 keys, 16 heads on 4, d = 128:
  // 254 us in one piece, 223 in two, 209 in three.
  const int least = c.split ? 512 : blocks >= 512 ? 2048 : 1024;
  int64_t s = blocks > 0 ? (want + blocks - 1) / blocks : 1;
  s = s < (keys + least - 1) / least ? s : (keys + least - 1) / least;
  if (s < 1) s = 1;
  c.chunk = (int)(((keys + s - 1) / s + 255) / 256 * 256);
  if (c.chunk < 256) c.chunk = 256;
  c.splits = (int)((keys + c.chunk - 1) / c.chunk);
  if (c.splits < 1) c.splits = 1;
  return c;
}

// Partial sums: of every column of plan_B sequences.
int64_t partials(const Cache8Attend& a, const Cut& c) {
  return c.splits > 1 ? (int64_t)a.plan_B * a.g.heads * a.L * (a.heads / a.g.heads) * c.splits : 0;
}

template <int D, class T, int QB, bool SPLIT>
hipError_t go(const Cache8Attend& a, const Cut& c, const T* q, T* out, hipStream_t s) {
  const int64_t probs = (int64_t)a.B * a.g.heads, n = partials(a, c);
  float* part = (float*)a.ws;
  float* ml = part + n * D;
  bool wide = (uintptr_t)q % 16 == 0 && (uintptr_t)out % 16 == 0;
  for (int i = 0; i < 3; ++i)
    wide = wide && a.sq[i] * sizeof(T) % 16 == 0 && a.so[i] * sizeof(T) % 16 == 0;
  const int64_t each = (int64_t)c.coltiles * c.splits, most = ((int64_t(1) << 32) - 1) / 256 / each;
  for (int64_t p0 = 0; p0 < probs; p0 += most) {
    const uint32_t np = (uint32_t)(probs - p0 < most ? probs - p0 : most);
    const unsigned blocks = (unsigned)(np * each);
    auto launch = [&](auto* kernel) {
      kernel<<<blocks, 256, 0, s>>>(a, q, out, part, ml, (uint32_t)p0, np, c.coltiles, c.splits,
                                    c.chunk, wide);
    };
    if constexpr (staged<D, sizeof(T) == 4, QB, SPLIT>()) {  // (only for such pages: cut_of)
      launch(k_cache8_attend<D, T, QB, SPLIT, true>);
    } else {
      if (a.g.page >= KT)
        launch(k_cache8_attend<D, T, QB, SPLIT, true>);
      else
        launch(k_cache8_attend<D, T, QB, SPLIT, false>);
    }
  }
  if (c.splits > 1) {
    int share = 1;  // some eight splits to a group
    while (share * 8 < c.splits && share < 256 / (D / 4)) share *= 2;
    const int64_t columns = probs * a.L * (a.heads / a.g.heads), per = 256 / (D / 4 * share);
    k_cache8_join<D, T><<<(unsigned)((columns + per - 1) / per), 256, 0, s>>>(
        a, out, part, ml, columns, c.splits, c.chunk, share);
  }
  return hipGetLastError();
}

template <int D, class T>
hipError_t go_d(const Cache8Attend& a, const T* q, T* out, hipStream_t s) {
  const Cut c = cut_of(a, sizeof(T) == 4);
  if (c.split)
    return c.qb == 1 ? go<D, T, 1, true>(a, c, q, out, s) : go<D, T, 2, true>(a, c, q, out, s);
  if constexpr (sizeof(T) == 4)
    return go<D, T, 1, false>(a, c, q, out, s);
  else if constexpr (D == 128)
    return c.qb == 1 ? go<D, T, 1, false>(a, c, q, out, s) : go<D, T, 2, false>(a, c, q, out, s);
  else
    return go<D, T, D <= 32 ? 4 : 2, false>(a, c, q, out, s);
}

}  // namespace

size_t cache8_attend_bytes(const Cache8Attend& a, bool f32) {
  return (size_t)partials(a, cut_of(a, f32)) * (a.g.d + 2) * 4;
}

template <class T>
hipError_t launch_cache8_attend(const Cache8Attend& a, const T* q, T* out, hipStream_t s) {
  switch (a.g.d) {
    case 16: return go_d<16>(a, q, out, s);
    case 32: return go_d<32>(a, q, out, s);
    case 64: return go_d<64>(a, q, out, s);
    default: return go_d<128>(a, q, out, s);
  }
}
template hipError_t launch_cache8_attend(const Cache8Attend&, const float*, float*, hipStream_t);
template hipError_t launch_cache8_attend(const Cache8Attend&, const bf16*, bf16*, hipStream_t);

}  // namespace tfm
