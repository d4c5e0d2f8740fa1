// Distillation from a teacher's top logits (declarations in vocab.h).
//
// With mt the largest logit outside the teacher's set J (the largest of all where there is no tail)
// and S = sum over those classes of exp((s_v - mt) / tau), every class outside J has the gradient
//     c exp((s_v - mt) / tau) + c1 exp(s_v - mt)
// with two factors per row, so a row is read once, summed and written once: it stays in registers
// between the two.  What J adds to the sums, the loss and J's own gradients come from its at most
// 256 entries, in 64 bits: the loss is a small difference of large logarithms where the student is
// near the teacher, and the error of S cancels in it to first order only if all else is exact.
//
// Rows of up to 1,024 classes go to groups of 8 to 64 lanes, longer ones to a workgroup each; few
// long rows are split over workgroups.  Bound by HBM (a read and a write of the logits) from some
// thousand classes on: 8,192 x 5,000 float32 81 us (4.1 TB/s; a copy takes 69), 4,096 x 50,021
// bfloat16 with a label's softmax at another temperature 227 us (3.6 TB/s; a copy 171: two
// exponentials per class and pass are 164 us of issue beside it).  Short rows are bound by what a row
// costs in 64 bits (2^21 x 10: 0.22 ns a row), few long ones by latency (7 x 131,072: 22 us in three
// launches, the first of which waits for the one workgroup that has the teacher's entries).
#include "math64.h"
#include "mfma.h"
#include "vocab.h"
#include "wave.h"

#include <hip/hip_runtime.h>

namespace tfm {
namespace {

constexpr float LOG2E = 1.44269504088896340736f;

template <int W, class V>
__device__ __forceinline__ V group_sum(V v) {
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
template <int W>
__device__ __forceinline__ float group_max(float v) {
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
// Over the NW waves of a workgroup; every thread gets the result.  buf: NW entries.
template <int NW>
__device__ __forceinline__ double block_sum(double v, double* buf) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
  __syncthreads();
  const int lane = threadIdx.x & 63;
  return wave_sum(lane < NW ? buf[lane] : 0.0);
}

// Partial sums of the weights in 64 bits: workgroup b sums a contiguous share.
__global__ __launch_bounds__(256) void k_distill_weights(const float* __restrict__ w, int64_t N,
                                                         int64_t share, double* __restrict__ part) {
  __shared__ double buf[4];
  const int64_t a = blockIdx.x * share, b = a + share < N ? a + share : N;
  double acc = 0.0;
  for (int64_t n = a + threadIdx.x; n < b; n += 1024) {
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = n + 256 * i < b ? w[n + 256 * i] : 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) acc += (double)v[i];
  }
  acc = block_sum<4>(acc, buf);
  if (threadIdx.x == 0) part[blockIdx.x] = acc;
}

// Sum of the weights from its parts (N where there are none); every lane of the wave gets it.
__device__ __forceinline__ double weight_total(const DistillGeo& g) {
  if (!g.weights) return (double)g.N;
  double s = 0.0;
  for (int i = threadIdx.x & 63; i < g.nwsum; i += 64) s += g.wsum[i];
  return wave_sum(s);
}

__device__ __forceinline__ int row_classes(const DistillGeo& g, int64_t n) {
  return g.ncls ? min(max(g.ncls[n], 0), g.V) : g.V;
}

// The row's scalars from its sums:
//   S_t, S_1    sums of exp((s - mt) / tau) and exp(s - mt) outside J
//   T_t, T_1    sums of exp((s - mj) / tau) and exp(s - mj) over J (unused without a tail; 0, or NaN
//               where J has a NaN, if no logit of J lies above -inf)
//   E, G        sums over J of e_j and e_j (log e_j - (s_j - mj) / tau), where p_j = e_j / E
//               without a tail and e_j with one
// m is the largest of all logits.  W lanes call it with the same values, W >= 8: each evaluates one
// of the exponentials, of the logarithms and of the quotients.
struct RowSums {
  double S_t, S_1, T_t, T_1, E, G;
};
struct RowOut {
  double loss;
  double j_q, j_1;    // gradient of class j in J: j_q exp((s_j - m) / tau) + j_1 exp(s_j - m)
  double j_p, label;  //   - j_p e_j, and of the label: - label
  float c_t, c_1;     // gradient outside J: c_t exp((s - mt) / tau) + c_1 exp(s - mt)
};
// The largest logit as a row goes on with it: -inf where all are -inf and the row is left out, but
// not where the others are NaN, which the maxima pass over and the sums do not.
__device__ __forceinline__ float row_max(float m, double S_t, double T_t) {
  return m == -INFINITY && !(S_t + T_t == 0.0) ? 0.f : m;
}
template <int W>
__device__ __forceinline__ double of_lane(double v, int i) {
  if constexpr (W == 64) return from_lane(v, i);
  else return __shfl(v, i, W);
}
template <int W>
__device__ __forceinline__ RowOut row_scalars(const DistillGeo& g, const RowSums& r, float mt,
                                              float mj, float m, double share, bool known,
                                              double s_label) {
  const int lane = threadIdx.x % W;
  const double tau = g.tau, alpha = g.alpha, itau = 1.0 / tau;
  const bool some = mt > -INFINITY, any = mj > -INFINITY;
  // where mt and mj lie below m
  const double back = some ? (double)mt - (double)m : 0.0, d = any ? (double)mj - (double)m : 0.0;
  const double x = exp64((lane & 2 ? d : back) * (lane & 1 ? 1.0 : itau));
  const double bt = of_lane<W>(x, 0), b1 = of_lane<W>(x, 1);
  double Zt = r.S_t * bt, Z1 = r.S_1 * b1;
  if (g.tail) {
    Zt += r.T_t * of_lane<W>(x, 2);
    Z1 += r.T_1 * of_lane<W>(x, 3);
  }
  // the teacher's mass: P in the set, pt outside
  const double one_over = 1.0 / (lane == 0 ? Zt : lane == 1 ? r.E : lane == 2 ? r.S_t : Z1);
  const double norm = g.tail || r.E == 0.0 ? 1.0 : of_lane<W>(one_over, 1);
  const double P = r.E * norm;
  double pt = 0.0;
  if (g.tail && some) {
    pt = 1.0 - P;
    if (pt <= 0.0) pt = 0.0;
  }
  const double l = log64(lane == 0 ? Zt : lane == 1 ? r.E : lane == 2 ? pt : lane == 3 ? r.S_t : Z1);
  const double lZt = of_lane<W>(l, 0);
  double D = (r.G - r.E * d * itau) * norm + lZt * P;
  if (!g.tail && r.E != 0.0) D -= of_lane<W>(l, 1);
  const double lp = of_lane<W>(l, 2), lS = of_lane<W>(l, 3), lZ1 = of_lane<W>(l, 4);
  if (!(pt == 0.0)) D += pt * (lp - (back * itau + lS - lZt));
  RowOut o;
  o.loss = alpha > 0.0 ? alpha * tau * tau * D : 0.0;
  const double cd = alpha * tau * share, cl = known ? (1.0 - alpha) * share : 0.0;
  if (known) o.loss += (1.0 - alpha) * (lZ1 - (s_label - (double)m));
  o.j_q = cd * (P + pt) * of_lane<W>(one_over, 0);
  o.j_1 = cl * of_lane<W>(one_over, 3);
  o.j_p = cd * norm;
  o.label = cl;
  o.c_t = (float)(o.j_q * bt - (pt > 0.0 ? cd * pt * of_lane<W>(one_over, 2) : 0.0));
  o.c_1 = (float)(o.j_1 * b1);
  return o;
}

// ---- rows of up to 1,024 classes ----------------------------------------------------------------
// W lanes to a row, class lane + W i in register i.  Bound by its 64-bit arithmetic and element loads:
// 65,536 x 300 float32 157 us (a copy 33), 32,768 x 1,000 206 (55).  Where one wave's registers end
// the kernel for longer rows is the faster one: 32,768 x 1,024 206 us here, x 1,028 146 there.
constexpr int SMALL_V = 1024;

template <class T, int W, int I>
__global__ __launch_bounds__(256) void k_distill_small(DistillGeo g, int64_t first,
                                                       const T* logits, T* dlogits) {
  // per class: the first of the teacher's entries on it, and that entry's logit
  __shared__ int32_t owner[256 * I];
  __shared__ float tval[256 * I];
  const int lane = threadIdx.x % W, grp = threadIdx.x / W;
  int32_t* own = owner + grp * W * I;
  float* tv = tval + grp * W * I;
  const double wtot = weight_total(g), itau = 1.0 / (double)g.tau;
  const float c = LOG2E / g.tau;
  const int64_t at = first + (int64_t)blockIdx.x * (256 / W) + grp;
  const bool mine = at < g.N;
  const int64_t n = mine ? at : g.N - 1;  // (no group leaves before the barriers)
  const T* s = logits + n * g.ld;
  const float wn = g.weights ? g.weights[n] : 1.f;
  const int V = row_classes(g, n);
  float x[I];
#pragma unroll
  for (int i = 0; i < I; ++i) {
    const int v = lane + W * i;
    x[i] = v < V ? ld(s + v) : -INFINITY;
    own[v] = 0x7fffffff;
  }
  __syncthreads();
  for (int j = lane; j < g.k; j += W) {
    const int v = g.idx[n * g.k + j];
    if (v >= 0 && v < V) atomicMin(&own[v], j);
  }
  __syncthreads();
  for (int j = lane; j < g.k; j += W) {
    const int v = g.idx[n * g.k + j];
    if (v >= 0 && v < V && own[v] == j) tv[v] = g.top[n * g.k + j];
  }
  __syncthreads();
  float m = -INFINITY, mt = -INFINITY, tm = -INFINITY;
  bool in[I];
  float t[I];
#pragma unroll
  for (int i = 0; i < I; ++i) {
    const int v = lane + W * i;
    in[i] = own[v] != 0x7fffffff;
    t[i] = in[i] ? tv[v] : -INFINITY;
    m = fmaxf(m, x[i]);
    if (!(in[i] && g.tail)) mt = fmaxf(mt, x[i]);
    tm = fmaxf(tm, t[i]);
  }
  m = group_max<W>(m);
  mt = group_max<W>(mt);
  tm = group_max<W>(tm);
  const float mr = mt > -INFINITY ? mt : 0.f;
  const double lse = g.tail ? (double)g.lse[n] : 0.0;
  float sum_t = 0.f, sum_1 = 0.f;
  RowSums r = {};
  double e[I];
#pragma unroll
  for (int i = 0; i < I; ++i) {
    e[i] = 0.0;
    if (!(in[i] && g.tail)) {
      sum_t += exp2_hw((x[i] - mr) * c);
      sum_1 += exp2_hw((x[i] - mr) * LOG2E);
    }
    if (in[i]) {
      const double d = m > -INFINITY ? (double)x[i] - (double)m : (double)x[i], y = d * itau;
      double lt;
      if (g.tail) {
        lt = (double)t[i] * itau - lse;
        r.T_t += exp64(y);
        r.T_1 += exp64(d);
      } else {
        lt = tm > -INFINITY ? ((double)t[i] - (double)tm) * itau : -INFINITY;
      }
      if (t[i] != t[i]) lt = NAN;
      e[i] = exp64(lt);
      r.E += e[i];
      if (!(e[i] == 0.0)) r.G += e[i] * (lt - y);
    }
  }
  r.S_t = group_sum<W>((double)sum_t);
  r.S_1 = group_sum<W>((double)sum_1);
  r.E = group_sum<W>(r.E);
  r.G = group_sum<W>(r.G);
  if (g.tail) {
    r.T_t = group_sum<W>(r.T_t);
    r.T_1 = group_sum<W>(r.T_1);
  }
  m = row_max(m, r.S_t, r.T_t);
  const bool left_out = wn == 0.f || m == -INFINITY;
  const int y = g.labels ? g.labels[n] : -1;
  const bool known = y >= 0 && y < V;
  float sy = -INFINITY;
#pragma unroll
  for (int i = 0; i < I; ++i)
    if (lane + W * i == y) sy = x[i];
  sy = __shfl(sy, known ? y % W : 0, W);
  const double share = wtot != 0.0 ? (double)wn / wtot : 0.0;
  const RowOut o = row_scalars<W>(g, r, mt, m, m, share, known, (double)sy);
  if (mine && lane == 0) g.row_loss[n] = left_out ? 0.f : (float)o.loss;
  if (dlogits && mine) {
    T* ds = dlogits + n * g.ld;
#pragma unroll
    for (int i = 0; i < I; ++i) {
      const int v = lane + W * i;
      if (v >= g.V) continue;
      float d = 0.f;
      if (!left_out && v < V) {
        if (in[i]) {
          const double dx = (double)x[i] - (double)m;
          double q = o.j_q * exp64(dx * itau) - o.j_p * e[i];
          if (known) q += o.j_1 * exp64(dx) - (v == y ? o.label : 0.0);
          d = (float)q;
        } else {
          d = o.c_t * exp2_hw((x[i] - mr) * c);
          if (known) d += o.c_1 * exp2_hw((x[i] - mr) * LOG2E) - (v == y ? (float)o.label : 0.f);
        }
      }
      st(ds + v, d);
    }
  }
}

// Most rows that are split, and the fewest classes.  The second launch and the hand-over take 4 us;
// bf16, k = 64, split against whole: 1 x 16,384 15.1 / 14.1 us, 1 x 32,768 15.1 / 19.7, 64 x 32,768
// 17.5 / 20.8, 64 x 131,072 24.8 / 31.1, 128 x 131,072 38.6 / 33.7.
constexpr int64_t SPLIT_ROWS = 64;
constexpr int32_t SPLIT_V = 24576;

// ---- longer rows ---------------------------------------------------------------------------------
// Pieces of 16 bytes on 16-byte boundaries; what a row has before the first and behind the last of
// them (at most 14 classes) goes to a thread each.
template <class T>
struct Piece {
  static constexpr int E = 16 / sizeof(T);
  uint4 u;
  __device__ __forceinline__ float get(int j) const {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[j]);
    else return __uint_as_float(j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16);
  }
};
__device__ __forceinline__ void store_piece(float* p, const float* d) {
  *reinterpret_cast<float4*>(p) = make_float4(d[0], d[1], d[2], d[3]);
}
__device__ __forceinline__ void store_piece(bf16* p, const float* d) {
  *reinterpret_cast<uint4*>(p) =
      make_uint4(pack2(d[0], d[1]), pack2(d[2], d[3]), pack2(d[4], d[5]), pack2(d[6], d[7]));
}

// What the two launches of a split row hand on (see k_distill_rows): of a part, and of J.
struct PartSums {
  double S_t, S_1;  // relative to mt
  float mt, pad;
};
struct SetSums {
  double E, G, T_t, T_1;
  float mj, tm;
  float s_label, pad;
};
struct SetEntry {
  int32_t idx;  // -1: none
  float s;      // its logit (the gradient may be written over the logits)
};
struct Split {
  PartSums* part;   // [N][parts]
  SetSums* set;     // [N]
  SetEntry* entry;  // [N][k]
  int32_t parts, len;
};
enum { WHOLE = 0, SUM = 1, APPLY = 2 };

// TH threads, I pieces per thread in registers.  WHOLE: one workgroup per row.  Few long rows are
// split into `parts` of `len` classes, a workgroup each, in two launches: SUM leaves every part's
// sums (and one more workgroup the set's), APPLY joins them and writes the part's gradients.
// I = 0: rows that the registers of a CU do not hold, read again for each of the three passes, and
// (dlogits not aligned as logits) rows written class by class.  TWO: the label's softmax has another
// temperature than the teacher's, a second exponential per class.
template <class T, int TH, int I, bool TWO, int STAGE>
__global__ __launch_bounds__(TH, I == 32 ? 3 : 1) void k_distill_rows(DistillGeo g, Split sp,
                                                                      int64_t first,
                                                                      const T* logits, T* dlogits) {
  constexpr int E = Piece<T>::E, NW = TH / 64;
  extern __shared__ uint32_t inside[];  // a bit per class, the first piece's from bit 0 on: in J
  __shared__ alignas(16) int32_t jidx[DISTILL_KMAX];
  __shared__ float fbuf[3][NW];
  __shared__ double dbuf[6][NW];
  __shared__ RowOut row;
  __shared__ float row_mt, row_m;
  __shared__ int again, label_in;
  const int tid = threadIdx.x, lane = tid & 63, w = wave_id();
  const double itau = 1.0 / (double)g.tau;
  const float c = LOG2E / g.tau;
  const int64_t n = first + (STAGE ? blockIdx.y : blockIdx.x);
  const T* s = logits + n * g.ld;
  T* ds = dlogits ? dlogits + n * g.ld : nullptr;
  const float wn = g.weights ? g.weights[n] : 1.f;
  const int V = row_classes(g, n);
  // this workgroup's classes [lo, hi)
  const int part = STAGE ? (int)blockIdx.x : 0;
  const int lo = STAGE ? min(part * sp.len, V) : 0, hi = STAGE ? min(lo + sp.len, V) : V;
  // classes before the first piece
  const int lead = min((int)(-(uintptr_t)(s + lo) % 16 / sizeof(T)), hi - lo);
  const int np = (hi - lo - lead) / E;
  // pieces lie at a uniform base plus a 32-bit offset (a 64-bit address each would cost registers)
  const char* s0 = reinterpret_cast<const char*>(s + lo + lead);
  char* ds0 = reinterpret_cast<char*>(ds + lo + lead);
  const uint32_t off = tid * 16u;
  // the class beside the pieces that this thread looks after, hi: none
  const int odd = tid < lead ? lo + tid : min(lo + tid + np * E, hi);
  // dlogits may lie otherwise than logits (I = 0 then)
  const bool whole = I > 0 || (uintptr_t)ds % 16 == (uintptr_t)s % 16;
  // zeros for the classes from v0 on
  auto zero_from = [&](int v0) __attribute__((always_inline)) {
    const int end = STAGE ? min((part + 1) * sp.len, g.V) : g.V;
    if (ds)
      for (int v = v0 + tid; v < end; v += TH) st(ds + v, 0.f);
  };
  if (wn == 0.f || V == 0) {
    if (STAGE == SUM) return;
    zero_from(STAGE ? part * sp.len : 0);
    if (part == 0 && tid == 0) g.row_loss[n] = 0.f;
    return;
  }
  // the teacher's entries
  int my = -1;
  float tj = -INFINITY, sj = -INFINITY, sy = -INFINITY, mj, tm;
  const int y = g.labels ? g.labels[n] : -1;
  const bool known = y >= 0 && y < V;
  const float lse = g.tail ? g.lse[n] : 0.f;
  if (tid < g.k) tj = g.top[n * g.k + tid];
  if (STAGE == APPLY) {
    if (tid < g.k) {
      const SetEntry e = sp.entry[n * g.k + tid];
      my = e.idx;
      sj = e.s;
    }
    mj = sp.set[n].mj;
    tm = sp.set[n].tm;
    sy = sp.set[n].s_label;
  } else {
    if (tid < g.k) my = g.idx[n * g.k + tid];
    if (my < 0 || my >= V) my = -1;
    if (my >= 0) sj = ld(s + my);
    if (known) sy = ld(s + y);
  }
  // bit of class v: shifted to where the first piece starts a word
  const int shift = 32 - lead - lo;
  for (int v = tid; v < (hi + shift + 31) / 32; v += TH) inside[v] = 0;
  if (tid == 0) {
    again = STAGE == SUM;  // (the set's workgroup has no bits to go by)
    label_in = 0;
  }
  if (tid < DISTILL_KMAX) jidx[tid] = my;
  __syncthreads();
  if (my >= lo && my < hi) {
    const uint32_t bit = 1u << ((my + shift) & 31);
    if (atomicOr(&inside[(my + shift) >> 5], bit) & bit) again = 1;
    if (my == y) label_in = 1;
  }
  __syncthreads();
  // log e_j of this thread's entry (RowSums)
  auto log_e = [&]() __attribute__((always_inline)) {
    if (tj != tj) return (double)NAN;
    if (g.tail) return (double)tj * itau - (double)lse;
    return tm > -INFINITY ? ((double)tj - (double)tm) * itau : (double)-INFINITY;
  };
  if (STAGE == WHOLE || (STAGE == SUM && part == sp.parts)) {
    if (again) {  // perhaps a repeated class: its first entry counts
      bool earlier = false;
      for (int j = 0; j < g.k; j += 16) {
#pragma unroll
        for (int q = 0; q < 16; q += 4) {
          const int4 v = *reinterpret_cast<const int4*>(jidx + j + q);
          earlier |= (v.x == my && j + q < tid) || (v.y == my && j + q + 1 < tid) ||
                     (v.z == my && j + q + 2 < tid) || (v.w == my && j + q + 3 < tid);
        }
      }
      if (earlier) my = -1;
    }
    // J's maxima, and its sums relative to them: done before the row arrives, so that their
    // registers are free when it does
    if (my < 0) tj = -INFINITY;
    mj = wave_max(my >= 0 ? sj : -INFINITY);
    tm = wave_max(tj);
    if (lane == 0) {
      fbuf[0][w] = mj;
      fbuf[1][w] = tm;
    }
    __syncthreads();
    mj = wave_max(lane < NW ? fbuf[0][lane] : -INFINITY);
    tm = wave_max(lane < NW ? fbuf[1][lane] : -INFINITY);
    double q[4] = {0.0, 0.0, 0.0, 0.0};
    if (w * 64 < g.k) {  // the waves that hold entries
      if (my >= 0) {
        const double d = mj > -INFINITY ? (double)sj - (double)mj : (double)sj, lt = log_e();
        q[0] = exp64(lt);
        if (!(q[0] == 0.0)) q[1] = q[0] * (lt - d * itau);
        q[2] = exp64(d * itau);
        q[3] = TWO ? exp64(d) : q[2];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = wave_sum(q[i]);
    }
    if (lane == 0)
#pragma unroll
      for (int i = 0; i < 4; ++i) dbuf[2 + i][w] = q[i];
    if (STAGE == SUM) {
      if (tid < g.k) sp.entry[n * g.k + tid] = {my, sj};
      __syncthreads();
      if (w == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = wave_sum(lane < NW ? dbuf[2 + i][lane] : 0.0);
        if (lane == 0) sp.set[n] = {q[0], q[1], q[2], q[3], mj, tm, sy, 0.f};
      }
      return;
    }
  }
  Piece<T> x[I > 0 ? I : 1];
  if constexpr (I > 0) {
#pragma unroll
    for (int i = 0; i < I; ++i)
      if (i * TH + tid < np) x[i].u = *reinterpret_cast<const uint4*>(s0 + i * TH * 16 + off);
  }
  const float xo = odd < hi ? ld(s + odd) : -INFINITY;
  auto each = [&](auto f) __attribute__((always_inline)) {
    if constexpr (I > 0) {
#pragma unroll
      for (int i = 0; i < I; ++i)
        if (i * TH + tid < np) f(x[i], i * TH);
    } else {
      for (int v0 = 0; v0 + tid < np; v0 += TH) {
        x[0].u = *reinterpret_cast<const uint4*>(s0 + v0 * 16 + off);
        f(x[0], v0);
      }
    }
  };
  float mt, m;
  if (STAGE != APPLY) {
    // f for every class that the sums do not leave out
    auto each_summed = [&](auto f) __attribute__((always_inline)) {
      each([&](const Piece<T>& p, int v0) __attribute__((always_inline)) {
        uint32_t o = 0;
        if (g.tail) {
          o = reinterpret_cast<const uint8_t*>(inside + 1)[(v0 * E >> 3) + (tid * E >> 3)];
          if (E == 4) o = o >> (tid & 1) * 4 & 15u;
        }
        if (o == 0) {
#pragma unroll
          for (int j = 0; j < E; ++j) f(p.get(j));
        } else {
#pragma unroll
          for (int j = 0; j < E; ++j) f(o >> j & 1 ? -INFINITY : p.get(j));
        }
      });
      if (odd < hi && !(g.tail && inside[(odd + shift) >> 5] >> ((odd + shift) & 31) & 1)) f(xo);
    };
    mt = -INFINITY;
    each_summed([&](float v) __attribute__((always_inline)) { mt = fmaxf(mt, v); });
    mt = wave_max(mt);
    if (lane == 0) fbuf[2][w] = mt;
    __syncthreads();
    mt = wave_max(lane < NW ? fbuf[2][lane] : -INFINITY);
    const float mr = mt > -INFINITY ? mt : 0.f;
    float sum_t = 0.f, sum_1 = 0.f;
    each_summed([&](float v) __attribute__((always_inline)) {
      const float d = v - mr;
      sum_t += exp2_hw(d * c);
      if (TWO) sum_1 += exp2_hw(d * LOG2E);
    });
    const double S = wave_sum((double)sum_t), S1 = TWO ? wave_sum((double)sum_1) : S;
    if (lane == 0) {
      dbuf[0][w] = S;
      dbuf[1][w] = S1;
    }
    __syncthreads();
  }
  if (w == 0) {
    double q[6];
#pragma unroll
    for (int i = 0; i < (STAGE == SUM ? 2 : 6); ++i)
      if (STAGE != APPLY) q[i] = wave_sum(lane < NW ? dbuf[i][lane] : 0.0);
    if (STAGE == SUM) {
      if (lane == 0) sp.part[n * sp.parts + part] = {q[0], q[1], mt, 0.f};
      return;
    }
    if (STAGE == APPLY) {  // the parts' sums relative to their largest logit
      const bool on = lane < sp.parts;
      const PartSums ps = sp.part[n * sp.parts + (on ? lane : 0)];
      mt = wave_max(on ? ps.mt : -INFINITY);
      const double d = ps.mt > -INFINITY ? (double)ps.mt - (double)mt : 0.0;
      q[0] = wave_sum(on ? ps.S_t * exp64(d * itau) : 0.0);
      q[1] = TWO ? wave_sum(on ? ps.S_1 * exp64(d) : 0.0) : q[0];
      const SetSums ss = sp.set[n];
      q[2] = ss.E; q[3] = ss.G; q[4] = ss.T_t; q[5] = ss.T_1;
    }
    m = row_max(fmaxf(mj, mt), q[0], q[4]);
    const double wtot = weight_total(g);
    const RowSums r = {q[0], q[1], q[4], q[5], q[2], q[3]};
    const RowOut o = row_scalars<64>(g, r, mt, mj, m, wtot != 0.0 ? (double)wn / wtot : 0.0,
                                     known, (double)sy);
    if (lane == 0) {
      row = o;
      row_mt = mt;
      row_m = m;
      if (part == 0) g.row_loss[n] = m == -INFINITY ? 0.f : (float)o.loss;
    }
  }
  if (STAGE == SUM) return;
  __syncthreads();
  mt = row_mt;
  m = row_m;
  if (!ds) return;
  if (m == -INFINITY) {  // nothing to learn from
    zero_from(STAGE ? part * sp.len : 0);
    return;
  }
  const float mr = mt > -INFINITY ? mt : 0.f;
  const float ct = TWO ? row.c_t : row.c_t + row.c_1, c1 = row.c_1;
  auto gradient = [&](float v) __attribute__((always_inline)) {
    const float z = v - mr;
    float d = ct * exp2_hw(z * c);
    if (TWO) d += c1 * exp2_hw(z * LOG2E);
    return d;
  };
  each([&](const Piece<T>& p, int v0) __attribute__((always_inline)) {
    float d[E];
#pragma unroll
    for (int j = 0; j < E; ++j) d[j] = gradient(p.get(j));
    T* at = reinterpret_cast<T*>(ds0 + v0 * 16 + off);
    if (whole) {
      store_piece(at, d);
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j) st(at + j, d[j]);
    }
  });
  if (odd < hi) st(ds + odd, gradient(xo));
  zero_from(STAGE ? max(part * sp.len, V) : V);
  __syncthreads();
  // then J's classes and the label's
  if (my >= lo && my < hi) {
    const double d = (double)sj - (double)m;
    double q = row.j_q * exp64(d * itau) - row.j_p * exp64(log_e());
    if (known) q += row.j_1 * exp64(d) - (my == y ? row.label : 0.0);
    st(ds + my, (float)q);
  }
  if (tid == 0 && y >= lo && y < hi && !label_in) {
    const double d = (double)sy - (double)mr;
    st(ds + y, (float)((double)row.c_t * exp64(d * itau) + (double)row.c_1 * exp64(d) - row.label));
  }
}

// sum_n w_n L_n in 64 bits: workgroup b of several takes a contiguous share (part), or one workgroup
// everything, or the shares' sums (parts > 0), and divides by the sum of the weights.
__global__ __launch_bounds__(1024) void k_distill_total(DistillGeo g, int64_t share,
                                                        const double* __restrict__ in, int parts,
                                                        double* __restrict__ part,
                                                        float* __restrict__ loss) {
  __shared__ double buf[16];
  double acc = 0.0;
  if (parts > 0) {
    if ((int)threadIdx.x < parts) acc = in[threadIdx.x];
  } else {
    const int64_t a = blockIdx.x * share, b = a + share < g.N ? a + share : g.N;
    for (int64_t n0 = a + threadIdx.x; n0 < b; n0 += 8192) {
      float l[8], w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int64_t n = n0 + 1024 * i;
        l[i] = n < b ? g.row_loss[n] : 0.f;
        w[i] = n < b ? (g.weights ? g.weights[n] : 1.f) : 0.f;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (w[i] != 0.f) acc += (double)w[i] * (double)l[i];
    }
  }
  acc = block_sum<16>(acc, buf);
  if (part) {
    if (threadIdx.x == 0) part[blockIdx.x] = acc;
    return;
  }
  const double wtot = weight_total(g);
  if (threadIdx.x == 0) *loss = wtot != 0.0 ? (float)(acc / wtot) : 0.f;
}

}  // namespace

hipError_t launch_distill_weights(DistillGeo& g, hipStream_t s) {
  const int64_t share = (g.N + DISTILL_WPARTS - 1) / DISTILL_WPARTS;
  const int64_t per = share < 1024 ? 1024 : share;
  g.nwsum = (int32_t)((g.N + per - 1) / per);
  k_distill_weights<<<(unsigned)g.nwsum, 256, 0, s>>>(g.weights, g.N, per, g.wsum);
  return hipGetLastError();
}

namespace {

template <class T, int W, int I>
hipError_t run_small(const DistillGeo& g, const T* logits, T* dlogits, hipStream_t s) {
  // (a launch holds fewer than 2^32 threads)
  constexpr int64_t most = MAX_THREADS / 256;
  for (int64_t first = 0; first < g.N; first += most * (256 / W)) {
    const int64_t blocks = (g.N - first + 256 / W - 1) / (256 / W);
    k_distill_small<T, W, I><<<(unsigned)(blocks < most ? blocks : most), 256, 0, s>>>(
        g, first, logits, dlogits);
  }
  return hipGetLastError();
}

size_t bit_bytes(int32_t classes) { return ((size_t)classes + 63) / 32 * 4; }

template <class T, int TH, int I>
hipError_t run_rows(const DistillGeo& g, const T* logits, T* dlogits, hipStream_t s) {
  constexpr int64_t most = MAX_THREADS / TH;
  const Split none = {};
  for (int64_t first = 0; first < g.N; first += most) {
    const unsigned blocks = (unsigned)(g.N - first < most ? g.N - first : most);
    if (g.labels && g.tau != 1.f)
      k_distill_rows<T, TH, I, true, WHOLE><<<blocks, TH, bit_bytes(g.V), s>>>(g, none, first, logits, dlogits);
    else
      k_distill_rows<T, TH, I, false, WHOLE><<<blocks, TH, bit_bytes(g.V), s>>>(g, none, first, logits, dlogits);
  }
  return hipGetLastError();
}

template <class T, int I>
hipError_t run_split(const DistillGeo& g, const Split& sp, const T* logits, T* dlogits,
                     hipStream_t s) {
  const dim3 grid((unsigned)sp.parts, (unsigned)g.N), more((unsigned)sp.parts + 1, (unsigned)g.N);
  const size_t lds = bit_bytes(sp.len);
  if (g.labels && g.tau != 1.f) {
    k_distill_rows<T, 256, I, true, SUM><<<more, 256, lds, s>>>(g, sp, 0, logits, dlogits);
    k_distill_rows<T, 256, I, true, APPLY><<<grid, 256, lds, s>>>(g, sp, 0, logits, dlogits);
  } else {
    k_distill_rows<T, 256, I, false, SUM><<<more, 256, lds, s>>>(g, sp, 0, logits, dlogits);
    k_distill_rows<T, 256, I, false, APPLY><<<grid, 256, lds, s>>>(g, sp, 0, logits, dlogits);
  }
  return hipGetLastError();
}

// Parts of a row of V classes (1: whole rows): rows that leave CUs idle are split once they are
// long enough to pay for the second launch.  Two workgroups per CU then, of 2,048 classes at least.
int split_parts(int64_t N, int32_t V, int32_t* len) {
  *len = V;
  if (N > SPLIT_ROWS || N < 1 || V < SPLIT_V) return 1;
  int64_t parts = 512 / N;
  if (parts > 64) parts = 64;
  int64_t l = (V + parts - 1) / parts;
  l = (l + 2047) / 2048 * 2048;
  *len = (int32_t)l;
  return (int)((V + l - 1) / l);
}

size_t align16(size_t x) { return (x + 15) / 16 * 16; }

}  // namespace

size_t distill_split_bytes(int64_t N, int32_t V, int32_t k) {
  int32_t len;
  const int parts = split_parts(N, V, &len);
  if (parts == 1) return 0;
  return (size_t)N * (parts * sizeof(PartSums) + sizeof(SetSums)) + align16(N * k * sizeof(SetEntry));
}

template <class T>
hipError_t launch_distill_rows(const DistillGeo& g, const T* logits, T* dlogits, hipStream_t s) {
  if (g.V <= SMALL_V) {
    // the narrowest group that holds the row in one register per lane, a wave from 64 classes on
    if (g.V <= 8) return run_small<T, 8, 1>(g, logits, dlogits, s);
    if (g.V <= 16) return run_small<T, 16, 1>(g, logits, dlogits, s);
    if (g.V <= 32) return run_small<T, 32, 1>(g, logits, dlogits, s);
    if (g.V <= 64) return run_small<T, 64, 1>(g, logits, dlogits, s);
    if (g.V <= 128) return run_small<T, 64, 2>(g, logits, dlogits, s);
    if (g.V <= 256) return run_small<T, 64, 4>(g, logits, dlogits, s);
    if (g.V <= 512) return run_small<T, 64, 8>(g, logits, dlogits, s);
    return run_small<T, 64, 16>(g, logits, dlogits, s);
  }
  constexpr int E = Piece<T>::E;
  const bool whole = !dlogits || ((uintptr_t)dlogits - (uintptr_t)logits) % 16 == 0;
  Split sp;
  sp.parts = split_parts(g.N, g.V, &sp.len);
  if (sp.parts > 1 && whole) {
    sp.part = (PartSums*)g.split;
    sp.set = (SetSums*)(sp.part + g.N * sp.parts);
    sp.entry = (SetEntry*)(sp.set + g.N);
    const int np = sp.len / E;
    if (np <= 256) return run_split<T, 1>(g, sp, logits, dlogits, s);
    if (np <= 512) return run_split<T, 2>(g, sp, logits, dlogits, s);
    if (np <= 1024) return run_split<T, 4>(g, sp, logits, dlogits, s);
    if (np <= 2048) return run_split<T, 8>(g, sp, logits, dlogits, s);
    return run_split<T, 0>(g, sp, logits, dlogits, s);
  }
  // Rows that the registers of a CU do not hold are read three times (512 rows: 65,536 float32 classes
  // 62 us, 65,540 94; 131,072 bfloat16 73, 131,080 88), and so are those whose gradient lies otherwise
  // to 16 bytes, which is then written element by element (8,192 x 5,000 float32 81 us, 263 so).
  // The fewest registers that hold the row, and few threads with many of them: more rows are in
  // flight on a CU, one being read while another is summed or written (4,096 x 50,021 bf16: 256
  // threads with 32 pieces, three rows, 224 us; 512 with 16, two, 244; 1,024 with 8, two, 270).
  const int np = g.V / E;
  if (!whole || np > 16384) return run_rows<T, 1024, 0>(g, logits, dlogits, s);
  if (np <= 256) return run_rows<T, 256, 1>(g, logits, dlogits, s);
  if (np <= 512) return run_rows<T, 256, 2>(g, logits, dlogits, s);
  if (np <= 1024) return run_rows<T, 256, 4>(g, logits, dlogits, s);
  if (np <= 2048) return run_rows<T, 256, 8>(g, logits, dlogits, s);
  if (np <= 4096) return run_rows<T, 256, 16>(g, logits, dlogits, s);
  if (np <= 8192) return run_rows<T, 256, 32>(g, logits, dlogits, s);
  return run_rows<T, 1024, 16>(g, logits, dlogits, s);
}
template hipError_t launch_distill_rows<float>(const DistillGeo&, const float*, float*, hipStream_t);
template hipError_t launch_distill_rows<bf16>(const DistillGeo&, const bf16*, bf16*, hipStream_t);

hipError_t launch_distill_total(const DistillGeo& g, float* loss, hipStream_t s) {
  // one workgroup reads 16,384 losses in about the time that a second launch takes (whole calls over
  // 10 classes: 16,385 rows 13.4 us in shares and 13.6 in one, 65,536 24 and 38, 2^21 470 and 1,070)
  if (g.N <= 16384) {
    k_distill_total<<<1, 1024, 0, s>>>(g, g.N, nullptr, 0, nullptr, loss);
    return hipGetLastError();
  }
  int64_t share = (g.N + DISTILL_WPARTS - 1) / DISTILL_WPARTS;
  if (share < 8192) share = 8192;
  const int parts = (int)((g.N + share - 1) / share);
  k_distill_total<<<(unsigned)parts, 1024, 0, s>>>(g, share, nullptr, 0, g.lsum, loss);
  k_distill_total<<<1, 1024, 0, s>>>(g, share, g.lsum, parts, nullptr, loss);
  return hipGetLastError();
}

}  // namespace tfm
