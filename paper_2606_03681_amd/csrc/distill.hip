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
// Rows of up to 1,024 classes go to groups of 8 to 64 lanes, longer ones to a workgroup each.
// Bound by HBM (a read and a write of the logits) from some thousand classes on.
#include "mfma.h"
#include "vocab.h"

#include <hip/hip_runtime.h>

namespace tfm {
namespace {

constexpr float LOG2E = 1.44269504088896340736f;

template <int W = 64, class V>
__device__ __forceinline__ V group_sum(V v) {
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
template <int W = 64>
__device__ __forceinline__ float group_max(float v) {
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
// Over the NW waves of a workgroup; every thread gets the result.  buf: NW entries.
template <int NW, class V>
__device__ __forceinline__ V block_sum(V v, V* buf) {
  v = group_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
  __syncthreads();
  V t = buf[0];
#pragma unroll
  for (int i = 1; i < NW; ++i) t += buf[i];
  return t;
}

// Partial sums of the weights in 64 bits: workgroup b sums a contiguous share.
__global__ __launch_bounds__(256) void k_distill_weights(const float* __restrict__ w, int64_t N,
                                                         int64_t share, double* __restrict__ part) {
  __shared__ double buf[4];
  const int64_t a = blockIdx.x * share, b = a + share < N ? a + share : N;
  double acc = 0.0;
  for (int64_t n = a + threadIdx.x; n < b; n += 256) acc += (double)w[n];
  acc = block_sum<4>(acc, buf);
  if (threadIdx.x == 0) part[blockIdx.x] = acc;
}

// Sum of the weights from its parts (N where there are none); every lane of the wave gets it.
__device__ __forceinline__ double weight_total(const DistillGeo& g) {
  if (!g.weights) return (double)g.N;
  double s = 0.0;
  for (int i = threadIdx.x & 63; i < g.nwsum; i += 64) s += g.wsum[i];
  return group_sum(s);
}

__device__ __forceinline__ int row_classes(const DistillGeo& g, int64_t n) {
  return g.ncls ? min(max(g.ncls[n], 0), g.V) : g.V;
}

// The row's scalars from its sums, relative to its largest logit m:
//   S_t, S_1    sums of exp((s - mt) / tau) and exp(s - mt) outside J
//   T_t, T_1    sums of exp((s - m) / tau) and exp(s - m) over J (0 without a tail)
//   E, G        sums over J of e_j and e_j (log e_j - (s_j - m) / tau), where p_j = e_j / E without
//               a tail and e_j with one
struct RowSums {
  double S_t, S_1, T_t, T_1, E, G;
};
struct RowOut {
  double loss;
  double j_q, j_1;    // gradient of class j in J: j_q exp((s_j - m) / tau) + j_1 exp(s_j - m)
  double j_p, label;  //   - j_p e_j, and of the label: - label
  float c_t, c_1;     // gradient outside J: c_t exp((s - mt) / tau) + c_1 exp(s - mt)
};
__device__ __forceinline__ RowOut row_scalars(const DistillGeo& g, const RowSums& r, float mt,
                                              float m, double share, bool known, double s_label) {
  const double tau = g.tau, alpha = g.alpha, itau = 1.0 / tau;
  const bool some = mt > -INFINITY;
  const double back = some ? (double)mt - (double)m : 0.0;
  const double bt = exp(back * itau), b1 = exp(back);
  const double Zt = r.S_t * bt + r.T_t, Z1 = r.S_1 * b1 + r.T_1;
  const double lZt = log(Zt);
  // the teacher's mass: P in the set, pt outside
  const double norm = g.tail || r.E == 0.0 ? 1.0 : 1.0 / r.E;
  double P = r.E * norm, pt = 0.0;
  double D = r.G * norm + lZt * P;
  if (!g.tail && r.E != 0.0) D -= log(r.E);
  if (g.tail && some) {
    pt = 1.0 - P;
    if (pt > 0.0) D += pt * (log(pt) - (back * itau + log(r.S_t) - lZt));
    else if (pt <= 0.0) pt = 0.0;
  }
  RowOut o;
  o.loss = alpha > 0.0 ? alpha * tau * tau * D : 0.0;
  const double cd = alpha * tau * share, cl = known ? (1.0 - alpha) * share : 0.0;
  if (known) o.loss += (1.0 - alpha) * (log(Z1) - (s_label - (double)m));
  o.j_q = cd * (P + pt) / Zt;
  o.j_1 = cl / Z1;
  o.j_p = cd * norm;
  o.label = cl;
  o.c_t = (float)(o.j_q * bt - (pt > 0.0 ? cd * pt / r.S_t : 0.0));
  o.c_1 = (float)(o.j_1 * b1);
  return o;
}

// ---- rows of up to 1,024 classes ----------------------------------------------------------------
// W lanes to a row, class lane + W i in register i.
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
  const bool left_out = wn == 0.f || m == -INFINITY;
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
      const double d = (double)x[i] - (double)m, y = d * itau;
      double lt;
      if (g.tail) {
        lt = (double)t[i] * itau - lse;
        r.T_t += exp(y);
        r.T_1 += exp(d);
      } else {
        lt = tm > -INFINITY ? ((double)t[i] - (double)tm) * itau : -INFINITY;
      }
      if (t[i] != t[i]) lt = NAN;
      e[i] = exp(lt);
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
  const int y = g.labels ? g.labels[n] : -1;
  const bool known = y >= 0 && y < V;
  float sy = -INFINITY;
#pragma unroll
  for (int i = 0; i < I; ++i)
    if (lane + W * i == y) sy = x[i];
  sy = __shfl(sy, known ? y % W : 0, W);
  const double share = wtot != 0.0 ? (double)wn / wtot : 0.0;
  const RowOut o = row_scalars(g, r, mt, m, share, known, (double)sy);
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
          double q = o.j_q * exp(dx * itau) - o.j_p * e[i];
          if (known) q += o.j_1 * exp(dx) - (v == y ? o.label : 0.0);
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

// ---- longer rows ---------------------------------------------------------------------------------
// A row in pieces of 16 bytes on 16-byte boundaries; its first class may lie `skip` elements into
// the first piece.
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

// Classes e0 .. of a row of V; -inf where there are none.
template <class T>
__device__ __forceinline__ Piece<T> load_piece(const T* s, int e0, int V) {
  Piece<T> p;
  if (e0 >= 0 && e0 + Piece<T>::E <= V) {
    p.u = *reinterpret_cast<const uint4*>(s + e0);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if constexpr (sizeof(T) == 4) {
        const int e = e0 + q;
        w[q] = e >= 0 && e < V ? __float_as_uint(s[e]) : 0xff800000u;
      } else {
        const int e = e0 + 2 * q;
        const uint32_t lo = e >= 0 && e < V ? s[e] : 0xff80u;
        const uint32_t hi = e + 1 >= 0 && e + 1 < V ? s[e + 1] : 0xff80u;
        w[q] = lo | hi << 16;
      }
    }
    p.u = make_uint4(w[0], w[1], w[2], w[3]);
  }
  return p;
}
template <class T>
__device__ __forceinline__ void store_piece(T* ds, int e0, int V, bool whole, const float* d) {
  constexpr int E = Piece<T>::E;
  if (whole && e0 >= 0 && e0 + E <= V) {
    if constexpr (sizeof(T) == 4)
      *reinterpret_cast<float4*>(ds + e0) = make_float4(d[0], d[1], d[2], d[3]);
    else
      *reinterpret_cast<uint4*>(ds + e0) =
          make_uint4(pack2(d[0], d[1]), pack2(d[2], d[3]), pack2(d[4], d[5]), pack2(d[6], d[7]));
  } else {
#pragma unroll
    for (int j = 0; j < E; ++j)
      if (e0 + j >= 0 && e0 + j < V) st(ds + e0 + j, d[j]);
  }
}

// One workgroup of TH threads per row, I pieces per thread in registers (I = 0: read again for each
// of the three passes: rows that the registers of a CU do not hold).  TWO: the label's softmax has
// another temperature than the teacher's, a second exponential per class.
template <class T, int TH, int I, bool TWO>
__global__ __launch_bounds__(TH) void k_distill_rows(DistillGeo g, int64_t first, const T* logits,
                                                     T* dlogits) {
  constexpr int E = Piece<T>::E, NW = TH / 64;
  extern __shared__ uint32_t inside[];  // a bit per class from the first piece on: in J
  __shared__ int32_t jidx[DISTILL_KMAX];
  __shared__ float fbuf[3][NW];
  __shared__ double dbuf[6][NW];
  __shared__ RowOut row;
  __shared__ int again, label_in;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const double itau = 1.0 / (double)g.tau;
  const float c = LOG2E / g.tau;
  const int64_t n = first + blockIdx.x;
  const T* s = logits + n * g.ld;
  T* ds = dlogits ? dlogits + n * g.ld : nullptr;
  const float wn = g.weights ? g.weights[n] : 1.f;
  const int V = row_classes(g, n);
  const int skip = (int)((uintptr_t)s % 16 / sizeof(T));
  const int np = (g.V + skip + E - 1) / E;
  // in whole pieces too where they lie as the logits' do
  const bool whole = ds && (uintptr_t)ds % 16 == (uintptr_t)s % 16;
  float zero[E] = {};
  if (wn == 0.f || V == 0) {
    if (ds)
      for (int v = tid; v < np; v += TH) store_piece(ds, v * E - skip, g.V, whole, zero);
    if (tid == 0) g.row_loss[n] = 0.f;
    return;
  }
  // the teacher's entries first, the row behind them
  int my = -1;
  float tj = -INFINITY;
  if (tid < g.k) {
    my = g.idx[n * g.k + tid];
    tj = g.top[n * g.k + tid];
    if (my < 0 || my >= V) my = -1;
  }
  const int y = g.labels ? g.labels[n] : -1;
  const bool known = y >= 0 && y < V;
  const float sj = my >= 0 ? ld(s + my) : -INFINITY;
  const float sy = known ? ld(s + y) : -INFINITY;
  Piece<T> x[I > 0 ? I : 1];
  if constexpr (I > 0) {
#pragma unroll
    for (int i = 0; i < I; ++i)
      if (i * TH + tid < np) x[i] = load_piece(s, (i * TH + tid) * E - skip, V);
  }
  auto each = [&](auto f) __attribute__((always_inline)) {
    if constexpr (I > 0) {
#pragma unroll
      for (int i = 0; i < I; ++i)
        if (i * TH + tid < np) f(x[i], i * TH + tid);
    } else {
      for (int v = tid; v < np; v += TH) f(load_piece(s, v * E - skip, V), v);
    }
  };
  for (int v = tid; v < (np * E + 31) / 32; v += TH) inside[v] = 0;
  if (tid == 0) again = label_in = 0;
  if (tid < DISTILL_KMAX) jidx[tid] = my;
  __syncthreads();
  if (my >= 0) {
    const uint32_t bit = 1u << ((my + skip) & 31);
    if (atomicOr(&inside[(my + skip) >> 5], bit) & bit) again = 1;
    if (my == y) label_in = 1;
  }
  __syncthreads();
  if (again) {  // a repeated class: its first entry counts
    for (int j = 0; j < tid && my >= 0; ++j)
      if (jidx[j] == my) my = -1;
  }
  if (my < 0) tj = -INFINITY;
  // bits of piece v's classes that the sums leave out
  auto out_of = [&](int v) __attribute__((always_inline)) -> uint32_t {
    if (!g.tail) return 0u;
    const uint32_t byte = reinterpret_cast<const uint8_t*>(inside)[v * E >> 3];
    return E == 8 ? byte : byte >> (v & 1) * 4 & 15u;
  };
  // maxima: of the classes that are summed, of J's logits, of the teacher's
  float mt = -INFINITY;
  each([&](const Piece<T>& p, int v) __attribute__((always_inline)) {
    const uint32_t o = out_of(v);
    if (o == 0) {
#pragma unroll
      for (int j = 0; j < E; ++j) mt = fmaxf(mt, p.get(j));
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j) mt = fmaxf(mt, o >> j & 1 ? -INFINITY : p.get(j));
    }
  });
  mt = group_max(mt);
  const float mj = group_max(my >= 0 ? sj : -INFINITY), tj_m = group_max(tj);
  if (lane == 0) {
    fbuf[0][w] = mt;
    fbuf[1][w] = mj;
    fbuf[2][w] = tj_m;
  }
  __syncthreads();
  // (a lane per wave's value: NW of them held at once would cost the registers of the row)
  mt = group_max<NW>(fbuf[0][lane % NW]);
  float m = group_max<NW>(fbuf[1][lane % NW]);
  const float tm = group_max<NW>(fbuf[2][lane % NW]);
  m = fmaxf(m, mt);
  if (m == -INFINITY) {  // nothing to learn from
    if (ds)
      for (int v = tid; v < np; v += TH) store_piece(ds, v * E - skip, g.V, whole, zero);
    if (tid == 0) g.row_loss[n] = 0.f;
    return;
  }
  const float mr = mt > -INFINITY ? mt : 0.f;
  // sums
  float sum_t = 0.f, sum_1 = 0.f;
  each([&](const Piece<T>& p, int v) __attribute__((always_inline)) {
    const uint32_t o = out_of(v);
#pragma unroll
    for (int j = 0; j < E; ++j) {
      const float d = (o >> j & 1 ? -INFINITY : p.get(j)) - mr;
      sum_t += exp2_hw(d * c);
      if (TWO) sum_1 += exp2_hw(d * LOG2E);
    }
  });
  double e = 0.0, xj = 0.0, ex_t = 0.0, ex_1 = 0.0, G = 0.0;
  if (w * 64 < g.k) {  // the waves that hold entries
    if (my >= 0) {
      const double d = (double)sj - (double)m;
      xj = d * itau;
      double lt;
      if (g.tail) lt = (double)tj * itau - (double)g.lse[n];
      else lt = tm > -INFINITY ? ((double)tj - (double)tm) * itau : -INFINITY;
      if (tj != tj) lt = NAN;
      e = exp(lt);
      ex_t = exp(xj);
      ex_1 = exp(d);
      if (!(e == 0.0)) G = e * (lt - xj);
    }
    const double q[4] = {group_sum(e), group_sum(G), group_sum(ex_t), group_sum(ex_1)};
    if (lane == 0)
#pragma unroll
      for (int i = 0; i < 4; ++i) dbuf[2 + i][w] = q[i];
  } else if (lane == 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) dbuf[2 + i][w] = 0.0;
  }
  const double S = group_sum((double)sum_t), S1 = TWO ? group_sum((double)sum_1) : S;
  if (lane == 0) {
    dbuf[0][w] = S;
    dbuf[1][w] = S1;
  }
  __syncthreads();
  if (w == 0) {
    double q[6];
#pragma unroll
    for (int i = 0; i < 6; ++i) q[i] = group_sum<NW>(dbuf[i][lane % NW]);
    const double wtot = weight_total(g);
    const RowSums r = {q[0], q[1], g.tail ? q[4] : 0.0, g.tail ? q[5] : 0.0, q[2], q[3]};
    const RowOut o = row_scalars(g, r, mt, m, wtot != 0.0 ? (double)wn / wtot : 0.0, known,
                                 (double)sy);
    if (lane == 0) {
      row = o;
      g.row_loss[n] = (float)o.loss;
    }
  }
  __syncthreads();
  if (ds) {
    const float ct = TWO ? row.c_t : row.c_t + row.c_1, c1 = row.c_1;
    each([&](const Piece<T>& p, int v) __attribute__((always_inline)) {
      float d[E];
#pragma unroll
      for (int j = 0; j < E; ++j) {
        const float z = p.get(j) - mr;
        d[j] = ct * exp2_hw(z * c);
        if (TWO) d[j] += c1 * exp2_hw(z * LOG2E);
      }
      store_piece(ds, v * E - skip, g.V, whole, d);
    });
    __syncthreads();
    // then J's classes and the label's
    if (my >= 0) {
      const double q = row.j_q * ex_t + row.j_1 * ex_1 - row.j_p * e - (my == y ? row.label : 0.0);
      st(ds + my, (float)q);
    }
    if (tid == 0 && known && !label_in) {
      const double d = (double)sy - (double)mr;
      st(ds + y, (float)((double)row.c_t * exp(d * itau) + (double)row.c_1 * exp(d) - row.label));
    }
  }
}

// loss = sum_n w_n L_n / sum_n w_n in 64 bits, one workgroup.
__global__ __launch_bounds__(1024) void k_distill_total(DistillGeo g, float* __restrict__ loss) {
  __shared__ double buf[16];
  double acc = 0.0;
  for (int64_t n = threadIdx.x; n < g.N; n += 1024) {
    const double w = g.weights ? (double)g.weights[n] : 1.0;
    if (w != 0.0) acc += w * (double)g.row_loss[n];
  }
  acc = block_sum<16>(acc, buf);
  const double wtot = weight_total(g);
  if (threadIdx.x == 0) *loss = wtot != 0.0 ? (float)(acc / wtot) : 0.f;
}

}  // namespace

hipError_t launch_distill_weights(DistillGeo& g, hipStream_t s) {
  const int64_t share = (g.N + DISTILL_WPARTS - 1) / DISTILL_WPARTS;
  const int64_t per = share < 4096 ? 4096 : share;
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

template <class T, int TH, int I>
hipError_t run_rows(const DistillGeo& g, const T* logits, T* dlogits, hipStream_t s) {
  constexpr int64_t most = MAX_THREADS / TH;
  const size_t lds = ((size_t)g.V + 64) / 32 * 4;
  for (int64_t first = 0; first < g.N; first += most) {
    const unsigned blocks = (unsigned)(g.N - first < most ? g.N - first : most);
    if (g.labels && g.tau != 1.f)
      k_distill_rows<T, TH, I, true><<<blocks, TH, lds, s>>>(g, first, logits, dlogits);
    else
      k_distill_rows<T, TH, I, false><<<blocks, TH, lds, s>>>(g, first, logits, dlogits);
  }
  return hipGetLastError();
}

}  // namespace

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
  // the fewest threads and registers that hold the row
  constexpr int E = Piece<T>::E;
  // pieces: at the rows' alignment, or at the worst if it changes from row to row
  const int skip = g.ld % E == 0 ? (int)((uintptr_t)logits % 16 / sizeof(T)) : E - 1;
  const int np = (g.V + skip + E - 1) / E;
  if (np <= 256) return run_rows<T, 256, 1>(g, logits, dlogits, s);
  if (np <= 512) return run_rows<T, 256, 2>(g, logits, dlogits, s);
  if (np <= 1024) return run_rows<T, 256, 4>(g, logits, dlogits, s);
  if (np <= 2048) return run_rows<T, 256, 8>(g, logits, dlogits, s);
  if (np <= 4096) return run_rows<T, 512, 8>(g, logits, dlogits, s);
  if (np <= 8192) return run_rows<T, 1024, 8>(g, logits, dlogits, s);
  if (np <= 16384) return run_rows<T, 1024, 16>(g, logits, dlogits, s);
  return run_rows<T, 1024, 0>(g, logits, dlogits, s);
}
template hipError_t launch_distill_rows<float>(const DistillGeo&, const float*, float*, hipStream_t);
template hipError_t launch_distill_rows<bf16>(const DistillGeo&, const bf16*, bf16*, hipStream_t);

hipError_t launch_distill_total(const DistillGeo& g, float* loss, hipStream_t s) {
  k_distill_total<<<1, 1024, 0, s>>>(g, loss);
  return hipGetLastError();
}

}  // namespace tfm
