// Distillation from a teacher's top logits (declarations in vocab.h).
#include "vocab.h"

#include <hip/hip_runtime.h>

namespace tfm {
namespace {

constexpr float LOG2E = 1.44269504088896340736f;

template <class V>
__device__ __forceinline__ V wave_sum(V v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
// Over the NW waves of a workgroup; every thread gets the result.  buf: NW entries.
template <int NW, class V>
__device__ __forceinline__ V block_sum(V v, V* buf) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
  __syncthreads();
  V t = buf[0];
#pragma unroll
  for (int i = 1; i < NW; ++i) t += buf[i];
  return t;
}
template <int NW>
__device__ __forceinline__ float block_max(float v, float* buf) {
  v = wave_max(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
  __syncthreads();
  float t = buf[0];
#pragma unroll
  for (int i = 1; i < NW; ++i) t = fmaxf(t, buf[i]);
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
  return wave_sum(s);
}

// One workgroup per row.
template <class T>
__global__ __launch_bounds__(256) void k_distill_rows(DistillGeo g, const T* logits, T* dlogits) {
  __shared__ uint32_t inside[VOCAB_VMAX / 32];
  __shared__ int32_t jidx[DISTILL_KMAX];   // class of the teacher's entry j, -1: absent
  __shared__ double jp[DISTILL_KMAX];      // its probability
  __shared__ float fbuf[4];
  __shared__ double dbuf[4];
  const int tid = threadIdx.x;
  const double wtot = weight_total(g);
  for (int64_t n = blockIdx.x; n < g.N; n += gridDim.x) {
    __syncthreads();
    const T* s = logits + n * g.ld;
    T* ds = dlogits ? dlogits + n * g.ld : nullptr;
    const float wn = g.weights ? g.weights[n] : 1.f;
    int V = g.V;
    if (g.ncls) V = min(max(g.ncls[n], 0), g.V);
    float m = -INFINITY;
    bool bad = false;
    for (int v = tid; v < V; v += 256) {
      const float x = ld(s + v);
      m = fmaxf(m, x);
      bad |= x != x;
    }
    m = block_max<4>(m, fbuf);
    bad = block_max<4>(bad ? 1.f : 0.f, fbuf) > 0.f;
    if (wn == 0.f || (m == -INFINITY && !bad)) {  // the row is left out
      if (tid == 0) g.row_loss[n] = 0.f;
      if (ds) for (int v = tid; v < g.V; v += 256) st(ds + v, 0.f);
      continue;
    }
    for (int v = tid; v < (g.V + 31) / 32; v += 256) inside[v] = 0;
    // the teacher's entries: the first of a repeated class counts
    int my = -1;
    if (tid < g.k) {
      my = g.idx[n * g.k + tid];
      if (my < 0 || my >= V) my = -1;
    }
    jidx[tid] = my;
    __syncthreads();
    for (int j = 0; j < tid && my >= 0; ++j)
      if (jidx[j] == my) my = -1;
    __syncthreads();
    jidx[tid] = my;
    if (my >= 0 && g.tail) atomicOr(&inside[my >> 5], 1u << (my & 31));
    const double itau = 1.0 / (double)g.tau;
    const double t = my >= 0 ? (double)g.top[n * g.k + tid] : -INFINITY;
    double lp = -INFINITY, p = 0.0;  // log p_j, p_j
    if (g.tail) {
      if (my >= 0) lp = t * itau - (double)g.lse[n];
      p = exp(lp);
    } else {
      const float tm = block_max<4>((float)t, fbuf);
      const double lw = tm == -INFINITY ? -INFINITY : (t - (double)tm) * itau;
      const double z = block_sum<4>(my >= 0 ? exp(lw) : 0.0, dbuf);
      if (z != 0.0 && my >= 0) lp = lw - log(z);
      p = exp(lp);
    }
    if (my < 0) p = 0.0;
    jp[tid] = p;
    const double sumP = block_sum<4>(p, dbuf);
    // the student's sums outside the set (all classes if there is no tail), relative to mt
    float mt = m;
    if (g.tail) {
      mt = -INFINITY;
      for (int v = tid; v < V; v += 256)
        if (!(inside[v >> 5] >> (v & 31) & 1)) mt = fmaxf(mt, ld(s + v));
      mt = block_max<4>(mt, fbuf);
    }
    const bool some = mt > -INFINITY;
    const float c = LOG2E / g.tau;
    float st1 = 0.f, stt = 0.f;
    for (int v = tid; v < V; v += 256) {
      const float x = ld(s + v);
      if (some && !(g.tail && (inside[v >> 5] >> (v & 31) & 1))) {
        stt += exp2f((x - mt) * c);
        st1 += expf(x - mt);
      }
    }
    const double S_t = block_sum<4>((double)stt, dbuf);
    const double S_1 = block_sum<4>((double)st1, dbuf);
    const double sj = my >= 0 ? (double)ld(s + my) : -INFINITY;
    double top_t = 0.0, top_1 = 0.0;
    if (g.tail) {
      top_t = block_sum<4>(my >= 0 ? exp((sj - (double)m) * itau) : 0.0, dbuf);
      top_1 = block_sum<4>(my >= 0 ? exp(sj - (double)m) : 0.0, dbuf);
    }
    // log-sum-exps relative to m
    const double back = some ? (double)mt - (double)m : 0.0;
    const double Zt = (some ? S_t * exp(back * itau) : 0.0) + top_t;
    const double Z1 = (some ? S_1 * exp(back) : 0.0) + top_1;
    const double lZt = log(Zt), lZ1 = log(Z1);
    double D = p > 0.0 || p != p ? p * (lp - ((sj - (double)m) * itau - lZt)) : 0.0;
    D = block_sum<4>(D, dbuf);
    double pt = 0.0;
    if (g.tail && some) {
      pt = 1.0 - sumP;
      if (pt > 0.0) D += pt * (log(pt) - (back * itau + log(S_t) - lZt));
      else if (pt <= 0.0) pt = 0.0;
    }
    int y = -1;
    if (g.labels) y = g.labels[n];
    const bool known = y >= 0 && y < V;
    double L = (double)g.alpha * g.tau * g.tau * D;
    if (known) L += (1.0 - (double)g.alpha) * (lZ1 - ((double)ld(s + y) - (double)m));
    if (bad) L = NAN;
    if (tid == 0) g.row_loss[n] = (float)L;
    if (!ds) continue;
    const double share = wtot != 0.0 ? (double)wn / wtot : 0.0;
    const double cd = (double)g.alpha * g.tau * share, cl = known ? (1.0 - (double)g.alpha) * share : 0.0;
    const float A = (float)(cd * (sumP + pt) / Zt), At = some && pt != 0.0 ? (float)(cd * pt / S_t) : 0.f;
    const float A1 = (float)(cl / Z1);
    // gradients of the entries' classes and the label before anything is written (in place)
    float gj = 0.f;
    if (my >= 0) {
      double e = cd * ((sumP + pt) * exp((sj - (double)m) * itau) / Zt - p);
      if (known) e += cl * (exp(sj - (double)m) / Z1 - (my == y ? 1.0 : 0.0));
      gj = (float)e;
    }
    __syncthreads();
    for (int v = tid; v < g.V; v += 256) {
      float d = 0.f;
      if (v < V) {
        const float x = ld(s + v);
        d = A * exp2f((x - m) * c);
        if (At != 0.f) d -= At * exp2f((x - mt) * c);
        if (known) d += A1 * expf(x - m) - (v == y ? (float)cl : 0.f);
      }
      st(ds + v, d);
    }
    __syncthreads();
    if (my >= 0) st(ds + my, gj);
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

template <class T>
hipError_t launch_distill_rows(const DistillGeo& g, const T* logits, T* dlogits, hipStream_t s) {
  const unsigned blocks = (unsigned)(g.N < 65536 ? g.N : 65536);
  k_distill_rows<T><<<blocks, 256, 0, s>>>(g, logits, dlogits);
  return hipGetLastError();
}
template hipError_t launch_distill_rows<float>(const DistillGeo&, const float*, float*, hipStream_t);
template hipError_t launch_distill_rows<bf16>(const DistillGeo&, const bf16*, bf16*, hipStream_t);

hipError_t launch_distill_total(const DistillGeo& g, float* loss, hipStream_t s) {
  k_distill_total<<<1, 1024, 0, s>>>(g, loss);
  return hipGetLastError();
}

}  // namespace tfm
