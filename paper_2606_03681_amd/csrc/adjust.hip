// Penalties, biases and masks on logits (declarations in vocab.h).
//
// A workgroup takes a slice of a row's classes, or several rows of few classes.  What is said about
// single classes is gathered in LDS first, a word of how often the class occurs in the history and one
// of its first bias entry (integers: no order matters), then one pass over the logits applies it.  A
// slice whose row has neither history nor biases has no such words.
#include "mfma.h"
#include "vocab.h"

namespace tfm {
namespace {

constexpr int SLICE = 4096, kMaxBlocks = 1 << 23;
constexpr uint32_t NONE = 0xffffffffu;

// 16 bytes of logits: V of them.
template <class T>
struct Vec {
  static constexpr int V = 16 / sizeof(T);
  uint32_t w[4];
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
};

// One class: x, how often it was seen, its bias entry, whether it is allowed.
struct Rule {
  float r, pres, freq;
};
__device__ __forceinline__ float adjusted(float x, uint32_t seen, uint32_t first, const float* bias,
                                          const Rule& u) {
#pragma clang fp contract(off)
  if (seen) {
    x = x > 0.f ? x / u.r : x * u.r;
    x = x - (u.pres + u.freq * (float)seen);
  }
  if (first != NONE) x = x + bias[first];
  return x;
}
__device__ __forceinline__ Rule rule_of(const AdjustGeo& g, int64_t n) {
  Rule u;
  u.r = g.repetition ? g.repetition[n] : 1.f;
  if (!(u.r > 0.f)) u.r = 1.f;
  u.pres = g.presence ? g.presence[n] : 0.f;
  u.freq = g.frequency ? g.frequency[n] : 0.f;
  return u;
}
__device__ __forceinline__ int classes_of(const AdjustGeo& g, int64_t n) {
  return g.ncls ? min(max(g.ncls[n], 0), g.V) : g.V;
}
__device__ __forceinline__ int said_of(const AdjustGeo& g, int64_t n) {
  return !g.history ? 0 : g.n_history ? min(max(g.n_history[n], 0), g.n_hist) : g.n_hist;
}

// A slice of one row.  WIDE: rows start at multiples of 16 bytes.
template <class T, bool WIDE>
__global__ __launch_bounds__(256) void k_adjust(AdjustGeo g, const T* logits, T* out, int slices,
                                                int64_t items) {
  __shared__ __attribute__((aligned(16))) uint32_t seen[SLICE], first[SLICE];
  constexpr int V = Vec<T>::V;
  const int tid = threadIdx.x;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t n = it / slices;
    const int v0 = (int)(it - n * slices) * SLICE, w = min(SLICE, g.V - v0);
    const int m = said_of(g, n), nb = g.n_bias;
    const bool any = m > 0 || nb > 0;
    const Rule u = rule_of(g, n);
    const int nc = classes_of(g, n);
    if (any) {
      __syncthreads();
      for (int i = 4 * tid; i < w; i += 1024) {
        *reinterpret_cast<uint4*>(seen + i) = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4*>(first + i) = make_uint4(NONE, NONE, NONE, NONE);
      }
      __syncthreads();
      const int32_t* h = g.history + n * g.ld_history;
      for (int j0 = 0; j0 < m; j0 += 2048) {
        uint32_t v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int j = j0 + i * 256 + tid;
          v[i] = j < m ? (uint32_t)h[j] - (uint32_t)v0 : NONE;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (v[i] < (uint32_t)w) atomicAdd(&seen[v[i]], 1u);
      }
      for (int j = tid; j < nb; j += 256) {
        const uint32_t v = (uint32_t)g.bias_idx[n * g.ld_bias + j] - (uint32_t)v0;
        if (v < (uint32_t)w) atomicMin(&first[v], (uint32_t)j);
      }
      __syncthreads();
    }
    const T* from = logits + n * g.ld + v0;
    T* to = out + n * g.ld_out + v0;
    const float* bias = g.bias + n * g.ld_bias;
    const uint32_t* mask = g.allowed ? g.allowed + n * g.ld_allowed + v0 / 32 : nullptr;
    const int here = nc - v0;  // classes of the slice that count
    if constexpr (WIDE) {
      for (int i = tid * V; i < w; i += 256 * V) {
        const uint32_t bits = mask ? mask[i / 32] >> (i % 32) : NONE;
        if (i + V <= w) {
          Vec<T> x;
          const uint4 z = *reinterpret_cast<const uint4*>(from + i);
          x.w[0] = z.x; x.w[1] = z.y; x.w[2] = z.z; x.w[3] = z.w;
          float y[V];
#pragma unroll
          for (int j = 0; j < V; ++j) y[j] = x.get(j);
          if (any) {
            uint32_t s[V], f[V];
#pragma unroll
            for (int j = 0; j < V; j += 4) {
              const uint4 a = *reinterpret_cast<const uint4*>(seen + i + j);
              const uint4 b = *reinterpret_cast<const uint4*>(first + i + j);
              s[j] = a.x; s[j + 1] = a.y; s[j + 2] = a.z; s[j + 3] = a.w;
              f[j] = b.x; f[j + 1] = b.y; f[j + 2] = b.z; f[j + 3] = b.w;
            }
#pragma unroll
            for (int j = 0; j < V; ++j)
              if (s[j] || f[j] != NONE) y[j] = adjusted(y[j], s[j], f[j], bias, u);
          }
#pragma unroll
          for (int j = 0; j < V; ++j)
            if (!(bits >> j & 1) || i + j >= here) y[j] = -INFINITY;
          uint4 o;
          if constexpr (sizeof(T) == 4)
            o = make_uint4(__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]),
                           __float_as_uint(y[3]));
          else
            o = make_uint4(pack2(y[0], y[1]), pack2(y[2], y[3]), pack2(y[4], y[5]), pack2(y[6], y[7]));
          *reinterpret_cast<uint4*>(to + i) = o;
        } else {
          for (int j = 0; i + j < w; ++j) {
            float y = ld(from + i + j);
            if (any) y = adjusted(y, seen[i + j], first[i + j], bias, u);
            st(to + i + j, (bits >> j & 1) && i + j < here ? y : -INFINITY);
          }
        }
      }
    } else {
      for (int i = tid; i < w; i += 256) {
        float y = ld(from + i);
        if (any) y = adjusted(y, seen[i], first[i], bias, u);
        const bool ok = i < here && (!mask || mask[i / 32] >> (i % 32) & 1);
        st(to + i, ok ? y : -INFINITY);
      }
    }
  }
}

// R whole rows, R V <= SLICE.
template <class T>
__global__ __launch_bounds__(256) void k_adjust_rows(AdjustGeo g, const T* logits, T* out, int R,
                                                     int64_t items) {
  __shared__ uint32_t seen[SLICE], first[SLICE];
  const int tid = threadIdx.x, V = g.V;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t n0 = it * R;
    const int rows = (int)min((int64_t)R, g.N - n0), w = rows * V;
    const bool any = g.n_hist > 0 || g.n_bias > 0;
    if (any) {
      __syncthreads();
      for (int i = tid; i < w; i += 256) seen[i] = 0, first[i] = NONE;
      __syncthreads();
      if (g.history) {
        for (int64_t i = tid; i < (int64_t)rows * g.n_hist; i += 256) {
          const int r = (int)(i / g.n_hist), j = (int)(i - (int64_t)r * g.n_hist);
          if (j >= said_of(g, n0 + r)) continue;
          const uint32_t v = (uint32_t)g.history[(n0 + r) * g.ld_history + j];
          if (v < (uint32_t)V) atomicAdd(&seen[r * V + v], 1u);
        }
      }
      for (int64_t i = tid; i < (int64_t)rows * g.n_bias; i += 256) {
        const int r = (int)(i / g.n_bias), j = (int)(i - (int64_t)r * g.n_bias);
        const uint32_t v = (uint32_t)g.bias_idx[(n0 + r) * g.ld_bias + j];
        if (v < (uint32_t)V) atomicMin(&first[r * V + v], (uint32_t)j);
      }
      __syncthreads();
    }
    for (int i = tid; i < w; i += 256) {
      const int r = i / V, v = i - r * V;
      const int64_t n = n0 + r;
      float y = ld(logits + n * g.ld + v);
      if (any) y = adjusted(y, seen[i], first[i], g.bias + n * g.ld_bias, rule_of(g, n));
      const bool ok = v < classes_of(g, n) &&
                      (!g.allowed || g.allowed[n * g.ld_allowed + v / 32] >> (v % 32) & 1);
      st(out + n * g.ld_out + v, ok ? y : -INFINITY);
    }
  }
}

}  // namespace

template <class T>
hipError_t launch_adjust(const AdjustGeo& g, const T* logits, T* out, hipStream_t s) {
  if (g.V <= SLICE / 4) {
    const int R = SLICE / 4 / g.V < 64 ? SLICE / 4 / g.V : 64;
    const int64_t items = (g.N + R - 1) / R;
    k_adjust_rows<T><<<(unsigned)(items < kMaxBlocks ? items : kMaxBlocks), 256, 0, s>>>(
        g, logits, out, R, items);
    return hipGetLastError();
  }
  const int slices = (g.V + SLICE - 1) / SLICE;
  const int64_t items = g.N * slices;
  const unsigned blocks = (unsigned)(items < kMaxBlocks ? items : kMaxBlocks);
  const bool wide = (uintptr_t)logits % 16 == 0 && (uintptr_t)out % 16 == 0 &&
                    g.ld * sizeof(T) % 16 == 0 && g.ld_out * sizeof(T) % 16 == 0;
  if (wide)
    k_adjust<T, true><<<blocks, 256, 0, s>>>(g, logits, out, slices, items);
  else
    k_adjust<T, false><<<blocks, 256, 0, s>>>(g, logits, out, slices, items);
  return hipGetLastError();
}
template hipError_t launch_adjust(const AdjustGeo&, const float*, float*, hipStream_t);
template hipError_t launch_adjust(const AdjustGeo&, const bf16*, bf16*, hipStream_t);

}  // namespace tfm
