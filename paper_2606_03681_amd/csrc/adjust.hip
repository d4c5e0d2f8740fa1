// Penalties, biases and masks on logits (declarations in vocab.h).
//
// A workgroup takes a slice of a row's classes, or several rows of few classes.  What is said about
// single classes is gathered in LDS first, then one pass over the logits, which are on their way
// meanwhile, applies it: for each class a word with how often it occurs in the history (low half) and
// the complement of its first bias entry (high half), or two words where either may not fit 16 bits.
// Integers: no order matters.  A slice whose row has neither history nor biases has no such words.
//
// Bound: HBM for long rows without much to note, else latency.  64 rows of 131,072 bfloat16 classes,
// each with up to 8192 earlier tokens, 32 biases and a mask: 20 us (7 of bytes; each of a row's 32 slices
// reads its whole history, from the caches, and counts with atomics in LDS); one row of 32,000 float32
// classes: 6 us, launch and three dependent loads.  With two words for each class in all cases (half as
// many workgroups to a CU) and the logits read behind the notes the 64 rows took 28 us.  Eight waves a
// SIMD leave 64 registers: whole float32 rows spill 24 (100 bytes of scratch a lane), bfloat16 ones 4; 64
// float32 rows of 131,072 with 8192 tokens each take 32 us (20 without; bfloat16 24 and 7).
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

// Notes about the classes of a slice: PACK, one word each.
template <bool PACK>
struct Notes {
  uint32_t* seen;   // PACK: both halves
  uint32_t* first;  // else
  __device__ __forceinline__ void bias(uint32_t v, int j) const {  // before count()
    if (PACK)
      atomicMax(&seen[v], (0xffffu - (uint32_t)j) << 16);
    else
      atomicMin(&first[v], (uint32_t)j);
  }
  __device__ __forceinline__ void count(uint32_t v) const { atomicAdd(&seen[v], 1u); }
  // how often class i occurs, and its first entry or NONE
  static __device__ __forceinline__ void split(uint32_t a, uint32_t b, uint32_t& n, uint32_t& j) {
    n = PACK ? a & 0xffffu : a;
    j = PACK ? (a >> 16 ? 0xffffu - (a >> 16) : NONE) : b;
  }
};

// A slice of one row.  WIDE: rows start at multiples of 16 bytes.
template <class T, bool WIDE, bool PACK>
__global__ __launch_bounds__(256, PACK ? 8 : 4) void k_adjust(AdjustGeo g, const T* logits, T* out, int slices,
                                                int64_t items) {
  __shared__ __attribute__((aligned(16))) uint32_t words[PACK ? SLICE : 2 * SLICE];
  constexpr int V = Vec<T>::V, NV = SLICE / (256 * V);
  const Notes<PACK> notes{words, words + (PACK ? 0 : SLICE)};
  const int tid = threadIdx.x;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t n = it / slices;
    const int v0 = (int)(it - n * slices) * SLICE, w = min(SLICE, g.V - v0);
    const T* from = logits + n * g.ld + v0;
    T* to = out + n * g.ld_out + v0;
    uint4 x[NV];
    uint32_t bits[NV];
    const uint32_t* mask = g.allowed ? g.allowed + n * g.ld_allowed + v0 / 32 : nullptr;
    if constexpr (WIDE) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int i = (k * 256 + tid) * V;
        if (i + V <= w) x[k] = *reinterpret_cast<const uint4*>(from + i);
        bits[k] = mask && i < w ? mask[i / 32] : NONE;
      }
    }
    const int m = said_of(g, n), nb = g.n_bias;
    const bool any = m > 0 || nb > 0;
    const Rule u = rule_of(g, n);
    const int nc = classes_of(g, n);
    if (any) {
      const int32_t* h = g.history + n * g.ld_history;
      uint32_t v[8];
      auto ask = [&](int j0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int j = j0 + i * 256 + tid;
          v[i] = j < m ? (uint32_t)h[j] - (uint32_t)v0 : NONE;
        }
      };
      ask(0);
      __syncthreads();  // the last slice's notes have been read
      for (int i = 4 * tid; i < (PACK ? w : SLICE + w); i += 1024) {
        const uint32_t z = PACK || i < SLICE ? 0 : NONE;
        *reinterpret_cast<uint4*>(words + i) = make_uint4(z, z, z, z);
      }
      __syncthreads();
      if (nb > 0) {
        for (int j = tid; j < nb; j += 256) {
          const uint32_t c = (uint32_t)g.bias_idx[n * g.ld_bias + j] - (uint32_t)v0;
          if (c < (uint32_t)w) notes.bias(c, j);
        }
        if (PACK) __syncthreads();
      }
      for (int j0 = 0; j0 < m;) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (v[i] < (uint32_t)w) notes.count(v[i]);
        j0 += 2048;
        if (j0 < m) ask(j0);
      }
      __syncthreads();
    }
    const float* bias = g.bias + n * g.ld_bias;
    const int here = nc - v0;  // classes of the slice that count
    if constexpr (WIDE) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int i = (k * 256 + tid) * V;
        if (i >= w) break;
        const uint32_t b = bits[k] >> (i % 32);
        if (i + V <= w) {
          Vec<T> z;
          z.w[0] = x[k].x; z.w[1] = x[k].y; z.w[2] = x[k].z; z.w[3] = x[k].w;
          float y[V];
#pragma unroll
          for (int j = 0; j < V; ++j) y[j] = z.get(j);
          if (any) {
            uint32_t s[V], f[V], some = 0;
#pragma unroll
            for (int j = 0; j < V; j += 4) {
              const uint4 a = *reinterpret_cast<const uint4*>(notes.seen + i + j);
              s[j] = a.x; s[j + 1] = a.y; s[j + 2] = a.z; s[j + 3] = a.w;
              some |= a.x | a.y | a.z | a.w;
              if constexpr (!PACK) {
                const uint4 c = *reinterpret_cast<const uint4*>(notes.first + i + j);
                f[j] = c.x; f[j + 1] = c.y; f[j + 2] = c.z; f[j + 3] = c.w;
                some |= ~(c.x & c.y & c.z & c.w);
              }
            }
            if (some) {
#pragma unroll
              for (int j = 0; j < V; ++j) {
                uint32_t count, first;
                notes.split(s[j], PACK ? 0 : f[j], count, first);
                if (count || first != NONE) y[j] = adjusted(y[j], count, first, bias, u);
              }
            }
          }
#pragma unroll
          for (int j = 0; j < V; ++j)
            if (!(b >> j & 1) || i + j >= here) y[j] = -INFINITY;
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
            if (any) {
              uint32_t count, first;
              notes.split(notes.seen[i + j], PACK ? 0 : notes.first[i + j], count, first);
              y = adjusted(y, count, first, bias, u);
            }
            st(to + i + j, (b >> j & 1) && i + j < here ? y : -INFINITY);
          }
        }
      }
    } else {
      for (int i = tid; i < w; i += 256) {
        float y = ld(from + i);
        if (any) {
          uint32_t count, first;
          notes.split(notes.seen[i], PACK ? 0 : notes.first[i], count, first);
          y = adjusted(y, count, first, bias, u);
        }
        const bool ok = i < here && (!mask || mask[i / 32] >> (i % 32) & 1);
        st(to + i, ok ? y : -INFINITY);
      }
    }
  }
}

// R whole rows, R V <= SLICE / 4 and, where R > 1, R n_hist and R n_bias at most SLICE.
constexpr int MOST_ROWS = 64;
template <class T>
__global__ __launch_bounds__(256) void k_adjust_rows(AdjustGeo g, const T* logits, T* out, int R,
                                                     int64_t items) {
  __shared__ uint32_t seen[SLICE / 4], first[SLICE / 4];
  __shared__ int said[MOST_ROWS];
  const int tid = threadIdx.x, V = g.V;
  // f(r, j) for j < n of each row r, four loads of it under way at a time; then(r, j, its value)
  auto each = [&](int rows, uint32_t n, auto f, auto then) {
    const uint32_t total = rows * n;
    for (uint32_t i0 = tid; i0 < total; i0 += 1024) {
      uint32_t r[4], v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t i = min(i0 + k * 256, total - 1);
        r[k] = i / n;
        v[k] = f(r[k], i - r[k] * n);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t i = i0 + k * 256;
        if (i < total) then(r[k], i - r[k] * n, v[k]);
      }
    }
  };
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t n0 = it * R;
    const int rows = (int)min((int64_t)R, g.N - n0), w = rows * V;
    const bool any = g.n_hist > 0 || g.n_bias > 0;
    if (any) {
      __syncthreads();
      for (int i = tid; i < w; i += 256) seen[i] = 0, first[i] = NONE;
      if (tid < rows) said[tid] = said_of(g, n0 + tid);
      __syncthreads();
      if (g.history)
        each(
            rows, g.n_hist,
            [&](int r, int j) {
              return j < said[r] ? (uint32_t)g.history[(n0 + r) * g.ld_history + j] : NONE;
            },
            [&](int r, int, uint32_t v) {
              if (v < (uint32_t)V) atomicAdd(&seen[r * V + v], 1u);
            });
      if (g.n_bias > 0)
        each(
            rows, g.n_bias,
            [&](int r, int j) { return (uint32_t)g.bias_idx[(n0 + r) * g.ld_bias + j]; },
            [&](int r, int j, uint32_t v) {
              if (v < (uint32_t)V) atomicMin(&first[r * V + v], (uint32_t)j);
            });
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
    // (883 rows of 4 classes, 2764 earlier ones each: 191 us with as many rows as there is room for, on
    // 14 workgroups, 12 with one)
    const int note = g.n_hist > g.n_bias ? g.n_hist : g.n_bias;
    int R = SLICE / 4 / g.V < MOST_ROWS ? SLICE / 4 / g.V : MOST_ROWS;
    if ((int64_t)R * note > SLICE) R = SLICE / note > 1 ? SLICE / note : 1;
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
  const bool pack = g.n_hist < 0xffff && g.n_bias < 0xffff;
  if (wide && pack)
    k_adjust<T, true, true><<<blocks, 256, 0, s>>>(g, logits, out, slices, items);
  else if (wide)
    k_adjust<T, true, false><<<blocks, 256, 0, s>>>(g, logits, out, slices, items);
  else if (pack)
    k_adjust<T, false, true><<<blocks, 256, 0, s>>>(g, logits, out, slices, items);
  else
    k_adjust<T, false, false><<<blocks, 256, 0, s>>>(g, logits, out, slices, items);
  return hipGetLastError();
}
template hipError_t launch_adjust(const AdjustGeo&, const float*, float*, hipStream_t);
template hipError_t launch_adjust(const AdjustGeo&, const bf16*, bf16*, hipStream_t);

}  // namespace tfm
