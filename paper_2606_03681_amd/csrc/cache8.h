// Contexts kept in 8 bits (include/tfm_cache.h): appending rows and attention over the pool.
#pragma once

#include "common.h"

namespace tfm {

constexpr int CACHE8_E_MIN = 79, CACHE8_E_MAX = 175;  // bytes of a block's power of two
constexpr float CACHE8_TOP = 448.0f;                  // largest e4m3 value
constexpr uint8_t CACHE8_NAN = 0x7f;

// A power's byte as it counts.
__device__ __forceinline__ int power_byte(uint32_t e) {
  return min(max((int)e, CACHE8_E_MIN), CACHE8_E_MAX);
}
__device__ __forceinline__ float two_to(int e) {  // 2^e, e in [-126, 127]
  return __uint_as_float((uint32_t)(e + 127) << 23);
}

// A pool and the page table of a batch of sequences.
struct Cache8Geo {
  int32_t heads, d, page, shift;  // page = 1 << shift
  int32_t n_pages, max_pages;
  uint8_t *keys, *values, *powers;
  const int32_t* pages;  // nullable: sequence b's pages from b max_pages on
};

// The page of entry e of sequence b, -1 for one outside the pool.
__device__ __forceinline__ int cache8_page(const Cache8Geo& g, int64_t b, int e) {
  const int64_t at = b * g.max_pages + e;
  const int64_t p = g.pages ? g.pages[at] : at;
  return p >= 0 && p < g.n_pages ? (int)p : -1;
}

struct Cache8Append {
  Cache8Geo g;
  int32_t B, L;
  int64_t sk[3], sv[3];
  const int32_t *lens, *n_new;  // nullable
};
template <class T>
hipError_t launch_cache8_append(const Cache8Append& a, const T* k, const T* v, hipStream_t s);

// A pool of n_pages pages at `at`: keys, values, powers.
inline Cache8Geo cache8_geo(int heads, int d, int page, int n_pages, void* at, int max_pages,
                            const int32_t* pages) {
  Cache8Geo g;
  g.heads = heads; g.d = d; g.page = page;
  g.shift = 31 - __builtin_clz((unsigned)page);
  g.n_pages = n_pages; g.max_pages = max_pages;
  g.keys = g.values = g.powers = nullptr;
  if (at) {
    const size_t half = (size_t)n_pages * heads * page * d;
    g.keys = (uint8_t*)at;
    g.values = g.keys + half;
    g.powers = g.values + half;
  }
  g.pages = pages;
  return g;
}
inline size_t cache8_pool_bytes(int heads, int d, int page, int64_t n_pages) {
  return (size_t)n_pages * heads * (2 * (size_t)page * d + 2);
}

struct Cache8Attend {
  Cache8Geo g;
  int32_t B, L, heads, causal;
  int32_t max_rows;          // of a sequence: the table's room, or less by the caller's word
  int32_t plan_B;            // B by which the work is cut (not less than B)
  float scale_log2;          // the scores' factor, with log2(e)
  int64_t sq[3], so[3];
  const int32_t *lens, *n_rows;  // n_rows nullable
  float* lse;                // nullable
  void* ws;
};
size_t cache8_attend_bytes(const Cache8Attend& a, bool f32);
template <class T>
hipError_t launch_cache8_attend(const Cache8Attend& a, const T* q, T* out, hipStream_t s);

}  // namespace tfm
