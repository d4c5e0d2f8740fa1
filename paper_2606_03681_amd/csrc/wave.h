// Sums and maxima over the 64 lanes of a wave by data-parallel primitives: no lane addresses to
// keep, and the result is a scalar.  Every lane of the wave must be active.
#pragma once

#include <hip/hip_runtime.h>

namespace tfm {

// Lane moves of a scan: 1, 2, 4, 8 lanes up within rows of 16, then the last lane of row 0 to row 1
// and of row 2 to row 3, then of row 1 to rows 2 and 3; lane 63 ends with the whole.  Lanes
// without a source get `none`.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t lane_move(uint32_t none, uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ float lane_move(float none, float v) {
  return __uint_as_float(lane_move<CTRL, ROWS>(__float_as_uint(none), __float_as_uint(v)));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t lane_move(uint64_t none, uint64_t v) {
  const uint32_t lo = lane_move<CTRL, ROWS>((uint32_t)none, (uint32_t)v);
  const uint32_t hi = lane_move<CTRL, ROWS>((uint32_t)(none >> 32), (uint32_t)(v >> 32));
  return (uint64_t)hi << 32 | lo;
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double lane_move(double none, double v) {
  return __longlong_as_double((long long)lane_move<CTRL, ROWS>(
      (uint64_t)__double_as_longlong(none), (uint64_t)__double_as_longlong(v)));
}

__device__ __forceinline__ uint32_t from_lane(uint32_t v, int lane) {
  return (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}
__device__ __forceinline__ float from_lane(float v, int lane) {
  return __uint_as_float(from_lane(__float_as_uint(v), lane));
}
__device__ __forceinline__ uint64_t from_lane(uint64_t v, int lane) {
  return (uint64_t)from_lane((uint32_t)(v >> 32), lane) << 32 | from_lane((uint32_t)v, lane);
}
__device__ __forceinline__ double from_lane(double v, int lane) {
  return __longlong_as_double((long long)from_lane((uint64_t)__double_as_longlong(v), lane));
}

// Inclusive scan: lane l gets op over lanes 0 .. l.
template <class V, class F>
__device__ __forceinline__ V wave_scan(V v, V none, F op) {
  v = op(v, lane_move<0x111, 0xf>(none, v));
  v = op(v, lane_move<0x112, 0xf>(none, v));
  v = op(v, lane_move<0x114, 0xf>(none, v));
  v = op(v, lane_move<0x118, 0xf>(none, v));
  v = op(v, lane_move<0x142, 0xa>(none, v));
  v = op(v, lane_move<0x143, 0xc>(none, v));
  return v;
}
template <class V>
__device__ __forceinline__ V wave_sum(V v) {
  return from_lane(wave_scan(v, V(0), [](V a, V b) { return a + b; }), 63);
}
__device__ __forceinline__ float wave_max(float v) {
  return from_lane(wave_scan(v, -INFINITY, [](float a, float b) { return fmaxf(a, b); }), 63);
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  return from_lane(wave_scan(v, 0u, [](uint32_t a, uint32_t b) { return a > b ? a : b; }), 63);
}
__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
  return from_lane(
      wave_scan(v, (uint64_t)0, [](uint64_t a, uint64_t b) { return a > b ? a : b; }), 63);
}

}  // namespace tfm
