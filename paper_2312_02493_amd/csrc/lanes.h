// Reductions over the lanes of a wave by data-parallel moves, which take a few cycles where a shuffle through LDS takes a hundred.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace artopk {

// Values of other lanes by data-parallel moves: a lane that has no source keeps `other`.  A row is sixteen lanes.
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ uint32_t moved(uint32_t v, uint32_t other) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)other, (int)v, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ float moved(float v, float other) {
  return __uint_as_float(moved<CTRL, ROWS>(__float_as_uint(v), __float_as_uint(other)));
}
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ uint64_t moved(uint64_t v, uint64_t other) {
  return (uint64_t)moved<CTRL, ROWS>((uint32_t)(v >> 32), (uint32_t)(other >> 32)) << 32 | moved<CTRL, ROWS>((uint32_t)v, (uint32_t)other);
}
__device__ __forceinline__ uint32_t lane_value(uint32_t v, int lane) { return __builtin_amdgcn_readlane(v, lane); }
__device__ __forceinline__ float lane_value(float v, int lane) { return __uint_as_float(lane_value(__float_as_uint(v), lane)); }
__device__ __forceinline__ uint64_t lane_value(uint64_t v, int lane) {
  return (uint64_t)lane_value((uint32_t)(v >> 32), lane) << 32 | lane_value((uint32_t)v, lane);
}

// f over all lanes of a wave, `zero` its neutral value: towards the end of each row, then of the rows, then from the last lane.
template <class T, class F>
__device__ __forceinline__ T over_wave(T v, T zero, F&& f) {
  v = f(v, moved<0x111>(v, zero));  // one lane, two, four and eight lanes back
  v = f(v, moved<0x112>(v, zero));
  v = f(v, moved<0x114>(v, zero));
  v = f(v, moved<0x118>(v, zero));
  v = f(v, moved<0x142, 0xa>(v, zero));  // rows 0 and 2 into 1 and 3
  v = f(v, moved<0x143, 0xc>(v, zero));  // row 1 into 2 and 3
  return lane_value(v, 63);
}

// f over sixteen lanes side by side, in each of them; f's order of arguments must not matter.
template <class T, class F>
__device__ __forceinline__ T over_sixteen(T v, F&& f) {
  v = f(v, moved<0xb1>(v, v));   // the neighbour
  v = f(v, moved<0x4e>(v, v));   // the other pair
  v = f(v, moved<0x141>(v, v));  // the eight backwards, then the sixteen
  return f(v, moved<0x140>(v, v));
}

__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  return over_wave(v, 0u, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
  return over_wave(v, (uint64_t)0, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
}

}  // namespace artopk
