// Reductions and prefix sums over a wavefront of 64 lanes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lda {

// Reductions over a wavefront by data-parallel moves (rows of 16 lanes, then
// across rows), which take a quarter of the time of exchanges through LDS; the
// result is in every lane.
template <int CONTROL, int ROWS>
__device__ __forceinline__ uint32_t moved(uint32_t other, uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)other, (int)x, CONTROL, ROWS, 0xF, false);
}

template <typename F>
__device__ __forceinline__ uint32_t wave_reduce(uint32_t x, uint32_t identity, F f) {
  x = f(x, moved<0x111, 0xF>(identity, x));  // from 1, 2, 4 and 8 lanes below in the row
  x = f(x, moved<0x112, 0xF>(identity, x));
  x = f(x, moved<0x114, 0xF>(identity, x));
  x = f(x, moved<0x118, 0xF>(identity, x));
  x = f(x, moved<0x142, 0xA>(identity, x));  // a row's last lane to the next row
  x = f(x, moved<0x143, 0xC>(identity, x));  // lane 31 to the upper half
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}

__device__ __forceinline__ float wave_max(float v) {
  const auto f = [](uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)));
  };
  return __builtin_bit_cast(float, wave_reduce(__builtin_bit_cast(uint32_t, v), 0xFF800000u, f));
}

__device__ __forceinline__ float wave_sum(float v) {
  const auto f = [](uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b));
  };
  return __builtin_bit_cast(float, wave_reduce(__builtin_bit_cast(uint32_t, v), 0u, f));
}

__device__ __forceinline__ uint32_t wave_min(uint32_t v) {
  return wave_reduce(v, 0xFFFFFFFFu, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
}

// The sum of the lanes up to and including this one.
__device__ __forceinline__ uint32_t wave_inclusive_sum(uint32_t x) {
  x += moved<0x111, 0xF>(0, x);
  x += moved<0x112, 0xF>(0, x);
  x += moved<0x114, 0xF>(0, x);
  x += moved<0x118, 0xF>(0, x);
  x += moved<0x142, 0xA>(0, x);
  x += moved<0x143, 0xC>(0, x);
  return x;
}

}  // namespace lda
