// Device pieces of the fixed-point sampler shared by the sampling kernel files.
#pragma once

#include "device_common.h"

namespace specdec {

namespace {

__device__ __forceinline__ uint64_t fp_weight(float r) {
  return r > 0.f ? (uint64_t)(r * 1099511627776.0f) : 0ull;  // exact: r * 2^40, truncation = floor
}
// floor(x * S / 2^32) without a 128-bit product (S < 2^56, x < 2^32).
__device__ __forceinline__ uint64_t scale_word(uint32_t x, uint64_t S) {
  return (uint64_t)x * (S >> 32) + (((uint64_t)x * (S & 0xffffffffull)) >> 32);
}

__device__ __forceinline__ uint64_t shfl_up_u64(uint64_t v, int o) {
  uint32_t lo = __shfl_up((uint32_t)v, o, kWave), hi = __shfl_up((uint32_t)(v >> 32), o, kWave);
  return ((uint64_t)hi << 32) | lo;
}

// Four consecutive entries of a row of V from j (a multiple of 4), `pad` past
// j1 (a multiple of 4, or V).
__device__ __forceinline__ void load_quad(const float* row, int j, int j1, int V, float pad, float (&v)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = pad;
  if ((V & 3) == 0 || j + 4 <= j1) {  // (first test uniform: whole quads need no second path)
    if (j < j1) {
      const f32x4 t = *(const f32x4_a4*)(row + j);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = t[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (j + e < j1) v[e] = row[j + e];
  }
}

}  // namespace

}  // namespace specdec
