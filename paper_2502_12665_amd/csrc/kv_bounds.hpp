// Bounds of blocks of keys per dimension, as the appends to cut caches keep them.
#pragma once
#include "common.hpp"
#include "kv_blocks.hpp"

namespace a2ats {

constexpr int kWaveRows = 16;   // rows that a wave of an append holds

// Four or eight waves: a slab of 64 rows, or the largest block.
constexpr int append_waves(int block) { return block > 64 ? 8 : 4; }

// min / max that keep a NaN once there is one.
__device__ __forceinline__ float low(float a, float b) { return (b < a || b != b) ? b : a; }
__device__ __forceinline__ float high(float a, float b) { return (b > a || b != b) ? b : a; }

__device__ __forceinline__ void put_elem(float* p, float v) { *p = v; }
__device__ __forceinline__ void put_elem(uint16_t* p, float v) { *p = (uint16_t)(__float_as_uint(v) >> 16); }   // (v was a bfloat16)
__device__ __forceinline__ float get_elem(const float* p) { return *p; }
__device__ __forceinline__ float get_elem(const uint16_t* p) { return bf16_to_f32(*p); }

// Plain min / max (fminf would first quiet both operands).
__device__ __forceinline__ float min2(float a, float b) { return __builtin_amdgcn_fmed3f(a, b, -INFINITY); }
__device__ __forceinline__ float max2(float a, float b) { return __builtin_amdgcn_fmed3f(a, b, INFINITY); }

// f over the four lane rows of eight values v[e]: lane row r is left with two of them, 4 (r / 2) + 2 (r % 2) + {0, 1}.
template <typename F>
__device__ __forceinline__ float2 over_lane_rows(const float (&v)[8], F f) {
  float h[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[e]), __float_as_uint(v[e + 4]), false, false);
    h[e] = f(__uint_as_float(s[0]), __uint_as_float(s[1]));
  }
  float q[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(h[e]), __float_as_uint(h[e + 2]), false, false);
    q[e] = f(__uint_as_float(s[0]), __uint_as_float(s[1]));
  }
  return make_float2(q[0], q[1]);
}

}  // namespace a2ats
