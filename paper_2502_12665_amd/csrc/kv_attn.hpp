// What the attention kernels over cut caches (8 and 4 bits) have in common: exchanges between the lanes of a wave, and operands
// of the matrix cores made of several terms.  Lane l of a wave is column l % 16 of lane row l / 16.
#pragma once
#include <cfloat>

#include "common.hpp"
#include "kv_blocks.hpp"

namespace a2ats {

constexpr int kPair = 32;               // rows that a wave takes at a time: two tiles of 16
constexpr float kNone = -FLT_MAX;       // the maximum of no rows
constexpr float kLogit = 0.12751743f;   // log2(e) / sqrt(128)

typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;

// Between what some lanes of a wave write to LDS and others of it read, and the other way round: no instruction (a wave's LDS
// operations are done in order), but what keeps the compiler from moving either past it.
__device__ __forceinline__ void wave_exchange() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ float power(float x) { return __builtin_amdgcn_exp2f(x); }

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
// Sum over the columns of a head, c, c + GP, .. of 16: the same bits in each of them (the terms of a weight, a column each, are
// only its terms if they are those of one number), as the first sums repeat after eight columns.
template <int GP>
__device__ __forceinline__ float head_sum(float v) {
  v += dpp<0x128>(v);                // row_ror:8
  if (GP == 4) v += dpp<0x124>(v);   // row_ror:4
  return v;
}
// Over the four lane rows, in every lane.
template <typename F>
__device__ __forceinline__ float over_rows(float v, F f) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float rows_max(float v) {
  return over_rows(v, [](float x, float y) { return fmaxf(x, y); });
}
__device__ __forceinline__ float rows_sum(float v) {
  return over_rows(v, [](float x, float y) { return x + y; });
}
// The upper halves of two floats, the first one below: bfloat16 by truncation.
__device__ __forceinline__ uint32_t upper_halves(float a, float b) {
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}
__device__ __forceinline__ uint32_t f16_bits(f16x2 v) { return __builtin_bit_cast(uint32_t, v); }
__device__ __forceinline__ f16x2 f16_pair(float a, float b) {
  typedef __attribute__((ext_vector_type(2))) float f32x2;
  return __builtin_convertvector((f32x2){a, b}, f16x2);   // (to the nearest)
}

template <int N>
__device__ __forceinline__ void load_elems(const float* p, float* x) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const float4 v = *(const float4*)(p + i);
    x[i] = v.x; x[i + 1] = v.y; x[i + 2] = v.z; x[i + 3] = v.w;
  }
}
template <int N>
__device__ __forceinline__ void load_elems(const uint16_t* p, float* x) {
#pragma unroll
  for (int i = 0; i < N; i += 8) {
    float y[8];
    load8(p + i, y);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[i + e] = y[e];
  }
}
__device__ __forceinline__ void store_elem(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_elem(uint16_t* p, float v) { *p = f32_to_bf16(v); }

// Logits times log2 e, from the queries on: the rounding is each element's own, and the factors behind are powers of two.
__device__ __forceinline__ void to_logits(float (&x)[32]) {
#pragma unroll
  for (int i = 0; i < 32; ++i) x[i] *= kLogit;
}

// The least e >= -97 with |x| < 2^e for all x of a head's row (32 elements in this lane, the others in the lane rows);
// ok: all are finite.  (-97: 2^(30 - e), by which an element becomes a whole number, is a float32 then, also for a row of zeros;
// what is below 2^-30 of 2^-97 is below the least normal number.)
__device__ __forceinline__ int row_exponent(const float (&x)[32], bool& ok) {
  uint32_t big = 0;
#pragma unroll
  for (int i = 0; i < 32; ++i) big = max(big, __float_as_uint(x[i]) & 0x7fffffffu);
  const auto a = __builtin_amdgcn_permlane32_swap(big, big, false, false);
  big = max(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(big, big, false, false);
  big = max(b[0], b[1]);
  ok = big < 0x7f800000u;
  return max((int)(big >> 23) - 126, -97);
}

// A query as float16 terms, for the columns of the first three (eight heads: two): x = 2^(e - 8) (t0 + t1 + t2) but for 2^-33 of 2^e
// (half the least float16) and, for eight heads, 2^-23 of x.  Returns 2^(e - 8).
template <int GP>
__device__ __forceinline__ float query_terms(const float (&x)[32], int term, bool active, f16x8 (&q)[4]) {
  bool ok;
  const int e = row_exponent(x, ok);
  const float down = ldexpf(active && term < 3 ? 1.f : 0.f, 8 - e);
  const float less1 = term >= 1 ? 1.f : 0.f, less2 = term >= 2 ? 1.f : 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float y = x[8 * i + j] * down;
      y -= less1 * (float)(_Float16)y;
      if (GP == 4) y -= less2 * (float)(_Float16)y;
      q[i][j] = (_Float16)y;
    }
  return ok ? ldexpf(1.f, e - 8) : __uint_as_float(0x7fc00000u);
}

}  // namespace a2ats
