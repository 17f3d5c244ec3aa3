// Appending tokens to a key/value cache cut into blocks: the 8-bit rows of the blocks that they complete,
// with a scale for each block and KV head, the rows of the block that they leave incomplete, and the
// per-channel bounds of the keys.
//
// A block is rounded once, when its last token is there, from the exact values: codes do not depend on how the
// tokens came (one by one, in chunks, all at once), and a later token with a larger magnitude never rounds
// older ones again.  Until then its rows stay in `k_tail` / `v_tail` in the type that they came in.
//
// The call is a stream, 2 * 128 * e bytes read and 2 * 128 written per token and KV head, so a row is read once:
// a wave keeps 16 rows in registers (32 floats a lane), a workgroup of 4 waves 64 rows (of 8 for blocks of 128);
// the largest magnitude of a block goes from wave to wave through LDS, and the rows are rounded where they are.  What is
// not 127 x / a at once (a code within the product's error of a half) is decided exactly, in float64 or, for bfloat16, whose
// products cannot come that close without being a half, by cutting the product to 20 bits.
//
// Measured: 8 KV heads x 32768 tokens, bfloat16 to int8 with bounds, 49 us = 4.2 TB/s of 206 MB, of which the bounds' minima and
// maxima (vector ALU) are 8; e4m3 without bounds runs at the rate of a large copy (4.9 TB/s).  4 x 4 x 4099 tokens, float32 to
// e4m3 in pages, 13.6 - 15 us = 3.4 - 3.8 TB/s.  Bounds alone, 8 KV heads x 32768 tokens: bfloat16 20.7 us = 3.4 TB/s (the minima and
// maxima), float32 29.7 us = 4.8 TB/s.  One token of 16 x 8 heads: 4.7 us (bounds alone 3.5), of which an empty launch is 1.6; the rest are
// the requests that wait for each other (length, rows, bounds).  Requesting the bounds and the tail's rows ahead of the barrier did
// not shorten it (4.9).
#include "internal.hpp"
#include "kv_bounds.hpp"

namespace a2ats {
namespace {

constexpr uint32_t kTinyBits = (127u - 100u) << 23;               // 2^-100
constexpr uint32_t kInfBits = 0x7f800000u;

// rint(127 x / a), ties to even, decided as for real numbers: within a half of k the two sides of  254 |x| <> (2 k + 1) a  are
// formed exactly in float64 (32 bits each).
__device__ __forceinline__ int code_i8_close(float x, float a) {
  const float r = fabsf(x) * (127.f / a);
  const float k = floorf(r);
  int c = (int)rintf(r);
  if (fabsf(r - k - 0.5f) < 0x1p-14f) {
    const double lhs = (double)fabsf(x) * 254.0, rhs = (double)(2.f * k + 1.f) * (double)a;
    c = (int)k + (lhs > rhs ? 1 : (lhs < rhs ? 0 : ((int)k & 1)));
  }
  return x < 0.f ? -c : c;
}

// CODES: the 8-bit cache is written (else only the bounds are).  E4M3: its format.  NW: waves of a workgroup.
template <typename T, bool CODES, bool E4M3, int NW>
__global__ __launch_bounds__(NW * 64) void append_kernel(BlockCache m, const T* __restrict__ k_new, const T* __restrict__ v_new,
                                                         int n_new, int ctx_len, const int32_t* __restrict__ seq_lens,
                                                         const int32_t* __restrict__ new_lens, int parts) {
  constexpr int D = kRowBytes, NT = NW * 64, SLAB = NW * kWaveRows;
  __shared__ uint32_t s_big[NW];
  __shared__ __align__(8) float s_lo[NW][D], s_hi[NW][D];
  // workgroups: [b][kv][part][key, value]
  const int of = CODES ? 2 : 1;
  const int what = blockIdx.x % of, rest = blockIdx.x / of, part = rest % parts, bh = rest / parts;
  const int b = bh / m.n_kv_heads, kv = bh % m.n_kv_heads;
  int n = seq_lens ? seq_lens[b] : ctx_len;
  n = min(max(n, 0), ctx_len);
  int cnt = new_lens ? new_lens[b] : n_new;
  cnt = min(max(cnt, 0), min(n_new, n));
  const int shift = m.shift, blk = 1 << shift, start = n - cnt;
  const int base = start >> shift << shift, r0 = base + part * SLAB;
  if (cnt == 0 || r0 >= n) return;   // (uniform)

  const T* fresh = (what ? v_new : k_new) + (size_t)bh * n_new * D;
  T* tail = (T*)(what ? m.v_tail : m.k_tail) + ((size_t)bh << shift) * D;
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int slot = lane >> 4, d0 = (lane & 15) * 8;
  const bool bounds = m.bounds != nullptr && what == 0;
  const int w0 = r0 + wv * kWaveRows, c = w0 >> shift;                 // the wave's rows lie in one block
  const bool live = (c << shift) < n;                                  // some of the block's tokens are there
  const bool whole = CODES && live && ((c + 1) << shift) <= n;
  const size_t at = live ? block_at(m, b, kv, c) : 0;

  float x[4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = w0 + i * 4 + slot;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[i][e] = 0.f;
    if (row >= start ? row < n && (whole || bounds) : whole)
      load8(row >= start ? fresh + (size_t)(row - start) * D + d0 : tail + (size_t)(row - base) * D + d0, x[i]);
  }
  // The block's largest magnitude, as bits: their order is that of the values, with what is not finite at the top.
  uint32_t big = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) big = max(big, __float_as_uint(x[i][e]) & 0x7fffffffu);
  const bool any_nan = __builtin_amdgcn_ballot_w64(big > kInfBits) != 0u;
  big = wave_max_to_last_lane(big);
  if (lane == 63) s_big[wv] = big;
  if (bounds) {
    float lo[8], hi[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) { lo[e] = INFINITY; hi[e] = -INFINITY; }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = w0 + i * 4 + slot;
      if (row >= start && row < n) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          lo[e] = any_nan ? low(lo[e], x[i][e]) : min2(lo[e], x[i][e]);
          hi[e] = any_nan ? high(hi[e], x[i][e]) : max2(hi[e], x[i][e]);
        }
      }
    }
    const int d = d0 + 4 * (slot >> 1) + 2 * (slot & 1);
    *(float2*)&s_lo[wv][d] = any_nan ? over_lane_rows(lo, low) : over_lane_rows(lo, min2);
    *(float2*)&s_hi[wv][d] = any_nan ? over_lane_rows(hi, high) : over_lane_rows(hi, max2);
  }
  __syncthreads();   // (also: every row that this workgroup takes from the tail has been read)

  const int per = blk / kWaveRows;   // waves of a block
  if (whole) {
    const int w_first = wv & ~(per - 1);
    uint32_t most = 0;
    for (int i = 0; i < per; ++i) most = max(most, s_big[w_first + i]);
    const float a = __uint_as_float(most);
    float scale, inv;
    const bool usable = most >= kTinyBits && most < kInfBits;
    if (!usable) {
      scale = most < kTinyBits ? 0.f : __uint_as_float(0x7fc00000u);
      inv = 0.f;
    } else if (E4M3) {
      // the least power of two with a <= 448 * scale, 448 = 1.75 * 2^8
      const int e = (int)(most >> 23) - 8 + ((most & 0x7fffffu) > 0x600000u ? 1 : 0);   // biased
      scale = __uint_as_float((uint32_t)e << 23);
      inv = __uint_as_float((uint32_t)(254 - e) << 23);
    } else {
      scale = a / 127.f;
      inv = 127.f / a;
    }
    if (wv == w_first && lane == 0) (what ? m.v_scale : m.k_scale)[at] = scale;
    uint8_t* rows = (what ? m.v : m.k) + ((at << shift) + (size_t)(w0 & (blk - 1))) * kRowBytes + d0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t w[2] = {0u, 0u};
      if (usable) {
        if (E4M3) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            int word = 0;
            word = __builtin_amdgcn_cvt_pk_fp8_f32(x[i][4 * h] * inv, x[i][4 * h + 1] * inv, word, false);
            word = __builtin_amdgcn_cvt_pk_fp8_f32(x[i][4 * h + 2] * inv, x[i][4 * h + 3] * inv, word, true);
            w[h] = (uint32_t)word;
          }
        } else {
          // A product + 3 * 2^22 has the rounded product as its low byte.
          float t[8];
          bool close = false;
          if (sizeof(T) == 2) {
            // x inv is off by less than 2^-22 of itself.  With significands of 8 bits, 127 x / a is a half k + 1/2 or at least
            // (k + 1/2) 2^-16 away from it (254 x - (2 k + 1) a is a multiple of the unit of x): in 20 bits it is on the right
            // side, or exact.
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const uint32_t r = __float_as_uint(x[i][e] * inv);
              t[e] = __uint_as_float((r + 4u) & ~7u) + 12582912.f;
            }
          } else {
            // The product is off by 127 * 2^-24 at most (the factor's rounding): a remainder within 2^-15 of a half is looked at.
            float left = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              t[e] = __builtin_fmaf(x[i][e], inv, 12582912.f);
              left = fmaxf(left, fabsf(__builtin_fmaf(x[i][e], inv, 12582912.f - t[e])));
            }
            close = left > 0.5f - 0x1p-15f;
          }
          if (close) {
#pragma unroll 1
            for (int e = 0; e < 8; ++e) {
              float xe = 0.f;
#pragma unroll
              for (int f = 0; f < 8; ++f) xe = e == f ? x[i][f] : xe;
              const uint32_t code = (uint32_t)(code_i8_close(xe, a) & 255) << (8 * (e & 3));
              w[0] |= e < 4 ? code : 0u;
              w[1] |= e < 4 ? 0u : code;
            }
          } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t p01 = __builtin_amdgcn_perm(__float_as_uint(t[4 * h + 1]), __float_as_uint(t[4 * h]), 0x0c0c0400u);
              w[h] = __builtin_amdgcn_perm(__float_as_uint(t[4 * h + 2]), p01, 0x0c040100u);
              w[h] = __builtin_amdgcn_perm(__float_as_uint(t[4 * h + 3]), w[h], 0x04020100u);
            }
          }
        }
      }
      *(uint2*)(rows + (size_t)(i * 4 + slot) * kRowBytes) = make_uint2(w[0], w[1]);
    }
  }
  if (bounds) {
    T* all = (T*)m.bounds;
    for (int i = tid; i < SLAB / blk * D; i += NT) {
      const int cb = i / D, d = i % D, ci = (r0 >> shift) + cb, t0 = ci << shift;
      if (t0 >= n) break;
      float lo = INFINITY, hi = -INFINITY;
      for (int w = cb * per; w < (cb + 1) * per; ++w) {
        lo = low(lo, s_lo[w][d]);
        hi = high(hi, s_hi[w][d]);
      }
      T* p = all + block_at(m, b, kv, ci) * 2 * D + d;
      if (t0 < start) {   // the block had tokens before
        lo = low(lo, get_elem(p));
        hi = high(hi, get_elem(p + D));
      }
      put_elem(p, lo);
      put_elem(p + D, hi);
    }
  }
  // The rows of the incomplete block, by the workgroup that has read what was there.
  if (CODES && part == 0) {
    const int from = max(start, n >> shift << shift);
    constexpr int V = 16 / sizeof(T), PER_ROW = D / V;
    const uint4* src = (const uint4*)(fresh + (size_t)(from - start) * D);
    uint4* dst = (uint4*)(tail + (size_t)(from & (blk - 1)) * D);
    for (int i = tid; i < (n - from) * PER_ROW; i += NT) dst[i] = src[i];
  }
}

}  // namespace

hipError_t launch_append(const a2ats_dims& d, const BlockCache& m, int kv_dtype, int format, bool codes, const void* k_new,
                         const void* v_new, int n_new, const int32_t* seq_lens, const int32_t* new_lens, hipStream_t stream) {
  const long bh = (long)d.batch * d.n_kv_heads;
  if (bh == 0 || n_new == 0 || d.ctx_len == 0) return hipSuccess;
  const int parts = append_parts(n_new, 1 << m.shift);
  const dim3 grid((unsigned)(bh * parts * (codes ? 2 : 1)));
#define A2ATS_APPEND(T, CODES, E4M3)                                                                                      \
  do {                                                                                                                  \
    if (append_waves(1 << m.shift) == 4)                                                                                \
      hipLaunchKernelGGL((append_kernel<T, CODES, E4M3, 4>), grid, dim3(256), 0, stream, m, (const T*)k_new,             \
                         (const T*)v_new, n_new, d.ctx_len, seq_lens, new_lens, parts);                                 \
    else                                                                                                                \
      hipLaunchKernelGGL((append_kernel<T, CODES, E4M3, 8>), grid, dim3(512), 0, stream, m, (const T*)k_new,             \
                         (const T*)v_new, n_new, d.ctx_len, seq_lens, new_lens, parts);                                 \
  } while (0)
  const bool e4m3 = format == A2ATS_E4M3;
  if (kv_dtype == A2ATS_BF16) {
    if (!codes) A2ATS_APPEND(uint16_t, false, false);
    else if (e4m3) A2ATS_APPEND(uint16_t, true, true);
    else A2ATS_APPEND(uint16_t, true, false);
  } else {
    if (!codes) A2ATS_APPEND(float, false, false);
    else if (e4m3) A2ATS_APPEND(float, true, true);
    else A2ATS_APPEND(float, true, false);
  }
#undef A2ATS_APPEND
  return hipGetLastError();
}

// Slabs from the beginning of the first block that gets tokens to the last one.
int append_parts(int n_new, int block) {
  const int slab = append_waves(block) * kWaveRows;
  return (int)(((long)n_new + block - 1 + slab - 1) / slab);
}
int append_threads(int block) { return append_waves(block) * 64; }

}  // namespace a2ats
