// Appending tokens to a key/value cache cut into blocks: the 8-bit rows of the blocks that they complete,
// with a scale for each block and KV head, the rows of the block that they leave incomplete, and the
// per-channel bounds of the keys.
//
// A block is rounded once, when its last token is there, from the exact values: codes do not depend on how the
// tokens came (one by one, in chunks, all at once), and a later token with a larger magnitude never rounds
// older ones again.  Until then its rows stay in `k_tail` / `v_tail` in the type that they came in.
//
// The call is a stream, 2 * 128 * e bytes read and 2 * 128 written per token and KV head, so a row is read once:
// a wave keeps 16 rows in registers (32 floats a lane), a workgroup of 8 waves 128 rows, which is the largest block;
// the largest magnitude of a block goes from wave to wave through LDS, and the rows are rounded where they are.
#include "internal.hpp"
#include "kv_blocks.hpp"

namespace a2ats {
namespace {

constexpr int kAppendThreads = 512;
constexpr int kWaveRows = 16;                                     // rows that a wave holds
constexpr int kSlabRows = kAppendThreads / 64 * kWaveRows;        // rows of a workgroup: the largest block
constexpr uint32_t kTinyBits = (127u - 100u) << 23;               // 2^-100
constexpr uint32_t kInfBits = 0x7f800000u;

// rint(127 x / a), ties to even, decided as for real numbers.  x * (127 / a) is off by less than 127 * 2^-23 (two
// roundings); within 2^-15 of a half the two sides of  254 |x| <> (2 k + 1) a  are formed exactly in float64 (32 bits each).
__device__ __forceinline__ int code_i8(float x, float a, float inv) {
  const float r = fabsf(x) * inv;
  const float k = floorf(r);
  int c = (int)rintf(r);
  if (fabsf(r - k - 0.5f) < 0x1p-15f) {
    const double lhs = (double)fabsf(x) * 254.0, rhs = (double)(2.f * k + 1.f) * (double)a;
    c = (int)k + (lhs > rhs ? 1 : (lhs < rhs ? 0 : ((int)k & 1)));
  }
  return x < 0.f ? -c : c;
}

// min / max that keep a NaN once there is one.
__device__ __forceinline__ float low(float a, float b) { return (b < a || b != b) ? b : a; }
__device__ __forceinline__ float high(float a, float b) { return (b > a || b != b) ? b : a; }

__device__ __forceinline__ void put_elem(float* p, float v) { *p = v; }
__device__ __forceinline__ void put_elem(uint16_t* p, float v) { *p = (uint16_t)(__float_as_uint(v) >> 16); }   // (v was a bfloat16)
__device__ __forceinline__ float get_elem(const float* p) { return *p; }
__device__ __forceinline__ float get_elem(const uint16_t* p) { return bf16_to_f32(*p); }

// CODES: the 8-bit cache is written (else only the bounds are).  E4M3: its format.
template <typename T, bool CODES, bool E4M3>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(BlockCache m, const T* __restrict__ k_new,
                                                                const T* __restrict__ v_new, int n_new, int ctx_len,
                                                                const int32_t* __restrict__ seq_lens,
                                                                const int32_t* __restrict__ new_lens, int parts) {
  constexpr int NW = kAppendThreads / 64, D = kRowBytes;
  __shared__ uint32_t s_big[NW];
  __shared__ float s_lo[NW][D], s_hi[NW][D];
  // workgroups: [b][kv][part][key, value]
  const int of = CODES ? 2 : 1;
  const int what = blockIdx.x % of, rest = blockIdx.x / of, part = rest % parts, bh = rest / parts;
  const int b = bh / m.n_kv_heads, kv = bh % m.n_kv_heads;
  int n = seq_lens ? seq_lens[b] : ctx_len;
  n = min(max(n, 0), ctx_len);
  int cnt = new_lens ? new_lens[b] : n_new;
  cnt = min(max(cnt, 0), min(n_new, n));
  const int shift = m.shift, blk = 1 << shift, start = n - cnt;
  const int base = start >> shift << shift, r0 = base + part * kSlabRows;
  if (cnt == 0 || r0 >= n) return;   // (uniform)

  const T* fresh = (what ? v_new : k_new) + (size_t)bh * n_new * D;
  T* tail = (T*)(what ? m.v_tail : m.k_tail) + ((size_t)bh << shift) * D;
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int slot = lane >> 4, d0 = (lane & 15) * 8;
  const bool bounds = m.bounds != nullptr && what == 0;
  const int w0 = r0 + wv * kWaveRows, c = w0 >> shift;                 // the wave's rows lie in one block
  const bool live = (c << shift) < n;                                  // some of the block's tokens are there
  const bool whole = CODES && live && ((c + 1) << shift) <= n;

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
          lo[e] = low(lo[e], x[i][e]);
          hi[e] = high(hi[e], x[i][e]);
        }
      }
    }
#pragma unroll
    for (int off = 16; off < 64; off <<= 1)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        lo[e] = low(lo[e], __shfl_xor(lo[e], off));
        hi[e] = high(hi[e], __shfl_xor(hi[e], off));
      }
    if (slot == 0) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s_lo[wv][d0 + e] = lo[e];
        s_hi[wv][d0 + e] = hi[e];
      }
    }
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
    const size_t at = block_at(m, b, kv, c);
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
#pragma unroll
          for (int e = 0; e < 8; ++e) w[e >> 2] |= (uint32_t)(code_i8(x[i][e], a, inv) & 255) << (8 * (e & 3));
        }
      }
      *(uint2*)(rows + (size_t)(i * 4 + slot) * kRowBytes) = make_uint2(w[0], w[1]);
    }
  }
  if (bounds) {
    T* all = (T*)m.bounds;
    for (int i = tid; i < kSlabRows / blk * D; i += kAppendThreads) {
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
    for (int i = tid; i < (n - from) * PER_ROW; i += kAppendThreads) dst[i] = src[i];
  }
}

}  // namespace

hipError_t launch_append(const a2ats_dims& d, const BlockCache& m, int kv_dtype, int format, bool codes, const void* k_new,
                         const void* v_new, int n_new, const int32_t* seq_lens, const int32_t* new_lens, hipStream_t stream) {
  const long bh = (long)d.batch * d.n_kv_heads;
  if (bh == 0 || n_new == 0 || d.ctx_len == 0) return hipSuccess;
  const int parts = append_parts(n_new, 1 << m.shift);
  const dim3 grid((unsigned)(bh * parts * (codes ? 2 : 1)));
#define A2ATS_APPEND(T, CODES, E4M3)                                                                                  \
  hipLaunchKernelGGL((append_kernel<T, CODES, E4M3>), grid, dim3(kAppendThreads), 0, stream, m, (const T*)k_new,       \
                     (const T*)v_new, n_new, d.ctx_len, seq_lens, new_lens, parts)
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

// Slabs of 128 rows from the beginning of the first block that gets tokens to the last one.
int append_parts(int n_new, int block) { return (int)(((long)n_new + block - 1 + kSlabRows - 1) / kSlabRows); }

}  // namespace a2ats
