// Appending tokens to a key/value cache held in 4 bits, and reading them back.
//
// A group of 32 dimensions of a token's key (or value) is rounded by itself: with a = max |x| its scale is the least power of
// two 2^e with a <= 6 * 2^e, and a code is x / 2^e to the nearest e2m1 number (0, 1/2, 1, 3/2, 2, 3, 4, 6), ties to even.  So a
// row depends on nothing but itself: there is no tail, and a token can be written again.  x / 2^e is exact, and
// v_cvt_scalef32_pk_fp4_f32 rounds it as for real numbers.
//
// Both are streams, 2 * 128 * e bytes against 136.
#include "internal.hpp"
#include "kv_bounds.hpp"

namespace a2ats {
namespace {

constexpr int D = 128;
constexpr uint32_t kTinyBits = (127u - 100u) << 23;    // 2^-100
constexpr uint32_t kHugeBits = (127u + 127u) << 23;    // 2^127

template <int CTRL>
__device__ __forceinline__ uint32_t lane_of(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false);
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E;              // quad_perm [1,0,3,2], [2,3,0,1]
constexpr int kNext4 = 0x12C, kNext8 = 0x128, kNext12 = 0x124;   // row_ror: of 16 lanes, the one 4, 8, 12 further on

// Eight elements of a row, of which 16 consecutive lanes have all, as codes, the first in the lowest bits; the scale byte of the
// group, which four lanes share.
__device__ __forceinline__ uint32_t codes8(const float (&x)[8], uint32_t& byte) {
  uint32_t big = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) big = max(big, __float_as_uint(x[e]) & 0x7fffffffu);
  big = max(big, lane_of<kXor1>(big));
  big = max(big, lane_of<kXor2>(big));
  const bool usable = big >= kTinyBits && big < kHugeBits;
  // 6 = 1.5 * 2^2
  byte = usable ? (big >> 23) - 2u + ((big & 0x7fffffu) > 0x400000u ? 1u : 0u) : (big < kTinyBits ? 0u : 255u);
  const float scale = kv4_scale(usable ? byte : 127u);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
  return usable ? w : 0u;
}

// A value's bytes in the order of the cache.  Lane j = 4 g + h of 16 has the dimensions 32 g + 8 h + 0 .. 7, bytes n = 4 h + 0 .. 3 of
// group g; it is left with the word of n = 4 h + g, byte i of group i.
struct ValueOrder {
  uint32_t first, second;   // (0x0c: a zero byte)
  __device__ __forceinline__ ValueOrder(int g) {
    auto put = [](uint32_t word, int at, int byte) { return word ^ (0x0cu ^ (uint32_t)byte) << (8 * (at & 3)); };
    first = put(put(0x0c0c0c0cu, g, g), g + 1, 4 + g);
    second = put(put(0x0c0c0c0cu, g + 2, g), g + 3, 4 + g);
  }
  __device__ __forceinline__ uint32_t apply(uint32_t w) const {
    const uint32_t w1 = lane_of<kNext4>(w), w2 = lane_of<kNext8>(w), w3 = lane_of<kNext12>(w);
    return __builtin_amdgcn_perm(w1, w, first) | __builtin_amdgcn_perm(w3, w2, second);
  }
};

// NW: waves of a workgroup, 16 rows each.
template <typename T, int NW>
__global__ __launch_bounds__(NW * 64) void kv4_append_kernel(Kv4Cache m, const T* __restrict__ k_new, const T* __restrict__ v_new,
                                                             int n_new, int ctx_len, const int32_t* __restrict__ seq_lens,
                                                             const int32_t* __restrict__ new_lens, int parts) {
  constexpr int NT = NW * 64, SLAB = NW * kWaveRows;
  __shared__ __align__(8) float s_lo[NW][D], s_hi[NW][D];
  // workgroups: [b][kv][part][key, value]
  const int what = blockIdx.x & 1, rest = blockIdx.x >> 1, part = rest % parts, bh = rest / parts;
  const int b = bh / m.at.n_kv_heads, kv = bh % m.at.n_kv_heads;
  int n = seq_lens ? seq_lens[b] : ctx_len;
  n = min(max(n, 0), ctx_len);
  int cnt = new_lens ? new_lens[b] : n_new;
  cnt = min(max(cnt, 0), min(n_new, n));
  const int shift = m.at.shift, blk = 1 << shift, start = n - cnt;
  const int base = start >> shift << shift, r0 = base + part * SLAB;
  if (cnt == 0 || r0 >= n) return;   // (uniform)

  const T* fresh = (what ? v_new : k_new) + (size_t)bh * n_new * D;
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int slot = lane >> 4, j = lane & 15, d0 = j * 8;
  const bool bounds = m.at.bounds != nullptr && what == 0;
  const int w0 = r0 + wv * kWaveRows;                                  // the wave's rows lie in one block
  const bool live = w0 < n && w0 + kWaveRows > start;                  // some of them are new

  float x[4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = w0 + i * 4 + slot;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[i][e] = 0.f;
    if (row >= start && row < n) load8(fresh + (size_t)(row - start) * D + d0, x[i]);
  }
  if (live) {
    const size_t at = (block_at(m.at, b, kv, w0 >> shift) << shift) + (size_t)(w0 & (blk - 1));
    const ValueOrder order(j >> 2);
    const int word = what ? 16 + 4 * (j & 3) + (j >> 2) : j;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = w0 + i * 4 + slot;
      uint32_t byte;
      uint32_t w = codes8(x[i], byte);
      if (what) w = order.apply(w);
      byte <<= 8 * (j >> 2);
      byte |= lane_of<kNext4>(byte);
      byte |= lane_of<kNext8>(byte);
      if (row >= start && row < n) {
        const size_t r = at + (size_t)(i * 4 + slot);
        *(uint32_t*)(m.rows + r * kKv4RowBytes + word * 4) = w;
        if (j == 0) *(uint32_t*)(m.scales + r * kKv4ScaleBytes + what * 4) = byte;
      }
    }
  }
  if (!bounds) return;   // (uniform)
  uint32_t big = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) big = max(big, __float_as_uint(x[i][e]) & 0x7fffffffu);
  const bool any_nan = __builtin_amdgcn_ballot_w64(big > 0x7f800000u) != 0u;
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
  const int d2 = d0 + 4 * (slot >> 1) + 2 * (slot & 1);
  *(float2*)&s_lo[wv][d2] = any_nan ? over_lane_rows(lo, low) : over_lane_rows(lo, min2);
  *(float2*)&s_hi[wv][d2] = any_nan ? over_lane_rows(hi, high) : over_lane_rows(hi, max2);
  __syncthreads();
  const int per = blk / kWaveRows;   // waves of a block
  T* all = (T*)m.at.bounds;
  for (int i = tid; i < SLAB / blk * D; i += NT) {
    const int cb = i / D, d = i % D, ci = (r0 >> shift) + cb, t0 = ci << shift;
    if (t0 >= n) break;
    float lo1 = INFINITY, hi1 = -INFINITY;
    for (int w = cb * per; w < (cb + 1) * per; ++w) {
      lo1 = low(lo1, s_lo[w][d]);
      hi1 = high(hi1, s_hi[w][d]);
    }
    T* p = all + block_at(m.at, b, kv, ci) * 2 * D + d;
    if (t0 < start) {   // the block had tokens before
      lo1 = low(lo1, get_elem(p));
      hi1 = high(hi1, get_elem(p + D));
    }
    put_elem(p, lo1);
    put_elem(p + D, hi1);
  }
}

// The eight numbers of a word of codes times a scale.
__device__ __forceinline__ void store_numbers(float* p, uint32_t w, float scale, bool bad) {
  float x[8];
#define A2ATS_PAIR(i)                                                             \
  {                                                                               \
    const auto f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, i);         \
    x[2 * i] = f[0];                                                              \
    x[2 * i + 1] = f[1];                                                          \
  }
  A2ATS_PAIR(0) A2ATS_PAIR(1) A2ATS_PAIR(2) A2ATS_PAIR(3)
#undef A2ATS_PAIR
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = bad ? __uint_as_float(0x7fc00000u) : x[i];
  *(float4*)p = make_float4(x[0], x[1], x[2], x[3]);
  *(float4*)(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store_numbers(uint16_t* p, uint32_t w, float scale, bool bad) {
  uint32_t x[4];
#define A2ATS_PAIR(i) x[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, i));
  A2ATS_PAIR(0) A2ATS_PAIR(1) A2ATS_PAIR(2) A2ATS_PAIR(3)
#undef A2ATS_PAIR
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = bad ? 0x7fc07fc0u : x[i];
  *(uint4*)p = make_uint4(x[0], x[1], x[2], x[3]);
}

// A wave has 16 rows, 16 lanes a row.
template <typename T>
__global__ __launch_bounds__(256) void kv4_read_kernel(Kv4Cache m, int n_rows, int ctx_len, const int32_t* __restrict__ seq_lens,
                                                       const int32_t* __restrict__ new_lens, T* __restrict__ k_out,
                                                       T* __restrict__ v_out, int parts) {
  const int part = blockIdx.x % parts, bh = blockIdx.x / parts;
  const int b = bh / m.at.n_kv_heads, kv = bh % m.at.n_kv_heads;
  int n = seq_lens ? seq_lens[b] : ctx_len;
  n = min(max(n, 0), ctx_len);
  int cnt = new_lens ? new_lens[b] : n_rows;
  cnt = min(max(cnt, 0), min(n_rows, n));
  const int start = n - cnt, shift = m.at.shift;
  const int tid = threadIdx.x, lane = tid & 63, slot = lane >> 4, j = lane & 15;
  const int t0 = part * kKv4ReadRows + (tid >> 6) * 16;
  uint32_t kw[4];
  uint4 vw[4];
  uint2 sc[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int t = t0 + i * 4 + slot;
    if (t >= cnt) continue;
    const int row = start + t;
    const size_t r = (block_at(m.at, b, kv, row >> shift) << shift) + (size_t)(row & ((1 << shift) - 1));
    kw[i] = *(const uint32_t*)(m.rows + r * kKv4RowBytes + j * 4);
    vw[i] = *(const uint4*)(m.rows + r * kKv4RowBytes + kKv4Half + (j & 3) * 16);
    sc[i] = *(const uint2*)(m.scales + r * kKv4ScaleBytes);
  }
  const int g = j >> 2;
  const uint32_t pick = 0x0c0c0000u | (uint32_t)(4 + g) << 8 | (uint32_t)g;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int t = t0 + i * 4 + slot;
    if (t >= cnt) continue;
    const size_t to = ((size_t)bh * n_rows + t) * D + j * 8;
    const uint32_t kb = (sc[i].x >> (8 * g)) & 255u, vb = (sc[i].y >> (8 * g)) & 255u;
    if (k_out) store_numbers(k_out + to, kw[i], kv4_scale(kb), kb == 255u);
    if (v_out) {
      const uint32_t lower = __builtin_amdgcn_perm(vw[i].y, vw[i].x, pick), upper = __builtin_amdgcn_perm(vw[i].w, vw[i].z, pick);
      store_numbers(v_out + to, lower | upper << 16, kv4_scale(vb), vb == 255u);
    }
  }
}

}  // namespace

hipError_t launch_kv4_append(const a2ats_dims& d, const Kv4Cache& m, int kv_dtype, const void* k_new, const void* v_new, int n_new,
                             const int32_t* seq_lens, const int32_t* new_lens, hipStream_t stream) {
  const long bh = (long)d.batch * d.n_kv_heads;
  if (bh == 0 || n_new == 0 || d.ctx_len == 0) return hipSuccess;
  const int parts = append_parts(n_new, 1 << m.at.shift);
  const dim3 grid((unsigned)(bh * parts * 2));
#define A2ATS_APPEND(T, NW)                                                                                                  \
  hipLaunchKernelGGL((kv4_append_kernel<T, NW>), grid, dim3(NW * 64), 0, stream, m, (const T*)k_new, (const T*)v_new, n_new, \
                     d.ctx_len, seq_lens, new_lens, parts)
  const bool four = append_waves(1 << m.at.shift) == 4;
  if (kv_dtype == A2ATS_BF16) {
    if (four) A2ATS_APPEND(uint16_t, 4);
    else A2ATS_APPEND(uint16_t, 8);
  } else {
    if (four) A2ATS_APPEND(float, 4);
    else A2ATS_APPEND(float, 8);
  }
#undef A2ATS_APPEND
  return hipGetLastError();
}

hipError_t launch_kv4_read(const a2ats_dims& d, const Kv4Cache& m, int n_rows, const int32_t* seq_lens, const int32_t* new_lens,
                           void* k_out, void* v_out, int out_dtype, hipStream_t stream) {
  const long bh = (long)d.batch * d.n_kv_heads;
  if (bh == 0 || n_rows == 0 || d.ctx_len == 0 || (!k_out && !v_out)) return hipSuccess;
  const int parts = (n_rows + kKv4ReadRows - 1) / kKv4ReadRows;
  const dim3 grid((unsigned)(bh * parts));
  if (out_dtype == A2ATS_BF16)
    hipLaunchKernelGGL((kv4_read_kernel<uint16_t>), grid, dim3(256), 0, stream, m, n_rows, d.ctx_len, seq_lens, new_lens,
                       (uint16_t*)k_out, (uint16_t*)v_out, parts);
  else
    hipLaunchKernelGGL((kv4_read_kernel<float>), grid, dim3(256), 0, stream, m, n_rows, d.ctx_len, seq_lens, new_lens,
                       (float*)k_out, (float*)v_out, parts);
  return hipGetLastError();
}

}  // namespace a2ats
