// Appending tokens to a key/value cache held in 4 bits, and reading them back.
//
// A group of 32 dimensions of a token's key (or value) is rounded by itself: with a = max |x| its scale is the least power of
// two 2^e with a <= 6 * 2^e, and a code is x / 2^e to the nearest e2m1 number (0, 1/2, 1, 3/2, 2, 3, 4, 6), ties to even.  So a
// row depends on nothing but itself: there is no tail, and a token can be written again.  x / 2^e is exact, and
// v_cvt_scalef32_pk_fp4_f32 rounds it as for real numbers.
//
// Both are streams, 2 * 128 * e bytes against 136.  16 lanes have a row, eight elements each: a group's largest is two steps over
// four lanes, and a wave stores whole rows of 64 bytes.  Keys and values have workgroups of their own (kv8_append.hip has them so, by which
// a token of 16 sequences is twice as many workgroups).  Measured: append of 32768 tokens of 8 heads in bfloat16 33 us with bounds (170 MB,
// 5.2 TB/s), 4 x 4 heads of 4099 tokens in float32 14.8 us (76 MB, 5.2 TB/s); a token of 16 x 8 heads 4.0 us: a launch, 1.6, and length -> rows.
// bfloat16 is rounded as it comes from memory, and its bounds are taken two at a time as whole numbers: as float32 it was 8 us more.  Reading back 65536
// tokens of 4 heads in bfloat16 27 us (170 MB, 6.2 TB/s; 35 with outputs that stay in L2), 4 x 4 heads of 4099 tokens in float32 11 us.  Both at
// a copy's rate: what is read once, and what is read back, passes the caches; the cache's own rows do not, 4 bytes a lane of two workgroups'
// lines (7 us more).
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

typedef __attribute__((ext_vector_type(2))) short i16x2;
typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

// Eight elements of a row, of which 16 consecutive lanes have all, as they come from memory.
template <typename T>
struct Eight;
template <>
struct Eight<float> {
  float x[8];
  __device__ __forceinline__ void load(const float* p) { load8(p, x); }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.f;
  }
  __device__ __forceinline__ uint32_t largest() const {   // magnitude, as bits
    uint32_t big = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) big = max(big, __float_as_uint(x[e]) & 0x7fffffffu);
    return big;
  }
  __device__ __forceinline__ uint32_t codes(float scale) const {   // the first in the lowest bits
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
    return w;
  }
};
template <>
struct Eight<uint16_t> {
  uint32_t x[4];
  __device__ __forceinline__ void load(const uint16_t* p) {
    typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
    const u32x4 v = __builtin_nontemporal_load((const u32x4*)p);   // (read once)
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = v[e];
  }
  __device__ __forceinline__ void zero() { x[0] = x[1] = x[2] = x[3] = 0u; }
  __device__ __forceinline__ uint32_t largest() const {   // (two at a time, 16 bits each)
    u16x2 big = __builtin_bit_cast(u16x2, x[0] & 0x7fff7fffu);
#pragma unroll
    for (int e = 1; e < 4; ++e) big = __builtin_elementwise_max(big, __builtin_bit_cast(u16x2, x[e] & 0x7fff7fffu));
    return (uint32_t)max(big[0], big[1]) << 16;
  }
  __device__ __forceinline__ uint32_t codes(float scale) const {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x[0]), scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x[1]), scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x[2]), scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x[3]), scale, 3);
    return w;
  }
};

// Their codes, and the scale byte of the group, which four lanes share.
template <typename T>
__device__ __forceinline__ uint32_t codes8(const Eight<T>& x, uint32_t& byte) {
  uint32_t big = x.largest();
  big = max(big, lane_of<kXor1>(big));
  big = max(big, lane_of<kXor2>(big));
  const bool usable = big >= kTinyBits && big < kHugeBits;
  // 6 = 1.5 * 2^2
  byte = usable ? (big >> 23) - 2u + ((big & 0x7fffffu) > 0x400000u ? 1u : 0u) : (big < kTinyBits ? 0u : 255u);
  const uint32_t w = x.codes(kv4_scale(usable ? byte : 127u));
  return usable ? w : 0u;
}

// The smallest and largest key of each of eight dimensions: of a lane's rows, then of the lane rows, whose bounds of two dimensions lane row r
// is left with (2 r and 2 r + 1), then of the waves (from LDS).
template <typename T>
struct Bounds;
template <>
struct Bounds<float> {
  typedef float Elem;
  float lo[8], hi[8];
  bool any_nan;
  __device__ __forceinline__ Bounds() : any_nan(false) {
#pragma unroll
    for (int e = 0; e < 8; ++e) { lo[e] = INFINITY; hi[e] = -INFINITY; }
  }
  // `there`: the row counts.
  __device__ __forceinline__ void add(const Eight<float> (&x)[4], const bool (&there)[4]) {
    uint32_t big = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) big = max(big, x[i].largest());
    any_nan = __builtin_amdgcn_ballot_w64(big > 0x7f800000u) != 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (there[i]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          lo[e] = any_nan ? low(lo[e], x[i].x[e]) : min2(lo[e], x[i].x[e]);
          hi[e] = any_nan ? high(hi[e], x[i].x[e]) : max2(hi[e], x[i].x[e]);
        }
      }
  }
  __device__ __forceinline__ void store(float* s_lo, float* s_hi) const {
    *(float2*)s_lo = any_nan ? over_lane_rows(lo, low) : over_lane_rows(lo, min2);
    *(float2*)s_hi = any_nan ? over_lane_rows(hi, high) : over_lane_rows(hi, max2);
  }
  static __device__ __forceinline__ float none_low() { return INFINITY; }
  static __device__ __forceinline__ float none_high() { return -INFINITY; }
  static __device__ __forceinline__ float of(float x) { return x; }
  static __device__ __forceinline__ float least(float a, float b) { return low(a, b); }
  static __device__ __forceinline__ float most(float a, float b) { return high(a, b); }
  static __device__ __forceinline__ void put(float* p, float lo, float hi) {
    p[0] = lo;
    p[D] = hi;
  }
};
// bfloat16, two at a time, as whole numbers of the same order: the lower 15 bits of negative ones turned over.  What is not a number is beyond
// the infinities, by its sign, and makes both bounds one at the end.
template <>
struct Bounds<uint16_t> {
  typedef short Elem;
  i16x2 lo[4], hi[4];
  __device__ __forceinline__ Bounds() {
#pragma unroll
    for (int e = 0; e < 4; ++e) { lo[e] = i16x2{0x7fff, 0x7fff}; hi[e] = i16x2{-0x8000, -0x8000}; }
  }
  __device__ __forceinline__ void add(const Eight<uint16_t> (&x)[4], const bool (&there)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (there[i]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const i16x2 y = __builtin_bit_cast(i16x2, x[i].x[e]);
          const i16x2 z = y ^ ((y >> 15) & i16x2{0x7fff, 0x7fff});
          lo[e] = __builtin_elementwise_min(lo[e], z);
          hi[e] = __builtin_elementwise_max(hi[e], z);
        }
      }
  }
  template <typename F>
  static __device__ __forceinline__ uint32_t pair(uint32_t a, uint32_t b, F f) {
    return __builtin_bit_cast(uint32_t, f(__builtin_bit_cast(i16x2, a), __builtin_bit_cast(i16x2, b)));
  }
  template <typename F>
  static __device__ __forceinline__ uint32_t over_rows(const i16x2 (&v)[4], F f) {
    uint32_t h[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const auto s = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v[e]), __builtin_bit_cast(uint32_t, v[e + 2]), false, false);
      h[e] = pair(s[0], s[1], f);
    }
    const auto s = __builtin_amdgcn_permlane16_swap(h[0], h[1], false, false);
    return pair(s[0], s[1], f);
  }
  __device__ __forceinline__ void store(short* s_lo, short* s_hi) const {
    *(uint32_t*)s_lo = over_rows(lo, [](i16x2 a, i16x2 b) { return __builtin_elementwise_min(a, b); });
    *(uint32_t*)s_hi = over_rows(hi, [](i16x2 a, i16x2 b) { return __builtin_elementwise_max(a, b); });
  }
  static __device__ __forceinline__ short none_low() { return 0x7fff; }
  static __device__ __forceinline__ short none_high() { return -0x8000; }
  static __device__ __forceinline__ short of(uint16_t x) { return (short)(x ^ (((short)x >> 15) & 0x7fff)); }
  static __device__ __forceinline__ short least(short a, short b) { return b < a ? b : a; }
  static __device__ __forceinline__ short most(short a, short b) { return b > a ? b : a; }
  static __device__ __forceinline__ void put(uint16_t* p, short lo, short hi) {
    const bool nan = hi > 0x7f80 || lo < -0x7f81;
    p[0] = nan ? (uint16_t)0x7fc0 : (uint16_t)of((uint16_t)lo);
    p[D] = nan ? (uint16_t)0x7fc0 : (uint16_t)of((uint16_t)hi);
  }
};

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
  typedef typename Bounds<T>::Elem Bound;
  __shared__ __align__(8) Bound s_lo[NW][D], s_hi[NW][D];
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

  Eight<T> x[4];
  bool there[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = w0 + i * 4 + slot;
    there[i] = row >= start && row < n;
    x[i].zero();
    if (there[i]) x[i].load(fresh + (size_t)(row - start) * D + d0);
  }
  if (live) {
    const size_t at = (block_at(m.at, b, kv, w0 >> shift) << shift) + (size_t)(w0 & (blk - 1));
    const ValueOrder order(j >> 2);
    const int word = what ? 16 + 4 * (j & 3) + (j >> 2) : j;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t byte;
      uint32_t w = codes8(x[i], byte);
      if (what) w = order.apply(w);
      byte <<= 8 * (j >> 2);
      byte |= lane_of<kNext4>(byte);
      byte |= lane_of<kNext8>(byte);
      if (there[i]) {
        const size_t r = at + (size_t)(i * 4 + slot);
        *(uint32_t*)(m.rows + r * kKv4RowBytes + word * 4) = w;
        if (j == 0) *(uint32_t*)(m.scales + r * kKv4ScaleBytes + what * 4) = byte;
      }
    }
  }
  if (!bounds) return;   // (uniform)
  Bounds<T> bd;
  bd.add(x, there);
  bd.store(&s_lo[wv][d0 + 2 * slot], &s_hi[wv][d0 + 2 * slot]);
  __syncthreads();
  const int per = blk / kWaveRows;   // waves of a block
  T* all = (T*)m.at.bounds;
  for (int i = tid; i < SLAB / blk * D; i += NT) {
    const int cb = i / D, d = i % D, ci = (r0 >> shift) + cb, t0 = ci << shift;
    if (t0 >= n) break;
    Bound lo = Bounds<T>::none_low(), hi = Bounds<T>::none_high();
    for (int w = cb * per; w < (cb + 1) * per; ++w) {
      lo = Bounds<T>::least(lo, s_lo[w][d]);
      hi = Bounds<T>::most(hi, s_hi[w][d]);
    }
    T* p = all + block_at(m.at, b, kv, ci) * 2 * D + d;
    if (t0 < start) {   // the block had tokens before
      lo = Bounds<T>::least(lo, Bounds<T>::of(p[0]));
      hi = Bounds<T>::most(hi, Bounds<T>::of(p[D]));
    }
    Bounds<T>::put(p, lo, hi);
  }
}

// What 16 lanes have of a row that is read back, and how they store its numbers: 16 bytes a lane, all of them behind each other, past the
// caches (27 us instead of 35 for 65536 tokens; probably as a launch does not end before what it left in L2 is written).
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
template <typename T>
struct ReadRow;
// bfloat16: lane j the dimensions 8 j + 0 .. 7, of group j / 4: a word of the key's codes, and the value's bytes n = 4 (j % 4) + 0 .. 3 of all groups.
template <>
struct ReadRow<uint16_t> {
  uint32_t k;
  uint4 v;
  uint2 sc;
  __device__ __forceinline__ void load(const uint8_t* row, const uint8_t* scales, int j) {
    k = *(const uint32_t*)(row + j * 4);
    v = *(const uint4*)(row + kKv4Half + (j & 3) * 16);
    sc = *(const uint2*)scales;
  }
  static __device__ __forceinline__ void put(uint16_t* to, int j, uint32_t w, uint32_t byte) {
    const float scale = kv4_scale(byte);
    u32x4 x;
#define A2ATS_PAIR(i) x[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, i));
    A2ATS_PAIR(0) A2ATS_PAIR(1) A2ATS_PAIR(2) A2ATS_PAIR(3)
#undef A2ATS_PAIR
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = byte == 255u ? 0x7fc07fc0u : x[i];
    __builtin_nontemporal_store(x, (u32x4*)(to + j * 8));
  }
  __device__ __forceinline__ void key(uint16_t* to, int j) const { put(to, j, k, (sc.x >> (8 * (j >> 2))) & 255u); }
  __device__ __forceinline__ void value(uint16_t* to, int j) const {
    const int g = j >> 2;
    const uint32_t pick = 0x0c0c0000u | (uint32_t)(4 + g) << 8 | (uint32_t)g;
    const uint32_t lower = __builtin_amdgcn_perm(v.y, v.x, pick), upper = __builtin_amdgcn_perm(v.w, v.z, pick);
    put(to, j, lower | upper << 16, (sc.y >> (8 * g)) & 255u);
  }
};
// float32: lane j the dimensions 4 j + 0 .. 3 and 64 + 4 j + 0 .. 3, of the groups j / 8 and 2 + j / 8: half of two words of the key's codes, and
// the value's bytes n = 2 (j % 8) + {0, 1} of all groups.
template <>
struct ReadRow<float> {
  uint32_t k[2];
  uint2 v, sc;
  __device__ __forceinline__ void load(const uint8_t* row, const uint8_t* scales, int j) {
    k[0] = *(const uint16_t*)(row + j * 2);
    k[1] = *(const uint16_t*)(row + 32 + j * 2);
    v = *(const uint2*)(row + kKv4Half + (j & 7) * 8);
    sc = *(const uint2*)scales;
  }
  static __device__ __forceinline__ void put(float* to, uint32_t w, uint32_t byte) {
    const float scale = kv4_scale(byte);
    const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
    f32x4 x = {a[0], a[1], b[0], b[1]};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = byte == 255u ? __uint_as_float(0x7fc00000u) : x[i];
    __builtin_nontemporal_store(x, (f32x4*)to);
  }
  __device__ __forceinline__ void key(float* to, int j) const {
#pragma unroll
    for (int h = 0; h < 2; ++h) put(to + 64 * h + 4 * j, k[h], (sc.x >> (16 * h + 8 * (j >> 3))) & 255u);
  }
  __device__ __forceinline__ void value(float* to, int j) const {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int g = 2 * h + (j >> 3);
      put(to + 64 * h + 4 * j, __builtin_amdgcn_perm(v.y, v.x, 0x0c0c0000u | (uint32_t)(4 + g) << 8 | (uint32_t)g), (sc.y >> (8 * g)) & 255u);
    }
  }
};

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
  ReadRow<T> x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int t = t0 + i * 4 + slot;
    if (t >= cnt) continue;
    const int row = start + t;
    const size_t r = (block_at(m.at, b, kv, row >> shift) << shift) + (size_t)(row & ((1 << shift) - 1));
    x[i].load(m.rows + r * kKv4RowBytes, m.scales + r * kKv4ScaleBytes, j);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int t = t0 + i * 4 + slot;
    if (t >= cnt) continue;
    const size_t to = ((size_t)bh * n_rows + t) * D;
    if (k_out) x[i].key(k_out + to, j);
    if (v_out) x[i].value(v_out + to, j);
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
