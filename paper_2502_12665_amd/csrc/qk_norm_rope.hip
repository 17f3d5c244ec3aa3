// Norms of queries and keys, head by head, and their rotation by the tokens' positions, in one pass:
//     y = x w / sqrt(mean(x^2) + eps),   y R_p,
// each output rounded once, from float32.  Where a sum of squares overflows, or is so small that squares are lost, it is that of
// x 2^-e, |x| < 2 * 2^e; e >= -60, so that eps 2^-2e does not overflow either.
//
// A stream: 128 e bytes a head in, as many for each output.  16 lanes a row, a wave four rows at a time of one token, so that
// the token's angles are loaded once for 16 heads.  Measured: 32768 tokens of 32 + 8 heads in bfloat16 with q_pos, k_norm and k_pos
// 146 us (755 MB, 5.2 TB/s; 159 with outputs that stay in L2, 163 with all squares scaled); 4 x 1021 tokens of 28 + 4 heads in float32
// 15 us (87 MB, in part from the caches; 20 with 32 bytes of a row a lane, which are half lines at a time); a token of 16 sequences 4.0 us: a launch,
// 1.6, and length -> row -> root.  (All of a pass in a graph.  Single kernels as rocprofv3 has them: 147 us and more for the 146, 154 on average; 4.5
// to 4.8 for the 4.0.)  32768 tokens of 8 + 1 heads 36 us and keys alone of 8 heads 27, a copy's rate; of 1 + 1 heads 23 against 12, as 14 of a wave's
// 16 places have no row.
#include "internal.hpp"
#include "kv_blocks.hpp"

namespace a2ats {
namespace {

constexpr int D = 128;
constexpr int kWaveHeads = 16;

template <int CTRL>
__device__ __forceinline__ uint32_t lane_of(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
template <int CTRL>
__device__ __forceinline__ float lane_of(float v) { return __uint_as_float(lane_of<CTRL>(__float_as_uint(v))); }
// Over the 16 lanes of a row.
template <typename T, typename F>
__device__ __forceinline__ T over_row(T v, F f) {
  v = f(v, lane_of<0xB1>(v));      // quad_perm [1,0,3,2]
  v = f(v, lane_of<0x4E>(v));      // quad_perm [2,3,0,1]
  v = f(v, lane_of<0x124>(v));     // row_ror:4
  return f(v, lane_of<0x128>(v));  // row_ror:8
}
__device__ __forceinline__ float sum_of_squares(const float (&x)[8]) {
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) sum += x[e] * x[e];
  return over_row(sum, [](float a, float b) { return a + b; });
}

// Eight elements of a row's 16 lanes, which are loaded and stored 16 bytes a lane, all of them behind each other: bfloat16 8 j + 0 .. 7, the other half of
// a rotated pair is eight lanes on; float32 4 j + 0 .. 3 and 64 + 4 j + 0 .. 3, the pair in one lane.  Outputs go past the caches: probably a launch
// does not end before what it left in L2 is written.
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
template <typename T>
struct Eight;
template <>
struct Eight<uint16_t> {
  template <typename U>
  static __device__ __forceinline__ void load(const U* row, int j, float (&x)[8]) { load8(row + j * 8, x); }
  // The angles' cos and sin, with the sign of the other half.
  static __device__ __forceinline__ void angles(const float* c, const float* s, int j, float (&cs)[8], float (&sn)[8]) {
    load8(c + (j & 7) * 8, cs);
    load8(s + (j & 7) * 8, sn);
#pragma unroll
    for (int e = 0; e < 8; ++e) sn[e] = j < 8 ? -sn[e] : sn[e];
  }
  static __device__ __forceinline__ float other_half(const float (&y)[8], int e) { return lane_of<0x128>(y[e]); }
  static __device__ __forceinline__ void store(uint16_t* row, int j, const float (&x)[8]) {
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){x[2 * i], x[2 * i + 1]}, bf16x2));   // (to the nearest)
    __builtin_nontemporal_store(w, (u32x4*)(row + j * 8));
  }
};
template <>
struct Eight<float> {
  static __device__ __forceinline__ void load(const float* row, int j, float (&x)[8]) {
    const f32x4 a = *(const f32x4*)(row + j * 4), b = *(const f32x4*)(row + 64 + j * 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) { x[e] = a[e]; x[e + 4] = b[e]; }
  }
  static __device__ __forceinline__ void angles(const float* c, const float* s, int j, float (&cs)[8], float (&sn)[8]) {
    const f32x4 a = *(const f32x4*)(c + j * 4), b = *(const f32x4*)(s + j * 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) { cs[e] = cs[e + 4] = a[e]; sn[e] = -b[e]; sn[e + 4] = b[e]; }
  }
  static __device__ __forceinline__ float other_half(const float (&y)[8], int e) { return y[e ^ 4]; }
  static __device__ __forceinline__ void store(float* row, int j, const float (&x)[8]) {
    __builtin_nontemporal_store(f32x4{x[0], x[1], x[2], x[3]}, (f32x4*)(row + j * 4));
    __builtin_nontemporal_store(f32x4{x[4], x[5], x[6], x[7]}, (f32x4*)(row + 64 + j * 4));
  }
};

// Waves: [b][token][chunk of 16 heads]; the queries' heads before the keys'.
template <typename T>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(QkNormArgs a, int batch, int Hq, int Hkv, int n_new, int ctx_len, int chunks) {
  const uint32_t wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  const uint32_t token = wave / (uint32_t)chunks;   // (fewer than 2^26; rows of outputs fewer than 2^30)
  const int chunk = (int)(wave % (uint32_t)chunks), b = (int)(token / (uint32_t)n_new), t = (int)(token % (uint32_t)n_new);
  if (b >= batch) return;
  int n = a.seq_lens ? a.seq_lens[b] : ctx_len;
  n = min(max(n, 0), ctx_len);
  int cnt = a.new_lens ? a.new_lens[b] : n_new;
  cnt = min(max(cnt, 0), min(n_new, n));
  if (t >= cnt) return;
  const int lane = threadIdx.x & 63, slot = lane >> 4, j = lane & 15;
  const int first = a.q ? 0 : Hq, last = a.k ? Hq + Hkv : Hq;
  const int h0 = first + chunk * kWaveHeads;

  float x[4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int h = h0 + i * 4 + slot;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[i][e] = 0.f;
    if (h < last) {
      const T* from = h < Hq ? (const T*)a.q + (size_t)token * a.q_stride + (size_t)h * D
                             : (const T*)a.k + (size_t)token * a.k_stride + (size_t)(h - Hq) * D;
      Eight<T>::load(from, j, x[i]);
    }
  }
  const bool turn = a.q_pos != nullptr || a.k_pos != nullptr;
  float cs[8], sn[8];
  if (turn) {
    const size_t at = (size_t)(n - cnt + t) * (D / 2);
    Eight<T>::angles(a.cos_pos + at, a.sin_pos + at, j, cs, sn);
  }
  float wq[8], wk[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) wq[e] = wk[e] = 1.f;
  if (a.q_weight) Eight<T>::load(a.q_weight, j, wq);
  if (a.k_weight) Eight<T>::load(a.k_weight, j, wk);
  float w[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int h = h0 + i * 4 + slot;
    const bool query = h < Hq;
    if (i == 0 || (h0 + i * 4 + 3 >= Hq && h0 + i * 4 - 4 < Hq)) {   // (uniform; else they are those of the heads before)
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = query ? wq[e] : wk[e];
    }
    float sum = sum_of_squares(x[i]), eps = a.eps;
    // Squares that are lost below 2^-126 are below 2^-59 of such a sum, or of such an eps.
    const bool far = !(sum < 0x1p126f) || (sum < 0x1p-60f && eps < 0x1p-60f);
    if (__builtin_amdgcn_ballot_w64(far)) {
      uint32_t big = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) big = max(big, __float_as_uint(x[i][e]) & 0x7fffffffu);
      big = over_row(big, [](uint32_t p, uint32_t q) { return max(p, q); });
      const int e0 = far ? min(max((int)(big >> 23) - 127, -60), 126) : 0;
      const float down = __uint_as_float((uint32_t)(127 - e0) << 23);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[i][e] *= down;
      sum = sum_of_squares(x[i]);
      eps = ldexpf(eps, -2 * e0);
    }
    const float r = rsqrtf(sum * (1.f / D) + eps);
    float y[8], z[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = x[i][e] * r * w[e];
    if (turn) {
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] = Eight<T>::other_half(y, e) * sn[e] + y[e] * cs[e];
    }
    if (h < last) {
      const uint32_t row = (uint32_t)(query ? b * Hq + h : b * Hkv + h - Hq) * (uint32_t)n_new + (uint32_t)t;
      const size_t to = (size_t)row * D;
      T* norm = (T*)(query ? a.q_norm : a.k_norm);
      T* pos = (T*)(query ? a.q_pos : a.k_pos);
      if (norm) Eight<T>::store(norm + to, j, y);
      if (pos) Eight<T>::store(pos + to, j, z);
    }
  }
}

}  // namespace

static int norm_chunks(const a2ats_dims& d, bool q, bool k) {
  return ((q ? d.n_q_heads : 0) + (k ? d.n_kv_heads : 0) + kWaveHeads - 1) / kWaveHeads;
}
long qk_norm_waves(const a2ats_dims& d, int n_new, bool q, bool k) { return (long)d.batch * n_new * norm_chunks(d, q, k); }

hipError_t launch_qk_norm_rope(const a2ats_dims& d, int dtype, int n_new, const QkNormArgs& a, hipStream_t stream) {
  const long waves = qk_norm_waves(d, n_new, a.q != nullptr, a.k != nullptr);
  if (waves == 0 || d.ctx_len == 0) return hipSuccess;
  const int chunks = norm_chunks(d, a.q != nullptr, a.k != nullptr);
  const dim3 grid((unsigned)((waves + 3) / 4));
  if (dtype == A2ATS_BF16)
    hipLaunchKernelGGL((qk_norm_rope_kernel<uint16_t>), grid, dim3(256), 0, stream, a, d.batch, d.n_q_heads, d.n_kv_heads, n_new,
                       d.ctx_len, chunks);
  else
    hipLaunchKernelGGL((qk_norm_rope_kernel<float>), grid, dim3(256), 0, stream, a, d.batch, d.n_q_heads, d.n_kv_heads, n_new,
                       d.ctx_len, chunks);
  return hipGetLastError();
}

}  // namespace a2ats
