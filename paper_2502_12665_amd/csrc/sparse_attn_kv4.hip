// Attention of one query token over sinks U selected tokens (or blocks) U window, from a cache held in 4 bits with a scale for
// each 32 dimensions of a token's key and value:
//     logit_j = (q~ . k_j) / sqrt(128)  (window rows: q R_delta for q~),  out = sum softmax(logit)_j v_j.
//
// A row is 128 bytes of codes and 8 of scales, 4 flop per byte and head: a gather.  Both products are on the matrix cores, also
// for one head, with the 16 columns of a tile used for the precision of the float32 operand:
//   - keys (A, 16 rows x 128) times queries (B).  Lane row r has the dimensions 32 r .. 32 r + 31 of its column's row, which is a group:
//     16 bytes of codes and one scale, with which they become bfloat16 (exact: two bits of significand) as they are converted.  The
//     query is three bfloat16 terms by truncation, all of its 24 bits, a column each (eight heads have two columns each, and a
//     second product for the third term).  The products of 4-bit and 8-bit operands with scales of their own would take the codes as
//     they are, but their sums are not those of float32 (off by up to 2^-13 of the sum of magnitudes, measured).
//   - values (A, 16 dimensions x 32 rows) times weights (B).  Logits leave the first product with a head in each column and
//     four rows of each of two tiles in each lane, which is the B operand of the second as it stands.  A row has four scales, which
//     multiply the weight: a column takes the scale of one group, and of a tile's products only the columns of its own group count.
//     One head: 16 columns are four groups times the three bfloat16 terms of a weight; up to four heads: head times group, and a
//     product for each term; eight: head times half the groups, and two sets of weights.  A lane loads four bytes of each of its 8 rows,
//     two dimensions of each group; two rows' words are put together by halves of bytes, and each byte is then a pair of
//     rows of one dimension, which converts to two bfloat16.
// Window rows are turned back by their distance, (q R_delta) . k = q . (k R_-delta), relative to the row's largest scale, and go
// in as two float16 terms (2^-23 of an element, 2^-26 of the row's largest).
// The statistics, all sums and the output are float32.  Logits are kept times log2 e, so that a weight is one exponential.
#include <algorithm>

#include "internal.hpp"
#include "kv_attn.hpp"

namespace a2ats {
namespace {

constexpr int kD = 128;
constexpr int kThreads = 256, kWaves = kThreads / 64;

struct Attn4Args {
  Kv4Cache cache;
  const void* q;
  const float* q_rot;
  const int32_t* sel_idx;
  const int32_t* sel_count;
  const float* cos_win;
  const float* sin_win;
  const int32_t* seq_lens;
  float* partial;
  void* out;
  int32_t ctx_len, n_sel, sel_shift, window, n_sink, group, shared, problems;
  int32_t parts, far_share, win_share;   // workgroups of a head's (KV head's) rows, and how many of them each takes
};

// The rows of a pair of tiles as they come from memory: 32 dimensions of the key of row `column` of either tile; of the values of
// the rows 4 * lane row + 0 .. 3 of either, two dimensions of each group.
struct PairRows {
  uint4 k[2];
  uint32_t v[8];
};
// Where the rows of two pairs are in the cache, the keys' scale bytes, what the finished product is multiplied by, 0 or, for a
// place without a row, all bits, and the values' scales by group: of a wave, in LDS.
struct alignas(16) PairPlaces {
  uint32_t row[2 * kPair];
  uint32_t ksc[2 * kPair];
  float ks[2 * kPair];
  uint32_t none[2 * kPair];
  float vs[4][2 * kPair];
};

// A wave's running softmax: a head in each column (the same m in all lane rows, l of the lane's own rows), and its output,
// o[t][i] being dimension 32 (t / 2) + 2 (4 * lane row + i) + t % 2, in the columns of group t / 2.
struct WaveState {
  float m, l;
  f32x4 o[8];
};

template <int NH>
struct Columns {
  static constexpr int kTerms = NH == 8 ? 2 : 4;   // of the query: columns of a head in the first product
  // Which head, term of the query, group (eight heads: half of the groups) and term of the weights a column has.
  static __device__ __forceinline__ int head(int col) { return NH == 1 ? 0 : col % NH; }
  static __device__ __forceinline__ int q_term(int col) { return NH == 1 ? col & 3 : col / NH; }
  static __device__ __forceinline__ int group(int col) { return NH == 1 ? col & 3 : col / NH; }
  static __device__ __forceinline__ int w_term(int col) { return NH == 1 ? col >> 2 : 0; }
  // The sum over the terms of the query: the same bits in each column of a head.
  static __device__ __forceinline__ float sum(float v) {
    if (NH == 1) {
      v += dpp<0xB1>(v);   // quad_perm [1,0,3,2]
      v += dpp<0x4E>(v);   // quad_perm [2,3,0,1]
      return v;
    }
    return head_sum<NH == 1 ? 4 : NH>(v);
  }
};

__device__ __forceinline__ void load_pair(const uint8_t* cache, const uint32_t* rows, int col, int lrow, PairRows& p) {
#pragma unroll
  for (int t = 0; t < 2; ++t) p.k[t] = *(const uint4*)(cache + (size_t)rows[t * 16 + col] * kKv4RowBytes + lrow * 16);
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const uint4 r4 = *(const uint4*)(rows + t * 16 + lrow * 4);
    const uint32_t r[4] = {r4.x, r4.y, r4.z, r4.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) p.v[4 * t + i] = *(const uint32_t*)(cache + (size_t)r[i] * kKv4RowBytes + kKv4Half + col * 4);
  }
}
// The keys of window rows: elements 16 * lane row + 0 .. 15 of either half.
__device__ __forceinline__ void load_turned_pair(const uint8_t* cache, const uint32_t* rows, int col, int lrow, PairRows& p) {
  load_pair(cache, rows, col, lrow, p);
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const uint8_t* from = cache + (size_t)rows[t * 16 + col] * kKv4RowBytes + lrow * 8;
    const uint2 a = *(const uint2*)from, b = *(const uint2*)(from + 32);
    p.k[t] = make_uint4(a.x, a.y, b.x, b.y);
  }
}

// The weights of the two tiles' rows of a lane, from their products with the queries (times log2 e / sqrt(128)); the state's
// maximum and sum.
__device__ __forceinline__ void pair_weights(const f32x4 (&dot)[2], const PairPlaces& pl, int first, int lrow, WaveState& st,
                                             float (&w)[8]) {
  float lg[8];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int at = first + t * 16 + lrow * 4;
    const float4 k4 = *(const float4*)(pl.ks + at);
    const uint4 n4 = *(const uint4*)(pl.none + at);
    const float kk[4] = {k4.x, k4.y, k4.z, k4.w};
    const uint32_t nn[4] = {n4.x, n4.y, n4.z, n4.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      lg[4 * t + i] = __uint_as_float((nn[i] & 0xff800000u) | (~nn[i] & __float_as_uint(dot[t][i] * kk[i])));   // (-inf)
  }
  float mx = lg[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) mx = fmaxf(mx, lg[i]);
  const float mn = fmaxf(st.m, rows_max(mx));
  if (__builtin_amdgcn_ballot_w64(mn > st.m)) {
    const float alpha = power(st.m - mn);
    st.l *= alpha;
#pragma unroll
    for (int t = 0; t < 8; ++t) st.o[t] *= alpha;
    st.m = mn;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    w[i] = power(lg[i] - mn);
    st.l += w[i];
  }
}

__device__ __forceinline__ bf16x8 pack8(const float (&x)[8]) {
  return __builtin_bit_cast(bf16x8, make_uint4(upper_halves(x[0], x[1]), upper_halves(x[2], x[3]), upper_halves(x[4], x[5]),
                                               upper_halves(x[6], x[7])));
}
// What is left of x without its upper half.
__device__ __forceinline__ float lower_part(float x) { return x - __uint_as_float(__float_as_uint(x) & 0xffff0000u); }

// The pair's values times its weights.
template <int NH>
__device__ __forceinline__ void absorb_values(const float (&weight)[8], const PairPlaces& pl, int first, int col, int lrow,
                                              const PairRows& p, WaveState& st) {
  // Weights times the scales of the column's group, as bfloat16 terms.
  constexpr int kSets = NH == 8 ? 2 : 1, kTerms = NH == 1 ? 1 : 3;
  bf16x8 b[kSets][kTerms];
#pragma unroll
  for (int set = 0; set < kSets; ++set) {
    const int g = NH == 8 ? 2 * Columns<NH>::group(col) + set : Columns<NH>::group(col);
    float x[8];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const float4 s4 = *(const float4*)(pl.vs[g] + first + t * 16 + lrow * 4);
      const float ss[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * t + i] = weight[4 * t + i] * ss[i];
    }
    if constexpr (NH == 1) {
      const int term = Columns<NH>::w_term(col);
      const uint32_t cut1 = term >= 1 ? 0xffff0000u : 0u, cut2 = term >= 2 ? 0xffff0000u : 0u, cut3 = term >= 3 ? 0u : ~0u;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] -= __uint_as_float(__float_as_uint(x[i]) & cut1);
        x[i] -= __uint_as_float(__float_as_uint(x[i]) & cut2);
        x[i] = __uint_as_float(__float_as_uint(x[i]) & cut3);
      }
      b[0][0] = pack8(x);
    } else {
#pragma unroll
      for (int term = 0; term < kTerms; ++term) {
        b[set][term] = pack8(x);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = lower_part(x[i]);
      }
    }
  }
  // Rows 2 i and 2 i + 1: byte g of even[i] has the first of the two dimensions of group g, of odd[i] the second; the lower half
  // of a byte is the first row's.
  uint32_t even[4], odd[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t a = p.v[2 * i], c = p.v[2 * i + 1];
    even[i] = (a & 0x0f0f0f0fu) | ((c << 4) & 0xf0f0f0f0u);
    odd[i] = ((a >> 4) & 0x0f0f0f0fu) | (c & 0xf0f0f0f0u);
  }
#define A2ATS_TILE(t)                                                                                                           \
  {                                                                                                                             \
    uint32_t w[4];                                                                                                              \
    _Pragma("unroll") for (int i = 0; i < 4; ++i)                                                                               \
        w[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((t) & 1 ? odd[i] : even[i], 1.f, (t) / 2)); \
    const bf16x8 vt = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));                                           \
    constexpr int set = NH == 8 ? (t) / 2 % 2 : 0;                                                                              \
    _Pragma("unroll") for (int term = 0; term < kTerms; ++term)                                                                 \
        st.o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, b[set][term], st.o[t], 0, 0, 0);                                  \
  }
  A2ATS_TILE(0) A2ATS_TILE(1) A2ATS_TILE(2) A2ATS_TILE(3) A2ATS_TILE(4) A2ATS_TILE(5) A2ATS_TILE(6) A2ATS_TILE(7)
#undef A2ATS_TILE
}

// The queries of far rows as the second operand: bfloat16 terms by truncation.
template <int NH>
struct FarQuery {
  bf16x8 q[4], q2[NH == 8 ? 4 : 1];   // (eight heads: the third term, in the first column of a head)
  // Elements 32 * lane row + 0 .. 31 of the column's head.
  __device__ __forceinline__ void set(const float (&x)[32], int term, bool active) {
    const uint32_t cut1 = term >= 1 ? 0xffff0000u : 0u, cut2 = term >= 2 ? 0xffff0000u : 0u;
    const uint32_t keep = active && term < 3 ? ~0u : 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float y[8], z[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        y[e] = x[8 * i + e];
        z[e] = lower_part(lower_part(y[e]));
        z[e] = __uint_as_float(__float_as_uint(z[e]) & (term == 0 ? keep : 0u));
        y[e] -= __uint_as_float(__float_as_uint(y[e]) & cut1);
        if (NH != 8) y[e] -= __uint_as_float(__float_as_uint(y[e]) & cut2);
        y[e] = __uint_as_float(__float_as_uint(y[e]) & keep);
      }
      q[i] = pack8(y);
      if constexpr (NH == 8) q2[i] = pack8(z);
    }
  }
  // Products of a tile's keys (32 elements of row `column`) with the queries: rows 4 * lane row + i.
  __device__ __forceinline__ f32x4 dot(const uint4& k, float scale) const {
    const uint32_t kw[4] = {k.x, k.y, k.z, k.w};
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t w[4];
#define A2ATS_PAIR(e) w[e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(kw[i], scale, e));
      A2ATS_PAIR(0) A2ATS_PAIR(1) A2ATS_PAIR(2) A2ATS_PAIR(3)
#undef A2ATS_PAIR
      const bf16x8 k8 = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k8, q[i], acc, 0, 0, 0);
      if constexpr (NH == 8) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k8, q2[i], acc, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = Columns<NH>::sum(acc[i]);
    return acc;
  }
};

// Products of a tile's window keys (elements 16 * lane row + 0 .. 15 of either half of row `column`, whose groups have the scales
// s_lower and s_upper), turned back by the row's angles, with the queries' float16 terms.
__device__ __forceinline__ f32x4 turned_dot(const uint4& k, float s_lower, float s_upper, const float (&cs)[16], const float (&sn)[16],
                                            const f16x8 (&q)[4]) {
  const uint32_t lw[2] = {k.x, k.y}, uw[2] = {k.z, k.w};
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 2; ++i) {   // eight pairs of elements
    float lower[8], upper[8];
#define A2ATS_PAIR(e)                                                                          \
  {                                                                                            \
    const auto dl = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(lw[i], s_lower, e);               \
    const auto du = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(uw[i], s_upper, e);               \
    _Pragma("unroll") for (int j = 0; j < 2; ++j) {                                            \
      lower[2 * e + j] = dl[j] * cs[8 * i + 2 * e + j] + du[j] * sn[8 * i + 2 * e + j];        \
      upper[2 * e + j] = du[j] * cs[8 * i + 2 * e + j] - dl[j] * sn[8 * i + 2 * e + j];        \
    }                                                                                          \
  }
    A2ATS_PAIR(0) A2ATS_PAIR(1) A2ATS_PAIR(2) A2ATS_PAIR(3)
#undef A2ATS_PAIR
    auto terms = [&](const float (&x)[8], const f16x8& qt) {
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f16x2 h = f16_pair(x[2 * j], x[2 * j + 1]);
        hi[j] = f16_bits(h);
        lo[j] = f16_bits(f16_pair(x[2 * j] - (float)h[0], x[2 * j + 1] - (float)h[1]));
      }
      acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, make_uint4(hi[0], hi[1], hi[2], hi[3])), qt, acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, make_uint4(lo[0], lo[1], lo[2], lo[3])), qt, acc, 0, 0, 0);
    };
    terms(lower, q[i]);
    terms(upper, q[2 + i]);
  }
  return acc;
}

// NH: heads that attend the same rows, one, or the G of a KV head if the selection is shared, padded to 4 or 8.
template <typename T, int NH>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void attn_kv4_kernel(Attn4Args a) {
  __shared__ __align__(16) union {
    struct {
      PairPlaces far[kWaves][2], win[kWaves];
    } places;
    float o[kWaves][NH][kD];
  } s;
  __shared__ float s_m[kWaves][NH], s_l[kWaves][NH];
  typedef Columns<NH> C;

  // All workgroups of a KV head run on one XCD, whose L2 then serves the rows that its heads have in common.
  const int G = a.group, nh = a.shared ? G : 1, per = a.shared ? a.parts : a.parts * G;
  int prob, pg;
  xcd_map(blockIdx.x, per, a.problems, prob, pg);
  const BlockCache& blocks = a.cache.at;
  const int Hkv = blocks.n_kv_heads, b = prob / Hkv, kv = prob % Hkv;
  const int part = a.shared ? pg : pg / G;
  const int head = prob * G + (a.shared ? 0 : pg % G);   // the first of the workgroup's heads
  const int sel = a.shared ? prob : head;                // whose selection it reads
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, lrow = lane >> 4;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int32_t* idx = a.sel_idx + (size_t)sel * a.n_sel;

  // This part's share of the far rows: row t is sink t, then row t - n_sink of the selection.  Places without a row are left
  // out: what a part has to fetch first does not depend on the sequence's length.
  const int n_sink = min(a.n_sink, a.ctx_len);
  const int f0 = part * a.far_share;
  auto unit_of = [&](int t) {   // (clamped: requested before it is known to count)
    return a.n_sel > 0 ? idx[min(max(t - n_sink, 0) >> a.sel_shift, a.n_sel - 1)] : 0;
  };

  const SeqRange sr = seq_range(a.ctx_len, a.seq_lens, b, a.window, a.n_sink, 0);
  const int shift = blocks.shift, blk = 1 << shift;
  const int cnt = min(max(a.sel_count[sel], 0), a.n_sel);
  const int f1 = min(f0 + a.far_share, n_sink + (cnt << a.sel_shift));
  // ... and of the window's rows, [w0, w1).
  const int w0 = sr.win_start + part * a.win_share, w1 = max(w0, min(w0 + a.win_share, sr.n));
  const int n_far = f1 > f0 && sr.n > 0 ? (f1 - f0 + kPair - 1) / kPair : 0, n_win = (w1 - w0 + kPair - 1) / kPair;
  // Wave by wave, the pairs win_first, win_first + kWaves, .. of the window, and of the far rows a stretch, so that all waves have
  // about as much to do: a pair of the window is as much as two others.  Which wave of the SIMDs is the first goes by the
  // workgroup (the waves with the window would else be on one SIMD in all workgroups of a CU).
  const int win_first = (wv + (int)(blockIdx.x >> 3) + (int)(blockIdx.x >> 8)) & (kWaves - 1);
  const int quota = (2 * n_win + n_far + kWaves - 1) / kWaves;
  int far_first = 0, far_end = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const int take = max(quota - 2 * ((n_win - w + kWaves - 1) / kWaves), 0);   // (n_win + kWaves > w)
    far_first += w < win_first ? take : 0;
    far_end += w <= win_first ? take : 0;
  }
  far_first = min(far_first, n_far);
  far_end = min(far_end, n_far);
  // Lane l places row l % 32 of a pair (l < 32) or of the next one.
  auto far_row = [&](int pair) { return f0 + pair * kPair + lane; };
  int unit = unit_of(far_row(far_first));

  // This lane's column: a head.
  const int hd = C::head(col);
  const bool active = hd < nh;
  const size_t q_at = (size_t)(head + min(hd, nh - 1)) * kD;

  // Where this lane's row is, and its scales, which are requested here and put beside it by put_scales.
  struct Place {
    size_t at;
    uint2 sc;
    bool in;
  };
  auto place = [&](PairPlaces& to, int j, bool in) {   // row j of the sequence
    Place pc;
    pc.in = in;
    j = in ? j : 0;   // (a place without a row: the sequence's first one, which has been written and counts for nothing)
    pc.at = (block_at(blocks, b, kv, j >> shift) << shift) + (size_t)(j & (blk - 1));
    wave_exchange();
    to.row[lane] = (uint32_t)pc.at;
    wave_exchange();
    return pc;
  };
  auto get_scales = [&](Place& pc) { pc.sc = *(const uint2*)(a.cache.scales + pc.at * kKv4ScaleBytes); };
  // turned: products are relative to the row's largest scale.
  auto put_scales = [&](PairPlaces& to, const Place& pc, bool turned) {
    uint32_t most = 0;
#pragma unroll
    for (int g = 0; g < 4; ++g) most = max(most, (pc.sc.x >> (8 * g)) & 255u);
    const float ks = turned ? kv4_scale(most) : 1.f;
    wave_exchange();
    to.ksc[lane] = pc.sc.x;
    to.ks[lane] = most == 255u ? __uint_as_float(0x7fc00000u) : ks;
    to.none[lane] = pc.in ? 0u : ~0u;
#pragma unroll
    for (int g = 0; g < 4; ++g) to.vs[g][lane] = pc.in ? kv4_scale((pc.sc.y >> (8 * g)) & 255u) : 0.f;
    wave_exchange();
  };
  PairPlaces &wp = s.places.win[wv], *fp = s.places.far[wv];
  auto place_far = [&](PairPlaces& to, int pair) {   // this pair and the next one
    const int t = far_row(pair);
    bool in = t < f1;
    int j = t;
    if (t >= n_sink) {
      in = in && unit >= 0 && unit <= (sr.n - 1) >> a.sel_shift;   // (an index from elsewhere must not leave the cache)
      j = in ? (unit << a.sel_shift) + ((t - n_sink) & ((1 << a.sel_shift) - 1)) : 0;
      in = in && j >= sr.sink_end && j < sr.win_start;
    } else {
      in = in && t < sr.sink_end;
    }
    return place(to, j, in);
  };
  auto place_win = [&](int pair) {
    const int j = w0 + pair * kPair + lane;
    return place(wp, j, lane < kPair && j < w1);
  };

  // A wave takes its pairs of the window, then those of the far rows, two of which are in flight at a time: a pair's keys and
  // values are requested when those of the pair two before it have been used.  What does not depend on other loads comes first.
  const int far_n = far_end - far_first;
  const bool has_win = win_first < n_win;
  WaveState st;
  PairRows pa, pc;
  Place far_place;
  st.m = kNone;
  st.l = 0.f;
#pragma unroll
  for (int t = 0; t < 8; ++t) st.o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  const uint8_t* rows = a.cache.rows;
  if (has_win) {
    float x[32];
    load_elems<16>((const T*)a.q + q_at + lrow * 16, x);
    load_elems<16>((const T*)a.q + q_at + kD / 2 + lrow * 16, x + 16);
    Place win_place = place_win(win_first);
    if (far_n > 0) far_place = place_far(fp[0], far_first);
    get_scales(win_place);
    if (far_n > 0) get_scales(far_place);
    load_turned_pair(rows, wp.row, col, lrow, pc);
    if (far_n > 0) load_pair(rows, fp[0].row, col, lrow, pa);
    f16x8 qw[4];
    to_logits(x);
    const float ww = query_terms<NH == 8 ? 8 : 4>(x, C::q_term(col), active, qw);
    if (far_n > 0) put_scales(fp[0], far_place, false);
#pragma unroll 1
    for (int pair = win_first; pair < n_win; pair += kWaves) {
      put_scales(wp, win_place, true);
      f32x4 dot[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int delta = min(max(sr.n - 1 - (w0 + pair * kPair + t * 16 + col), 0), a.window - 1);
        float cs[16], sn[16];
        load_elems<16>(a.cos_win + (size_t)delta * (kD / 2) + lrow * 16, cs);
        load_elems<16>(a.sin_win + (size_t)delta * (kD / 2) + lrow * 16, sn);
        const uint32_t sc = wp.ksc[t * 16 + col];
        uint32_t most = 0;
#pragma unroll
        for (int g = 0; g < 4; ++g) most = max(most, (sc >> (8 * g)) & 255u);
        const int down = 127 - (int)most;
        const uint32_t lower = (sc >> (8 * (lrow >> 1))) & 255u, upper = (sc >> (16 + 8 * (lrow >> 1))) & 255u;
        const f32x4 acc = turned_dot(pc.k[t], kv4_scale((uint32_t)max((int)lower + down, 0)),
                                     kv4_scale((uint32_t)max((int)upper + down, 0)), cs, sn, qw);
#pragma unroll
        for (int i = 0; i < 4; ++i) dot[t][i] = C::sum(acc[i]) * ww;
      }
      float w[8];
      pair_weights(dot, wp, 0, lrow, st, w);
      absorb_values<NH>(w, wp, 0, col, lrow, pc, st);
      if (pair + kWaves < n_win) {
        win_place = place_win(pair + kWaves);
        get_scales(win_place);
        load_turned_pair(rows, wp.row, col, lrow, pc);
      }
    }
    if (far_n > 1) load_pair(rows, fp[0].row + kPair, col, lrow, pc);
  }
  if (far_n > 0) {
    FarQuery<NH> fq;
    float x[32];
    load_elems<32>(a.q_rot + q_at + lrow * 32, x);
    if (!has_win) {
      far_place = place_far(fp[0], far_first);
      get_scales(far_place);
      load_pair(rows, fp[0].row, col, lrow, pa);
      if (far_n > 1) load_pair(rows, fp[0].row + kPair, col, lrow, pc);
      put_scales(fp[0], far_place, false);
    }
    if (far_n > 2) unit = unit_of(far_row(far_first + 2));
    to_logits(x);
    fq.set(x, C::q_term(col), active);
    auto use = [&](const PairRows& p, const PairPlaces& pl, int first) {
      f32x4 dot[2];
#pragma unroll
      for (int t = 0; t < 2; ++t)
        dot[t] = fq.dot(p.k[t], kv4_scale(((const uint8_t*)(pl.ksc + first + t * 16 + col))[lrow]));
      float w[8];
      pair_weights(dot, pl, first, lrow, st, w);
      absorb_values<NH>(w, pl, first, col, lrow, p, st);
    };
    int buf = 0;
#pragma unroll 1
    for (int i = 0; i < far_n; i += 2) {
      const PairPlaces& pl = fp[buf];
      PairPlaces& next = fp[buf ^ 1];
      const bool more = i + 2 < far_n;
      if (more) {
        far_place = place_far(next, far_first + i + 2);
        get_scales(far_place);
        if (i + 4 < far_n) unit = unit_of(far_row(far_first + i + 4));
      }
      use(pa, pl, 0);
      if (more) load_pair(rows, next.row, col, lrow, pa);
      if (i + 1 < far_n) use(pc, pl, kPair);
      if (i + 3 < far_n) load_pair(rows, next.row + kPair, col, lrow, pc);
      if (more) put_scales(next, far_place, false);
      buf ^= 1;
    }
  }
  __syncthreads();   // (the places are written again, with the outputs)

  // The terms of a weight are added up, each tile's from the columns of its own group, and the waves merged.
  const float l_all = rows_sum(st.l);
#pragma unroll
  for (int t = 0; t < 8; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float o = NH == 1 ? head_sum<4>(st.o[t][i]) : st.o[t][i];
      if (NH == 1 ? col == t / 2 : C::group(col) == (NH == 8 ? t / 4 : t / 2))
        s.o[wv][hd][32 * (t / 2) + 2 * (4 * lrow + i) + t % 2] = o;
    }
  if (lane < NH) {
    s_m[wv][lane] = st.m;
    s_l[wv][lane] = l_all;
  }
  __syncthreads();
  for (int i = tid; i < nh * kD; i += kThreads) {
    const int g = i / kD, d = i % kD;
    float m = s_m[0][g], l = 0.f, o = 0.f;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) m = fmaxf(m, s_m[w][g]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = power(s_m[w][g] - m);
      l += s_l[w][g] * f;
      o += s.o[w][g][d] * f;
    }
    if (a.parts == 1) {
      store_elem((T*)a.out + (size_t)(head + g) * kD + d, l == 0.f ? 0.f : o / l);
    } else {
      float* to = a.partial + ((size_t)(head + g) * a.parts + part) * (kD + 2);
      to[d] = o;
      if (d == 0) {
        to[kD] = m;
        to[kD + 1] = l;
      }
    }
  }
}

}  // namespace

Kv4Plan make_kv4_plan(const a2ats_dims& d, long sel_rows, int window, bool shared) {
  Kv4Plan p;
  const long problems = (long)d.batch * (shared ? d.n_kv_heads : d.n_q_heads);
  const long rows = std::min<long>(sel_rows, d.ctx_len) + std::min(window, d.ctx_len);
  long parts = 1;
  if (problems <= 64) parts = rows < 350 ? 1 : std::min(std::min(problems > 0 ? 256 / problems : 1, rows / 72), 12l);
  else if (problems <= 128) parts = rows >= 1600 ? 4 : (rows >= 800 ? 2 : 1);
  else if (problems < 512) parts = rows >= 1600 ? 2 : 1;
  p.parts = (int)parts;
  p.bytes = parts > 1 ? (size_t)d.batch * d.n_q_heads * parts * (kD + 2) * sizeof(float) : 0;
  return p;
}

template <typename T>
static void launch_heads(const Attn4Args& a, long workgroups, hipStream_t stream) {
  const dim3 grid((unsigned)workgroups), block(kThreads);
  if (!a.shared || a.group == 1) hipLaunchKernelGGL((attn_kv4_kernel<T, 1>), grid, block, 0, stream, a);
  else if (a.group <= 4) hipLaunchKernelGGL((attn_kv4_kernel<T, 4>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((attn_kv4_kernel<T, 8>), grid, block, 0, stream, a);
}

hipError_t launch_sparse_attn_kv4(const a2ats_dims& d, const Kv4Cache& m, int kv_dtype, const void* q, const float* q_rot,
                                  const int32_t* sel_idx, const int32_t* sel_count, int n_sel, int sel_shift, bool shared, int window,
                                  int n_sink, const float* cos_win, const float* sin_win, const int32_t* seq_lens, void* out,
                                  void* ws, hipStream_t stream) {
  if (d.batch == 0) return hipSuccess;
  const Kv4Plan p = make_kv4_plan(d, (long)n_sel << sel_shift, window, shared);
  Attn4Args a;
  a.cache = m;
  a.q = q;
  a.q_rot = q_rot;
  a.sel_idx = sel_idx;
  a.sel_count = sel_count;
  a.cos_win = cos_win;
  a.sin_win = sin_win;
  a.seq_lens = seq_lens;
  a.partial = (float*)ws;
  a.out = out;
  a.ctx_len = d.ctx_len;
  a.n_sel = n_sel;
  a.sel_shift = sel_shift;
  a.window = window;
  a.n_sink = n_sink;
  a.group = d.n_q_heads / d.n_kv_heads;
  a.shared = shared;
  a.parts = p.parts;
  const long far = ((long)n_sel << sel_shift) + std::min(n_sink, d.ctx_len), win = std::min(window, d.ctx_len);
  a.far_share = (int)((far + p.parts - 1) / p.parts);
  a.win_share = (int)((win + p.parts - 1) / p.parts);
  a.problems = d.batch * d.n_kv_heads;
  const long workgroups = (long)a.problems * p.parts * (shared ? 1 : a.group);
  if (kv_dtype == A2ATS_BF16) launch_heads<uint16_t>(a, workgroups, stream);
  else launch_heads<float>(a, workgroups, stream);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || p.parts == 1 ? e : launch_attn_merge(kv_dtype, (const float*)ws, out, d.batch * d.n_q_heads, p.parts, stream);
}

}  // namespace a2ats
