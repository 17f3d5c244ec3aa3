// Attention of one query token over sinks U selected tokens (or blocks) U window, from a cache held in 4 bits with a scale for
// each 32 dimensions of a token's key and value:
//     logit_j = (q~ . k_j) / sqrt(128)  (window rows: q R_delta for q~),  out = sum softmax(logit)_j v_j.
//
// A row is 128 bytes of codes and 8 of scales, 4 flop per byte and head: a gather, of whole lines of memory.  Both products are on the
// matrix cores, also for one head, with the 16 rows or columns of a tile used for the precision of the float32 operand:
//   - queries (A, 16 rows) times keys (B, 16 rows of the cache).  A lane has 32 dimensions of a key, which are a group: 16 bytes of codes
//     and one scale, with which they become bfloat16 (exact: two bits of significand) as they are converted.  The query is three
//     bfloat16 terms by truncation, all of its 24 bits, each a row of the tile (eight heads have two rows each, and a second product for the
//     third term); its rows are ordered so that a lane has all terms of its heads' logits of one key.  With one head a lane has
//     one logit: with the keys as the first operand it had 16, and the softmax of 32 x 28 heads of 2176 rows took 4 us more.
//     The products of 4-bit and 8-bit operands with scales of their own would take the codes as they are, but their sums are not those of
//     float32 (off by up to 2^-13 of the sum of magnitudes, measured).
//   - values (A, 16 dimensions x 32 rows) times weights (B).  A row has four scales, which multiply the weight: a column takes the scale of
//     one group, and of a tile's products only the columns of its own group count.  One head: 16 columns are four groups times
//     the three bfloat16 terms of a weight; up to four heads: head times group, and a product for each term; eight: head times
//     half the groups, and two sets of weights.  Weights go to their columns through LDS.  So do the values, which come from memory 16
//     bytes a lane; a lane then takes four bytes of each of its 8 rows, two dimensions of each group.  Two rows' words are put
//     together by halves of bytes, and each byte is then a pair of rows of one dimension, which converts to two bfloat16.
// Window rows are turned back by their distance, (q R_delta) . k = q . (k R_-delta): one head on the vector ALU, in float32; heads that share
// a selection by products of queries with turned keys, relative to the row's largest scale, that go in as two float16 terms (2^-23 of an
// element, 2^-26 of the row's largest).  (For one head those products took as long with a window, 71.1 against 71.9 us, and 62.5 against
// 60.1 without one, by their registers.)
// The statistics, all sums and the output are float32.  Logits are kept times log2 e, so that a weight is one exponential.
//
// What bounds it: the gather.  Bare loads of the 1.95 million rows of 32 x 28 heads that attend 2176 rows each take 54 us by whole lines (4.9
// TB/s of the 265 MB that they are); this kernel 60 us without a window and 72 us with 128 rows of window, whose angles, 64 KB for a
// head, pass through the first-level cache.  A row's key and value are requested one after the other, as they are one line: by
// tiles of keys and then tiles of values it took 67 us.  With few heads it is the latency of a unit (64 rows a wave, of which the next is
// in flight): 4 x 32 heads of 2304 rows 16.5 us and 3 us of a pass (4.1 to 4.7 by itself) to join their parts, 7.6 us at the rate of a copy.  Workgroups of 8 and 16 waves
// instead of 4 take as long or longer at nearly all sizes (128 problems, 2304 rows 18.5 and 20.7 us against 19.4; 896 problems 60.8 with
// four), two units in flight for each wave too.
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

constexpr int kUnit = 64;   // rows that a wave takes at a time: four tiles of 16, a row for each lane

// Heads that attend the same rows, padded to NH: what rows and columns of the tiles stand for.
//   first product: row m of the queries is (head, term); its results are rows 4 * lane row + i, so that the terms of a head are in one lane:
//     NH 1: term m % 4, in each lane row alike; 4: head m / 4, term m % 4; 8: head m / 2, term m % 2 (the third one is a product of its own)
//   second product: column c of the weights is
//     NH 1: term c / 4 and group c % 4; 4: head c / 4 and group c % 4; 8: head c / 2 and half c % 2 of the groups, of which there are two sets
template <int NH>
struct Layout {
  static constexpr int kOwn = NH == 1 ? 1 : (NH == 4 ? 4 : 8);   // logits of a lane in a unit
  static constexpr int kHeads = NH == 8 ? 2 : 1;                 // heads that a lane has logits of
  static constexpr int kColumns = NH == 1 ? 13 : 48;             // of weights in LDS (one head: 12 and one of zeros; else 3 terms of 16)
  static __device__ __forceinline__ int q_head(int m) { return NH == 1 ? 0 : m * NH / 16; }
  static __device__ __forceinline__ int q_term(int m) { return NH == 8 ? m & 1 : m & 3; }
  static __device__ __forceinline__ int col_head(int c) { return NH == 1 ? 0 : c * NH / 16; }
};

// A wave's working memory in LDS.
template <int NH>
struct alignas(16) WaveMemory {
  uint16_t weights[Layout<NH>::kColumns][kUnit];   // bfloat16
  i32x4 values[kUnit][4];                          // a unit's values as they come from memory
  uint32_t row[2][kUnit];                          // where a unit's rows are, and the next one's
  uint32_t ksc[kUnit];                             // scale bytes of the keys
  uint32_t vsc[NH == 1 ? 1 : kUnit];               // ... of the values (one head: a lane has its own row's)
  float ks[NH == 1 ? 1 : kUnit];                   // 1, or NaN for a key that is; -1 without a row
  int32_t win_exp[NH == 1 ? 1 : kUnit];            // window rows: the exponent of the largest of the key's scales
  float alpha[8];
};

// The queries as the first operand, of a workgroup: made once, and read again for each unit (16 registers that four waves a SIMD do
// not have).
template <int NH>
struct alignas(16) Queries {
  uint4 far[4][64];
  uint4 third[NH == 8 ? 4 : 1][64];
  uint4 win[NH == 1 ? 1 : 4][64];
  int32_t win_exp[64];
  float win_query[kD];   // one head
};

// The upper half of a float: bfloat16 by truncation, and what is left.
__device__ __forceinline__ float lower_part(float x) { return x - __uint_as_float(__float_as_uint(x) & 0xffff0000u); }
__device__ __forceinline__ uint16_t upper_half(float x) { return (uint16_t)(__float_as_uint(x) >> 16); }

__device__ __forceinline__ bf16x8 pack8(const float (&x)[8]) {
  return __builtin_bit_cast(bf16x8, make_uint4(upper_halves(x[0], x[1]), upper_halves(x[2], x[3]), upper_halves(x[4], x[5]),
                                               upper_halves(x[6], x[7])));
}

// Slice i of the far queries: elements 32 * lane row + 8 i + 0 .. 7 of the head of the lane's row, as bfloat16 terms by truncation.
template <int NH>
__device__ __forceinline__ void put_far_queries(const float* from, int i, bool active, int lane, Queries<NH>& to) {
  const int term = Layout<NH>::q_term(lane & 15);
  const uint32_t cut1 = term >= 1 ? 0xffff0000u : 0u, cut2 = term >= 2 ? 0xffff0000u : 0u, keep = active && term < 3 ? ~0u : 0u;
  float y[8], z[8];
  load8(from + 8 * i, y);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    y[e] *= kLogit;
    z[e] = __uint_as_float(__float_as_uint(lower_part(lower_part(y[e]))) & (term == 0 ? keep : 0u));
    y[e] -= __uint_as_float(__float_as_uint(y[e]) & cut1);
    if (NH != 8) y[e] -= __uint_as_float(__float_as_uint(y[e]) & cut2);
    y[e] = __uint_as_float(__float_as_uint(y[e]) & keep);
  }
  to.far[i][lane] = __builtin_bit_cast(uint4, pack8(y));
  if (NH == 8) to.third[NH == 8 ? i : 0][lane] = __builtin_bit_cast(uint4, pack8(z));
}

// The first of the eight elements of either half that a lane row has of a turned row; the next eight are 16 on.
__device__ __forceinline__ int turned_from(int lrow) { return 32 * (lrow & 1) + 8 * (lrow >> 1); }

// One head's window query times log2 e / sqrt(128).
template <typename T>
__device__ __forceinline__ void put_win_query(const T* from, int lane, float (&to)[kD]) {
  if (lane < kD / 8) {
    float x[8];
    load8(from + lane * 8, x);
#pragma unroll
    for (int e = 0; e < 8; ++e) to[lane * 8 + e] = x[e] * kLogit;
  }
}

// Slice i of the window's queries (0, 1: eight elements of the lower half each, 2, 3: of the upper one), as float16 terms of x 2^(8 - e),
// |x| < 2^e for all of the head: x = 2^(e - 8) (t0 + t1 + t2) but for 2^-33 of 2^e (half the least float16) and, for eight heads with their
// two terms, 2^-23 of x.  e >= -97: what is below 2^-30 of that is below the least normal number.
template <typename T, int NH>
__device__ __forceinline__ void put_win_queries(const T* from, int i, bool active, int lane, Queries<NH>& to) {
  const int term = Layout<NH>::q_term(lane & 15), at = turned_from(lane >> 4);
  float big = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float x[8];
    load8(from + at + 16 * (j & 1) + kD / 2 * (j >> 1), x);
#pragma unroll
    for (int e = 0; e < 8; ++e) big = fmaxf(big, fabsf(x[e]));   // (a NaN stays one in its own terms)
  }
  big = rows_max(big) * kLogit;
  const int e0 = max((int)(__float_as_uint(big) >> 23) - 126, -97);
  // (an infinite element makes all of its head's terms NaN)
  const float down = big < INFINITY ? ldexpf(active && term < 3 ? 1.f : 0.f, 8 - e0) : __uint_as_float(0x7fc00000u);
  const float less1 = term >= 1 ? 1.f : 0.f, less2 = term >= 2 ? 1.f : 0.f;
  float y[8];
  load8(from + at + 16 * (i & 1) + kD / 2 * (i >> 1), y);
  f16x8 q;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float z = y[e] * kLogit * down;
    z -= less1 * (float)(_Float16)z;
    if (NH != 8) z -= less2 * (float)(_Float16)z;
    q[e] = (_Float16)z;
  }
  to.win[i][lane] = __builtin_bit_cast(uint4, q);
  if (i == 0) to.win_exp[lane] = e0 - 8;
}

// Byte `at` of row r.  PAGED: of a pool, which may have more than 2^32 bytes; otherwise of a sequence and KV head, at most 2^20 rows.
template <bool PAGED>
__device__ __forceinline__ const uint8_t* row_byte(const uint8_t* rows, uint32_t r, int at) {
  if (PAGED) return rows + (size_t)r * kKv4RowBytes + at;
  return rows + (r * kKv4RowBytes + (uint32_t)at);
}
// A unit's keys and values as they come from memory: 16 bytes of either of row `column` of each tile, by lane row; a row's two requests, which are
// for the same line, one after the other.  (Values by words of the rows that a lane needs would be four times as many requests: bare
// loads of the rows of 32 x 28 heads take 65 us so, 56 like this, 54 by whole lines.)
template <bool PAGED>
__device__ __forceinline__ void load_rows(const uint8_t* cache, const uint32_t* rows, int lane, i32x4 (&k)[4], i32x4 (&v)[4]) {
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const uint8_t* p = row_byte<PAGED>(cache, rows[t * 16 + (lane & 15)], (lane >> 4) * 16);
    k[t] = *(const i32x4*)p;
    v[t] = *(const i32x4*)(p + kKv4Half);
  }
}

// Products of the queries with a unit's far keys: row `column` of tile t in dot[t].
template <int NH>
__device__ __forceinline__ void far_dots(const i32x4 (&k)[4], const uint8_t* scales, int lane, const Queries<NH>& queries, f32x4 (&dot)[4]) {
  float scale[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    scale[t] = kv4_scale(scales[(t * 16 + (lane & 15)) * 4 + (lane >> 4)]);
    dot[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bf16x8 q = __builtin_bit_cast(bf16x8, queries.far[i][lane]);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      uint32_t w[4];
#define A2ATS_PAIR(e) w[e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((uint32_t)k[t][i], scale[t], e));
      A2ATS_PAIR(0) A2ATS_PAIR(1) A2ATS_PAIR(2) A2ATS_PAIR(3)
#undef A2ATS_PAIR
      const bf16x8 k8 = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
      dot[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q, k8, dot[t], 0, 0, 0);
      if (NH == 8)
        dot[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, queries.third[NH == 8 ? i : 0][lane]), k8, dot[t], 0, 0, 0);
    }
  }
}

// The same of a tile's window keys, turned back by the row's angles (cs, sn: its rows of the tables).  The other half of an element is two
// lane rows on, so these lane rows exchange words: the first two have words 0 and 2 of both, the others 1 and 3.  sc: the row's scale bytes;
// the products are relative to the largest.
template <int NH>
__device__ __forceinline__ f32x4 turned_dot(const i32x4& k, uint32_t sc, const float* cs_row, const float* sn_row, int lane,
                                            const Queries<NH>& queries) {
  const int lrow = lane >> 4;
  uint32_t most = 0;
#pragma unroll
  for (int g = 0; g < 4; ++g) most = max(most, (sc >> (8 * g)) & 255u);
  const int down = 127 - (int)most;
  const uint32_t lower_byte = (sc >> (8 * (lrow & 1))) & 255u, upper_byte = (sc >> (16 + 8 * (lrow & 1))) & 255u;
  const float s_lower = kv4_scale((uint32_t)max((int)lower_byte + down, 0)), s_upper = kv4_scale((uint32_t)max((int)upper_byte + down, 0));
  float cs[2][8], sn[2][8];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    load8(cs_row + turned_from(lrow) + 16 * i, cs[i]);
    load8(sn_row + turned_from(lrow) + 16 * i, sn[i]);
  }
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 2; ++i) {   // eight pairs of elements
    const auto words = __builtin_amdgcn_permlane32_swap((uint32_t)k[2 * i], (uint32_t)k[2 * i + 1], false, false);
    float lower[8], upper[8];
#define A2ATS_PAIR(e)                                                                          \
  {                                                                                            \
    const auto dl = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(words[0], s_lower, e);            \
    const auto du = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(words[1], s_upper, e);            \
    _Pragma("unroll") for (int j = 0; j < 2; ++j) {                                            \
      lower[2 * e + j] = dl[j] * cs[i][2 * e + j] + du[j] * sn[i][2 * e + j];                  \
      upper[2 * e + j] = du[j] * cs[i][2 * e + j] - dl[j] * sn[i][2 * e + j];                  \
    }                                                                                          \
  }
    A2ATS_PAIR(0) A2ATS_PAIR(1) A2ATS_PAIR(2) A2ATS_PAIR(3)
#undef A2ATS_PAIR
    auto terms = [&](const float (&x)[8], const uint4& query) {
      const f16x8 qt = __builtin_bit_cast(f16x8, query);
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f16x2 h = f16_pair(x[2 * j], x[2 * j + 1]);
        hi[j] = f16_bits(h);
        lo[j] = f16_bits(f16_pair(x[2 * j] - (float)h[0], x[2 * j + 1] - (float)h[1]));
      }
      acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(qt, __builtin_bit_cast(f16x8, make_uint4(hi[0], hi[1], hi[2], hi[3])), acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(qt, __builtin_bit_cast(f16x8, make_uint4(lo[0], lo[1], lo[2], lo[3])), acc, 0, 0, 0);
    };
    terms(lower, queries.win[i][lane]);
    terms(upper, queries.win[2 + i][lane]);
  }
  __builtin_amdgcn_sched_barrier(0);   // (several tiles at once would not fit the registers)
  return acc;
}

// One head: products of the query, turned by the row's angles, with a tile's window keys, on the vector ALU: of a pair of elements,
//   (q R) . k = (q_l cos - q_u sin) k_l + (q_l sin + q_u cos) k_u,
// six operations, where the terms of turned keys are twelve.  (The angles go to the query: products of elements that do not meet, as those of
// a pair's two halves in the last token's row, may be beyond float32.)  Angles of eight pairs:
struct Angles {
  float cs[8], sn[8];
  __device__ __forceinline__ void load(const float* cos_win, const float* sin_win, int delta, int lrow, int i) {
    load8(cos_win + (size_t)delta * (kD / 2) + turned_from(lrow) + 16 * i, cs);
    load8(sin_win + (size_t)delta * (kD / 2) + turned_from(lrow) + 16 * i, sn);
  }
};
// ... pairs i of the lane row's two eights (see turned_dot): what the lane adds.
__device__ __forceinline__ float turned_part(const i32x4& k, int i, float s_lower, float s_upper, const Angles& a, const float* query, int lrow) {
  const auto words = __builtin_amdgcn_permlane32_swap((uint32_t)k[2 * i], (uint32_t)k[2 * i + 1], false, false);
  float sum = 0.f;
#define A2ATS_PAIR(e)                                                                          \
  {                                                                                            \
    const auto kl = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(words[0], s_lower, e);            \
    const auto ku = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(words[1], s_upper, e);            \
    _Pragma("unroll") for (int j = 0; j < 2; ++j) {                                            \
      const int x = 2 * e + j;                                                                 \
      sum += (ql[x % 4] * a.cs[x] - qu[x % 4] * a.sn[x]) * kl[j] + (ql[x % 4] * a.sn[x] + qu[x % 4] * a.cs[x]) * ku[j]; \
    }                                                                                          \
  }
#define A2ATS_FOUR(at, first, second)                                                          \
  {                                                                                            \
    int from = turned_from(lrow) + 16 * i + at;                                                \
    asm volatile("" : "+v"(from));                                                             \
    const f32x4 ql = *(const f32x4*)(query + from), qu = *(const f32x4*)(query + kD / 2 + from); \
    A2ATS_PAIR(first) A2ATS_PAIR(second)                                                       \
    __builtin_amdgcn_sched_barrier(0);                                                         \
  }
  // (The query is read again for each tile, four numbers of either half at a time: more would not fit the registers.)
  A2ATS_FOUR(0, 0, 1)
  A2ATS_FOUR(4, 2, 3)
#undef A2ATS_FOUR
#undef A2ATS_PAIR
  return sum;
}

// The bits of a where the mask has ones, else those of b.
__device__ __forceinline__ uint32_t select_bits(uint32_t mask, uint32_t a, uint32_t b) { return (mask & a) | (~mask & b); }

// Rows of a unit in LDS.  A lane has elements e = 0 .. 7 of either half h as operands of the second product: one head, rows 32 h + 4 e + lane
// row; else rows 16 (e % 4) + 8 h + 2 lane row + e / 4, so that the four rows that a lane has weights of lie behind each other.  Values lie
// so that what the lanes of a wave read at a time is in one piece.
template <int NH>
__device__ __forceinline__ int value_slot(int tile, int col) { return tile * 16 + (NH == 1 ? col : (col & 1) << 3 | col >> 1); }
__device__ __forceinline__ int weight_at(int row) { return (row & 32) | (row & 3) << 3 | (row >> 2 & 7); }   // one head

// A half's values, of which a lane has a word (two dimensions of each group) of its eight rows, two rows' words together: byte g of even[i]
// has the first of the two dimensions of group g of the rows e = 2 i and 2 i + 1, of odd[i] the second; the lower half of a byte is the
// first row's.
template <int NH>
struct Values {
  uint32_t even[4], odd[4];
  __device__ __forceinline__ Values(const uint32_t* v, int h) {   // word `column` of slot `lane row`
    auto word = [&](int e) { return v[(NH == 1 ? 32 * h + 4 * e : 16 * (e & 3) + 8 * (e >> 2) + 4 * h) * 16]; };
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t a = word(2 * i), c = word(2 * i + 1);
      even[i] = select_bits(0x0f0f0f0fu, a, c << 4);
      odd[i] = select_bits(0x0f0f0f0fu, a >> 4, c);
    }
  }
};

// Their products with the weights (columns of LDS; one head: a term a column, else three terms), added to the outputs: o[t][i] is
// dimension 32 (t / 2) + 2 (4 * lane row + i) + t % 2, in the columns of group t / 2.  SET: eight heads, groups SET and 2 + SET.
template <int NH, int SET>
__device__ __forceinline__ void absorb(const Values<NH>& v, const uint16_t* weights, f32x4 (&o)[8]) {
  constexpr int kTerms = NH == 1 ? 1 : 3;
  bf16x8 b[kTerms];
#pragma unroll
  for (int term = 0; term < kTerms; ++term) b[term] = __builtin_bit_cast(bf16x8, *(const uint4*)(weights + term * 16 * kUnit));
#define A2ATS_TILE(t)                                                                                                                 \
  if (NH != 8 || (t) / 2 % 2 == SET) {                                                                                                \
    uint32_t w[4];                                                                                                                    \
    _Pragma("unroll") for (int i = 0; i < 4; ++i)                                                                                     \
        w[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((t) & 1 ? v.odd[i] : v.even[i], 1.f, (t) / 2)); \
    const bf16x8 vt = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));                                                 \
    _Pragma("unroll") for (int term = 0; term < kTerms; ++term)                                                                       \
        o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, b[term], o[t], 0, 0, 0);                                                   \
  }
  A2ATS_TILE(0) A2ATS_TILE(1) A2ATS_TILE(2) A2ATS_TILE(3) A2ATS_TILE(4) A2ATS_TILE(5) A2ATS_TILE(6) A2ATS_TILE(7)
#undef A2ATS_TILE
}

// Over the 16 lanes of a lane row, in each of them.
template <typename F>
__device__ __forceinline__ float over_columns(float v, F f) {
  v = f(v, dpp<0xB1>(v));    // quad_perm [1,0,3,2]
  v = f(v, dpp<0x4E>(v));    // quad_perm [2,3,0,1]
  v = f(v, dpp<0x124>(v));   // row_ror:4
  return f(v, dpp<0x128>(v));
}
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float sum_of(float a, float b) { return a + b; }

// NH: heads that attend the same rows, one, or the G of a KV head if the selection is shared, padded to 4 or 8.
template <typename T, int NH, bool PAGED>
__global__ __launch_bounds__(kWaves * 64, NH == 1 ? 4 : 2) void attn_kv4_kernel(Attn4Args a) {
  typedef Layout<NH> L;
  __shared__ __align__(16) union {
    struct {
      Queries<NH> queries;
      WaveMemory<NH> wave[kWaves];
    } in;
    float o[kWaves][NH][kD];
  } s;
  __shared__ float s_m[kWaves][NH], s_l[kWaves][NH];

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
  const size_t first_row = PAGED ? 0 : ((size_t)prob * (size_t)blocks.blocks_per_seq) << blocks.shift;
  const uint8_t *rows = a.cache.rows + first_row * kKv4RowBytes, *scales = a.cache.scales + first_row * kKv4ScaleBytes;

  // The part's share of the far rows (row t is sink t, then row t - n_sink of the selection) and of the window's is dealt out to the waves by
  // tiles, those of the window first.  It goes by what the call allows, not by the sequence: what has to be fetched first does not
  // wait for its length.
  const int n_sink = min(a.n_sink, a.ctx_len);
  const int win_tiles = (a.win_share + 16 * kWaves - 1) / (16 * kWaves), far_tiles = (a.far_share + 16 * kWaves - 1) / (16 * kWaves);
  const int f0 = part * a.far_share + (wv * far_tiles - win_tiles) * 16, w0 = part * a.win_share + wv * win_tiles * 16;
  auto unit_of = [&](int u, int lane) {   // (clamped: requested before it is known to count)
    return a.n_sel > 0 ? idx[min(max(f0 + u * kUnit + lane - n_sink, 0) >> a.sel_shift, a.n_sel - 1)] : 0;
  };
  int index = unit_of(0, lane);
  const SeqRange sr = seq_range(a.ctx_len, a.seq_lens, b, a.window, a.n_sink, 0);
  const int cnt = min(max(a.sel_count[sel], 0), a.n_sel);
  const int f1 = min(min((part + 1) * a.far_share, f0 + (win_tiles + far_tiles) * 16), n_sink + (cnt << a.sel_shift));
  const int w1 = min(sr.n, sr.win_start + (part + 1) * a.win_share);
  // Units with a row: of the window, or of far rows.
  const int win_units = min(max(w1 - sr.win_start - w0 + kUnit - 1, 0) / kUnit, (win_tiles + 3) / 4);
  const int units = sr.n > 0 ? max(win_units, (max(f1 - f0, 0) + kUnit - 1) / kUnit * (f1 > f0 + win_tiles * 16)) : 0;

  WaveMemory<NH>& wm = s.in.wave[wv];
  // Lane l places row l of a unit, and requests its scales.
  struct Place {
    uint2 sc;
    bool in;
  };
  auto place = [&](uint32_t* to, int u, int lane) {
    const int tile = 4 * u + (lane >> 4), t = f0 + u * kUnit + lane;
    bool in;
    int j = t;
    if (tile < win_tiles) {
      j = sr.win_start + w0 + u * kUnit + lane;
      in = j < w1;
    } else {
      in = t < f1 && u < units;
      if (t >= n_sink) {
        in = in && index >= 0 && index <= (sr.n - 1) >> a.sel_shift;   // (an index from elsewhere must not leave the cache)
        j = in ? (index << a.sel_shift) + ((t - n_sink) & ((1 << a.sel_shift) - 1)) : 0;
        in = in && j >= sr.sink_end && j < sr.win_start;
      } else {
        in = in && t < sr.sink_end;
      }
    }
    Place pc;
    pc.in = in;
    j = in ? j : 0;   // (a place without a row: the sequence's first one, which has been written and counts for nothing)
    uint32_t at = (uint32_t)j;
    if (PAGED) at = (uint32_t)((block_at(blocks, b, kv, j >> blocks.shift) << blocks.shift) + (size_t)(j & ((1 << blocks.shift) - 1)));
    wave_exchange();
    to[lane] = at;
    wave_exchange();
    pc.sc = *(const uint2*)(PAGED ? scales + (size_t)at * kKv4ScaleBytes : scales + at * (uint32_t)kKv4ScaleBytes);
    return pc;
  };

  // A wave has one unit in flight: the next one's rows are requested when a unit's keys have become products, and its values are in LDS.
  // Requests are made whether there is a next unit or not (then for the sequence's first row): the wait for what a unit needs would be one
  // for all requests if it were not known how many come after it.
  float m[L::kHeads], l[L::kHeads];   // running maximum of a head, and the sum of the lane's own weights
  f32x4 o[8];
  i32x4 k[4], v[4];
  Place at, next;
  if (units > 0) {
    at = place(wm.row[0], 0, lane);
    load_rows<PAGED>(rows, wm.row[0], lane, k, v);
    index = unit_of(1, lane);
  }
  {
    const size_t q_at = (size_t)(head + min(L::q_head(col), nh - 1)) * kD;
    const bool active = L::q_head(col) < nh;
    put_far_queries<NH>(a.q_rot + q_at + lrow * 32, wv, active, lane, s.in.queries);
    if (a.window > 0) {
      if constexpr (NH != 1) put_win_queries<T, NH>((const T*)a.q + q_at, wv, active, lane, s.in.queries);
      else if (wv == 0) put_win_query((const T*)a.q + q_at, lane, s.in.queries.win_query);
    }
  }
  if (NH == 1) wm.weights[NH == 1 ? 12 : 0][lane] = 0;
  __syncthreads();
#pragma unroll
  for (int h = 0; h < L::kHeads; ++h) {
    m[h] = kNone;
    l[h] = 0.f;
  }
#pragma unroll
  for (int t = 0; t < 8; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};

#pragma unroll 1
  for (int u = 0; u < units; ++u) {
    int lane = tid & 63;
    asm volatile("" : "+v"(lane));   // (else a dozen addresses are kept in registers, which there are not)
    const int col = lane & 15, lrow = lane >> 4;
    const uint16_t* my_weights = wm.weights[NH == 1 ? min(col, 12) : col] + lrow * 8;
    // The scales of this unit's rows, for the lanes that have them as keys, and the values, from where they are read again by rows.
    uint32_t most = 0;
#pragma unroll
    for (int g = 0; g < 4; ++g) most = max(most, (at.sc.x >> (8 * g)) & 255u);
    const float ks = most == 255u ? __uint_as_float(0x7fc00000u) : 1.f;
    wave_exchange();
    wm.ksc[lane] = at.sc.x;
    if (NH != 1) {
      wm.vsc[NH == 1 ? 0 : lane] = at.in ? at.sc.y : 0u;
      wm.ks[NH == 1 ? 0 : lane] = at.in ? ks : -1.f;
    }
    if (NH != 1 && 4 * u < win_tiles) wm.win_exp[NH == 1 ? 0 : lane] = (int)most - 127;
#pragma unroll
    for (int t = 0; t < 4; ++t) wm.values[value_slot<NH>(t, col)][lrow] = v[t];
    wave_exchange();
    uint32_t* next_rows = wm.row[(u & 1) ^ 1];
    next = place(next_rows, u + 1, lane);
    index = unit_of(u + 2, lane);

    f32x4 dot[4];
    far_dots<NH>(k, (const uint8_t*)wm.ksc, lane, s.in.queries, dot);
    float lg[4];   // one head
#pragma unroll
    for (int t = 0; t < 4; ++t) lg[t] = dot[t][0] + dot[t][1] + dot[t][2];
    if (4 * u < win_tiles) {
      __builtin_amdgcn_sched_barrier(0);
      auto distance = [&](int t) { return min(max(sr.n - 1 - (sr.win_start + w0 + u * kUnit + t * 16 + col), 0), a.window - 1); };
      if constexpr (NH == 1) {   // (the angles of the next eight pairs are requested before these are used)
        Angles x, y;
        x.load(a.cos_win, a.sin_win, distance(0), lrow, 0);
        const int tiles = min(win_tiles - 4 * u, 4);
#pragma unroll 1
        for (int t = 0; t < tiles; ++t) {
          const i32x4 kt = t < 2 ? (t == 0 ? k[0] : k[1]) : (t == 2 ? k[2] : k[3]);
          const uint32_t sc = wm.ksc[t * 16 + col];
          const float s_lower = kv4_scale((sc >> (8 * (lrow & 1))) & 255u), s_upper = kv4_scale((sc >> (16 + 8 * (lrow & 1))) & 255u);
          y.load(a.cos_win, a.sin_win, distance(t), lrow, 1);
          float sum = turned_part(kt, 0, s_lower, s_upper, x, s.in.queries.win_query, lrow);
          x.load(a.cos_win, a.sin_win, distance(t + 1), lrow, 0);
          sum += turned_part(kt, 1, s_lower, s_upper, y, s.in.queries.win_query, lrow);
          sum = rows_sum(sum);
#pragma unroll
          for (int i = 0; i < 4; ++i) lg[i] = t == i ? sum : lg[i];
        }
        // The angles requested last are used by nobody: here, else all units wait for what is requested at this place.
        __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
      } else {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          if (4 * u + t >= win_tiles) break;
          const int delta = distance(t);
          dot[t] = turned_dot<NH>(k[t], wm.ksc[t * 16 + col], a.cos_win + (size_t)delta * (kD / 2), a.sin_win + (size_t)delta * (kD / 2), lane,
                                  s.in.queries);
          // (The query's row 4 * lane row: the terms of a head have the same.  By the sum of both exponents: as factors, of up to 2^125 and
          // 2^120 or 2^-105, they would overflow ahead of the logit, also where this is 0.)
          const int ke = wm.win_exp[NH == 1 ? 0 : t * 16 + col];
          const int4 qe = *(const int4*)(s.in.queries.win_exp + 4 * lrow);
          dot[t] = f32x4{ldexpf(dot[t][0], qe.x + ke), ldexpf(dot[t][1], qe.y + ke), ldexpf(dot[t][2], qe.z + ke), ldexpf(dot[t][3], qe.w + ke)};
        }
      }
    }
    load_rows<PAGED>(rows, next_rows, lane, k, v);

    // Logits: one head, of the lane's own row; else of row `column` of each tile, of the lane row's heads.
    float p[L::kOwn];
    if constexpr (NH == 1) {
      const float x = (lrow & 2) ? ((lrow & 1) ? lg[3] : lg[2]) : ((lrow & 1) ? lg[1] : lg[0]);
      p[0] = at.in ? x * ks : -INFINITY;
    } else {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const float kt = wm.ks[NH == 1 ? 0 : t * 16 + col];
#pragma unroll
        for (int h = 0; h < L::kHeads; ++h) {
          const float x = NH == 8 ? dot[t][2 * h] + dot[t][2 * h + 1] : dot[t][0] + dot[t][1] + dot[t][2];
          p[t * L::kHeads + h] = kt < 0.f ? -INFINITY : x * kt;
        }
      }
    }
    float mn[L::kHeads];
    bool rise = false;
#pragma unroll
    for (int h = 0; h < L::kHeads; ++h) {
      float mx = p[h];
#pragma unroll
      for (int i = h + L::kHeads; i < L::kOwn; i += L::kHeads) mx = fmaxf(mx, p[i]);
      mx = over_columns(mx, larger);
      if (NH == 1) mx = rows_max(mx);
      mn[h] = fmaxf(m[h], mx);
      rise = rise || mn[h] > m[h];
    }
    if (__builtin_amdgcn_ballot_w64(rise)) {
      float alpha;
      if constexpr (NH == 1) {
        alpha = power(m[0] - mn[0]);
        l[0] *= alpha;
      } else {   // from the lane rows that have a head's logits to the columns that have its output
        wave_exchange();
#pragma unroll
        for (int h = 0; h < L::kHeads; ++h) {
          const float f = power(m[h] - mn[h]);
          l[h] *= f;
          if (col == 0) wm.alpha[lrow * L::kHeads + h] = f;
        }
        wave_exchange();
        alpha = wm.alpha[L::col_head(col)];
      }
#pragma unroll
      for (int t = 0; t < 8; ++t) o[t] *= alpha;
#pragma unroll
      for (int h = 0; h < L::kHeads; ++h) m[h] = mn[h];
    }
#pragma unroll
    for (int i = 0; i < L::kOwn; ++i) {
      p[i] = power(p[i] - mn[i % L::kHeads]);
      l[i % L::kHeads] += p[i];
    }

    // Weights times the scales of the groups, as three bfloat16 terms, into the columns of the second product.
    const uint32_t* words = (const uint32_t*)&wm.values[lrow][0] + col;
    if constexpr (NH == 1) {
      const uint32_t vsc = at.in ? at.sc.y : 0u;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        float x = p[0] * kv4_scale((vsc >> (8 * g)) & 255u);
#pragma unroll
        for (int term = 0; term < 3; ++term) {
          wm.weights[4 * term + g][weight_at(lane)] = upper_half(x);
          x = lower_part(x);
        }
      }
      wave_exchange();
      absorb<NH, 0>(Values<NH>(words, 0), my_weights, o);
      absorb<NH, 0>(Values<NH>(words, 1), my_weights + kUnit / 2, o);
    } else {
#pragma unroll
      for (int set = 0; set < (NH == 8 ? 2 : 1); ++set) {
        wave_exchange();
#pragma unroll
        for (int g = 0; g < (NH == 8 ? 2 : 4); ++g) {
          float sc[4];
#pragma unroll
          for (int t = 0; t < 4; ++t) sc[t] = kv4_scale((wm.vsc[NH == 1 ? 0 : t * 16 + col] >> (8 * (NH == 8 ? 2 * g + set : g))) & 255u);
#pragma unroll
          for (int h = 0; h < L::kHeads; ++h) {
            float x[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) x[t] = p[t * L::kHeads + h] * sc[t];
#pragma unroll
            for (int term = 0; term < 3; ++term) {
              *(uint2*)&wm.weights[16 * term + (NH == 8 ? 2 * (2 * lrow + h) + g : 4 * lrow + g)][4 * col] =
                  make_uint2(upper_halves(x[0], x[1]), upper_halves(x[2], x[3]));
#pragma unroll
              for (int t = 0; t < 4; ++t) x[t] = lower_part(x[t]);
            }
          }
        }
        wave_exchange();
        if (set == 0) {
          absorb<NH, 0>(Values<NH>(words, 0), my_weights, o);
          absorb<NH, 0>(Values<NH>(words, 1), my_weights + kUnit / 2, o);
        } else {
          absorb<NH, 1>(Values<NH>(words, 0), my_weights, o);
          absorb<NH, 1>(Values<NH>(words, 1), my_weights + kUnit / 2, o);
        }
      }
    }
    at = next;
  }
  __syncthreads();   // (the waves' memory is written again, with the outputs)

  // The terms of a weight are added up (one head), each tile's from the columns of its own group, and the waves merged.
#pragma unroll
  for (int t = 0; t < 8; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = NH == 1 ? head_sum<4>(o[t][i]) : o[t][i];
      const int g = t / 2;
      if (NH == 1 ? col == g : (NH == 4 ? (col & 3) == g : (col & 1) == g / 2))
        s.o[wv][L::col_head(col)][32 * g + 2 * (4 * lrow + i) + t % 2] = x;
    }
#pragma unroll
  for (int h = 0; h < L::kHeads; ++h) {
    float all = over_columns(l[h], sum_of);
    if (NH == 1) all = rows_sum(all);
    if (NH == 1 ? lane == 0 : col == 0) {
      s_m[wv][NH == 1 ? 0 : lrow * L::kHeads + h] = m[h];
      s_l[wv][NH == 1 ? 0 : lrow * L::kHeads + h] = all;
    }
  }
  __syncthreads();
  for (int i = tid; i < nh * kD; i += kThreads) {
    const int g = i / kD, d = i % kD;
    float mx = s_m[0][g], ls = 0.f, x = 0.f;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) mx = fmaxf(mx, s_m[w][g]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = power(s_m[w][g] - mx);
      ls += s_l[w][g] * f;
      x += s.o[w][g][d] * f;
    }
    if (a.parts == 1) {
      store_elem((T*)a.out + (size_t)(head + g) * kD + d, ls == 0.f ? 0.f : x / ls);
    } else {
      float* to = a.partial + ((size_t)(head + g) * a.parts + part) * (kD + 2);
      to[d] = x;
      if (d == 0) {
        to[kD] = mx;
        to[kD + 1] = ls;
      }
    }
  }
}

}  // namespace

// The most parts that a head's (KV head's) rows are shared out to, whatever their number: as many workgroups as CUs, or two parts.
static long most_parts(long problems) {
  if (problems <= 128) return problems > 0 ? std::min(256 / problems, 12l) : 1;
  return problems > 256 && (problems - 1) % 256 < 128 ? 2 : 1;
}

// Parts: a second launch that joins them, 3 us of a pass, against units of 64 rows that a wave has to take one after the other, 1.5 us each
// (2.6 for heads that share a selection) while there is a workgroup a CU at most.  So: the least parts that leave a wave the fewest units, with no
// more workgroups than CUs, where that saves two units.  (Units of selected rows and of the window: sinks are shared out with the selected rows but not
// counted, as they are few.)  Measured for 2 to 896 problems of 160 to 4160 rows with 1 to 16 parts (bfloat16, window
// 64), us with one part -> with the parts taken: 2 problems, 576 rows 10.1 -> 9.5 (3 parts), 2304 rows 18.1 -> 10.4 (12); 32 problems, 1152
// rows 12.9 -> 10.0 (6), 4160 rows 28.5 -> 13.0 (6); 128 problems, 2304 rows 19.3 -> 17.1 (2; four: 18.5); 256 problems, 2304 rows would be
// 20.2 -> 23.9; shared by four heads, 8 problems, 1152 rows 19.2 -> 12.4 (6), 128 problems, 1152 rows 20.4 -> 19.7 (2).
// More problems than CUs, of which half a round of CUs or less is left over: two parts make half a round of it, which pays for many rows, from 16 units a
// wave on (shared selections, of which fewer workgroups are resident: 24).  One part -> two, problems of 4160 rows: 264 44.0 -> 45.3, 288 42.0 ->
// 39.7, 376 46.9 -> 46.6, 384 42.1 -> 39.7, 520 74.3 -> 65.8, 640 62.0 -> 60.5, 784 95.1 -> 91.2, 896 85.1 -> 83.4, 1152 105 -> 107;
// of 15256 rows: 288 124 -> 104, 520 222 -> 189, 896 262 -> 239, 1152 331 -> 303.  More than half a round left over, 4160 rows: 392 47.5 -> 56.3, 656 73.4
// -> 76.3, 904 96 -> 102; 2304 rows: 384 28.3 -> 28.9, 896 53.1 -> 57.5.  Shared by four heads, 6064 rows: 264 74.5 -> 71.3, 520 124 -> 113, 640 133 -> 125, 896
// 168 -> 172, by eight 208 -> 203; 4160 rows, four heads: 384 58.0 -> 59.7, 520 94.6 -> 90.1, 896 126 -> 136.
Kv4Plan make_kv4_plan(const a2ats_dims& d, long sel_rows, int window, bool shared) {
  const long problems = (long)d.batch * (shared ? d.n_kv_heads : d.n_q_heads), most = most_parts(problems);
  const long far = std::min<long>(sel_rows, d.ctx_len), win = std::min(window, d.ctx_len);
  auto units = [&](long parts) {
    const long f = (far + parts - 1) / parts, w = (win + parts - 1) / parts;
    return ((f + 16 * kWaves - 1) / (16 * kWaves) + (w + 16 * kWaves - 1) / (16 * kWaves) + 3) / 4;
  };
  long parts = 1;
  if (problems > 128) {
    if (units(1) >= (shared && d.n_q_heads > d.n_kv_heads ? 24 : 16)) parts = most;
  } else {
    for (long p = 2; p <= most; ++p)
      if (units(p) < units(parts)) parts = p;
    if (units(1) - units(parts) < 2) parts = 1;
  }
  Kv4Plan p;
  p.parts = (int)parts;
  p.bytes = parts > 1 ? (size_t)d.batch * d.n_q_heads * parts * (kD + 2) * sizeof(float) : 0;
  return p;
}

// What every call with at most so many selected tokens and such a window needs.  (A plan of two parts or more has three units at least, which are more
// than 4 * kUnit rows.)
size_t kv4_ws_bytes(const a2ats_dims& d, long sel_rows, int window) {
  const long rows = std::min<long>(sel_rows, d.ctx_len) + std::min(window, d.ctx_len);
  size_t need = 0;
  for (int shared = 0; shared < 2; ++shared) {
    const long parts = most_parts((long)d.batch * (shared ? d.n_kv_heads : d.n_q_heads));
    if (parts > 1 && rows > 4 * kUnit) need = std::max(need, (size_t)d.batch * d.n_q_heads * parts * (kD + 2) * sizeof(float));
  }
  return need;
}

template <typename T, bool PAGED>
static void launch_heads(const Attn4Args& a, long workgroups, hipStream_t stream) {
  const dim3 grid((unsigned)workgroups), block(kThreads);
  if (!a.shared || a.group == 1) hipLaunchKernelGGL((attn_kv4_kernel<T, 1, PAGED>), grid, block, 0, stream, a);
  else if (a.group <= 4) hipLaunchKernelGGL((attn_kv4_kernel<T, 4, PAGED>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((attn_kv4_kernel<T, 8, PAGED>), grid, block, 0, stream, a);
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
  const bool paged = m.at.pages != nullptr;
  if (kv_dtype == A2ATS_BF16) {
    if (paged) launch_heads<uint16_t, true>(a, workgroups, stream);
    else launch_heads<uint16_t, false>(a, workgroups, stream);
  } else {
    if (paged) launch_heads<float, true>(a, workgroups, stream);
    else launch_heads<float, false>(a, workgroups, stream);
  }
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || p.parts == 1 ? e : launch_attn_merge(kv_dtype, (const float*)ws, out, d.batch * d.n_q_heads, p.parts, stream);
}

}  // namespace a2ats
