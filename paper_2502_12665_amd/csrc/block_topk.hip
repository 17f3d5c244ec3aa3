// Selection of blocks: every block of a cache has an upper bound of its tokens' logits, and the top-K blocks of each
// query head (or of each KV head) are selected.
//
// Under WRoPE all tokens outside the window see the query at one offset, q~ = q R_b, so a bound over pre-RoPE keys holds:
//     q~ . k_j  <=  s = sum_d max(q~_d lo_d, q~_d hi_d)                  (lo, hi: the block's bounds per dimension)
//               =  sum_d max(q~_d, 0) hi_d + min(q~_d, 0) lo_d           (two products of matrices)
//               =  1/2 sum_d q~_d (lo_d + hi_d) + |q~_d| (hi_d - lo_d) . (two products per dimension without a choice)
// Shared selection: the sum over the G heads of a KV head has the same forms with the heads' sums, so it costs one head.
// Scores are defined as float64 sums, rounded once to float32.
//
// The scores are a stream over the bounds, 2 * 128 * e bytes per block and KV head, read once for all G heads; in float64 the
// arithmetic takes longer than the stream (4 x 8 KV heads x 8192 blocks, 4 heads each: 39 us against 27).  So bfloat16 bounds are
// scored on the matrix cores, by the first form: they are operands as they stand, and the 16 columns of a tile are the heads'
// queries in four bfloat16 terms each (their 24 bits and more).  Such a score s~ is off by at most
//     e = 2^-12 |q~|_1 max |bound| :   1024 products are exact and summed in float32, each sum off by 2^-23 of at most
//                                      |q~|_1 max |bound| (1 + 2^-6), however it is ordered, rounded or truncated
// and decides all but a band.  With one digit of a radix select the K-th largest s~ is known to lie in a bin [l, h] of values;
// then the K-th largest s is at least l - e and at most h + e, blocks with s~ > h + 2 e are selected and those with s~ < l - 2 e
// are not.  The others, a handful, get their float64 scores, and are ranked by these (equal scores: the lower block first).
// float32 bounds are scored in float64 right away (e = 0).  A band of more than kBandMost blocks (many equal scores, or bounds
// that are not finite) has all blocks of the head scored in float64 and a select over all digits.
//
// Two launches: the scores, and a workgroup a head that selects from them.  Measured, 4 x 8 KV heads of 8192 blocks, 4 heads
// each: scores 27.7 us = 4.85 TB/s of 134 MB (the rate of a large copy), selection 11 (a chain of a dozen phases of 0.5 to 2 us:
// range, one digit, band, its exact scores, ranks, output).  float32 bounds, scores: 4 x 8 KV heads of 4096 blocks, 4 heads each,
// 34.5 us = 3.9 TB/s of 134 MB; 8 x 4 of 2048, one selection for 7 heads 17.3 = 3.9 TB/s, 7 heads 20.4, 4 x 8 of 2048 with 8 heads
// 21.6 = 3.1 TB/s (from 7 heads on two waves a SIMD, 180 and 202 registers); selections 5 to 7.
// Selecting in the last of a head's score workgroups, one launch for both, was slower: its phases do not overlap the stream of
// the others by as much as they then cost.
#include <algorithm>

#include "internal.hpp"
#include "kv_blocks.hpp"

namespace a2ats {
namespace {

constexpr int kScoreThreads = 256;
constexpr int kPickBins = 2048;
constexpr int kBandMost = 1024;
constexpr int kD = kRowBytes;

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, 0xf, 0xf, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, 0xf, 0xf, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// Sum over the 16 lanes of a DPP row, in every lane.
template <typename F>
__device__ __forceinline__ F row16_sum(F v) {
  v += dpp<0xB1>(v);    // quad_perm [1,0,3,2]
  v += dpp<0x4E>(v);    // quad_perm [2,3,0,1]
  v += dpp<0x141>(v);   // row_half_mirror
  v += dpp<0x140>(v);   // row_mirror
  return v;
}

// A float's order as that of unsigned numbers.
__device__ __forceinline__ uint32_t order_key(float f) {
  const uint32_t u = __float_as_uint(f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
// A score as it is written: one zero, and what is not a number counts as infinite.
__device__ __forceinline__ float score_of(double sum) {
  const float f = (float)sum + 0.f;
  return f != f ? INFINITY : f;
}

struct TopkArgs {
  BlockCache cache;
  const void* q;
  const float* cos_b;
  const float* sin_b;
  float* q_rot;
  float* scores;        // [head][total_blocks]
  uint32_t* largest;    // [sequence, KV head][chunk]: of the magnitudes of a chunk's bounds, a float's bits
  const int32_t* seq_lens;
  int32_t* block_idx;
  int32_t* block_count;
  float* block_score;
  int32_t* token_idx;
  int32_t* token_count;
  int32_t total_blocks, chunks, problems, ctx_len, window, n_sink, top_blocks, heads, group, shared;
};

// Blocks of a sequence with n candidates that each of its workgroups scores: tiles of 16, shared out among as many as there are for
// the longest sequence.
__device__ __forceinline__ int chunk_blocks(int n, int chunks) { return ((n + chunks - 1) / chunks + 15) & ~15; }

// The rotated elements of eight dimensions of a head and, with them, those of the other half: q R_b in float64, rounded once.
template <typename T>
__device__ __forceinline__ void rotate8(const T* row, int t, const float* cos_b, const float* sin_b, float (&lower)[8], float (&upper)[8]) {
  float a[8], b[8], cs[8], sn[8];
  load8(row + t, a);
  load8(row + kD / 2 + t, b);
  load8(cos_b + t, cs);
  load8(sin_b + t, sn);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    lower[e] = (float)((double)a[e] * cs[e] - (double)b[e] * sn[e]);
    upper[e] = (float)((double)b[e] * cs[e] + (double)a[e] * sn[e]);
  }
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  *(float4*)p = make_float4(x[0], x[1], x[2], x[3]);
  *(float4*)(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}

// ------------------------------------------------------------------------------------------
// float64 scores
// ------------------------------------------------------------------------------------------

// NH heads' queries for 8 dimensions of each of 16 lanes.
template <int NH, bool SUMS>
struct ExactQuery {
  double q[NH][8], mag[SUMS ? NH : 1][8];   // SUMS: of several heads, and of their magnitudes
  __device__ __forceinline__ void add(int h, bool first, const float (&r)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      q[h][e] = (first ? 0.0 : q[h][e]) + (double)r[e];
      if constexpr (SUMS) mag[h][e] = (first ? 0.0 : mag[h][e]) + (double)fabsf(r[e]);
    }
  }
  __device__ __forceinline__ void scores(const float (&lo)[8], const float (&hi)[8], float (&f)[NH]) const {
    double s[NH];
#pragma unroll
    for (int g = 0; g < NH; ++g) s[g] = 0.0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const double l = lo[e], h = hi[e], mid = l + h, half = h - l;
#pragma unroll
      for (int g = 0; g < NH; ++g) {
        s[g] = __builtin_fma(q[g][e], mid, s[g]);
        s[g] = __builtin_fma(SUMS ? mag[SUMS ? g : 0][e] : __builtin_fabs(q[g][e]), half, s[g]);
      }
    }
#pragma unroll
    for (int g = 0; g < NH; ++g) f[g] = score_of(row16_sum(s[g]) * 0.5);
  }
};

// float32 bounds.  G: query heads of a KV head.
template <int G, bool SHARED>
__global__ __launch_bounds__(kScoreThreads) void score_blocks_f64_kernel(TopkArgs a) {
  constexpr int NH = SHARED ? 1 : G;
  constexpr int U = 2, GROUPS = kScoreThreads / 16;   // blocks of a group of 16 lanes whose bounds are requested together
  int prob, part;
  xcd_map(blockIdx.x, a.chunks, a.problems, prob, part);
  const int b = prob / a.cache.n_kv_heads, kv = prob % a.cache.n_kv_heads;
  const int lane = threadIdx.x & 63, d0 = (lane & 15) * 8, group = threadIdx.x >> 4;
  const SeqRange sr = seq_range(a.ctx_len, a.seq_lens, b, a.window, a.n_sink, 0);
  int first, last;
  candidate_blocks(sr, a.cache.shift, first, last);
  ExactQuery<NH, SHARED> eq;
#pragma unroll
  for (int g = 0; g < G; ++g) {
    float lower[8], upper[8];
    rotate8((const float*)a.q + ((size_t)prob * G + g) * kD, d0 & (kD / 2 - 1), a.cos_b, a.sin_b, lower, upper);
    float r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = d0 < kD / 2 ? lower[e] : upper[e];
    if (part == 0 && threadIdx.x < 16) store8(a.q_rot + ((size_t)prob * G + g) * kD + d0, r);
    eq.add(SHARED ? 0 : g, !SHARED || g == 0, r);
  }
  const int chunk = chunk_blocks(last - first, a.chunks), begin = first + part * chunk, end = min(last, begin + chunk);
  const float* bounds = (const float*)a.cache.bounds;
  for (int c0 = begin + group; c0 - (group & 3) < end; c0 += U * GROUPS) {
    float lo[U][8], hi[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float* p = bounds + block_at(a.cache, b, kv, min(c0 + u * GROUPS, end - 1)) * 2 * kD + d0;
      load8(p, lo[u]);
      load8(p + kD, hi[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float f[NH];
      eq.scores(lo[u], hi[u], f);
      const int c = c0 + u * GROUPS;
#pragma unroll
      for (int g = 0; g < NH; ++g)
        if ((lane & 15) == 0 && c < end) a.scores[((size_t)prob * NH + g) * a.total_blocks + c] = f[g];
    }
  }
}

// ------------------------------------------------------------------------------------------
// Scores on the matrix cores (bfloat16 bounds)
// ------------------------------------------------------------------------------------------

// The i-th of four bfloat16 terms of x, by truncation, in the upper half: x is their sum.
__device__ __forceinline__ uint32_t term_bits(float x, uint32_t cut1, uint32_t cut2, uint32_t cut3) {
  x -= __uint_as_float(__float_as_uint(x) & cut1);
  x -= __uint_as_float(__float_as_uint(x) & cut2);
  x -= __uint_as_float(__float_as_uint(x) & cut3);
  return __float_as_uint(x);
}

// Queries as the second operand: a column is a head (column % GP) and a term (column / GP; GP = 8: two sets of two terms).
// Dimensions of step s of lane row r: 8 (4 s + r) + 0 .. 7.
template <int GP>
struct MatrixQuery {
  static constexpr int SETS = GP / 4;
  struct Shared {
    uint4 op[4][SETS][2][64];   // [step][set][max(q, 0), min(q, 0)][lane]
  };
  bf16x8 hi[SETS][4], lo[SETS][4];
  __device__ __forceinline__ void load(const Shared& sh) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 0; k < SETS; ++k)
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        hi[k][s] = __builtin_bit_cast(bf16x8, sh.op[s][k][0][lane]);
        lo[k][s] = __builtin_bit_cast(bf16x8, sh.op[s][k][1][lane]);
      }
  }
  // Rows 4 * lane row + i of 16 blocks (row `column` of which is in w: lower bounds, then upper ones), in every column of a head.
  __device__ __forceinline__ f32x4 scores(const uint4 (&w)[8]) const {
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < SETS; ++k)
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w[s]), lo[k][s], acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w[4 + s]), hi[k][s], acc, 0, 0, 0);
      }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (GP == 4) acc[i] += dpp<0x124>(acc[i]);   // row_ror:4
      acc[i] += dpp<0x128>(acc[i]);                // row_ror:8
    }
    return acc;
  }
};

typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;
__device__ __forceinline__ uint32_t max_magnitudes(uint32_t m, uint32_t w) {
  const u16x2 x = __builtin_bit_cast(u16x2, w & 0x7fff7fffu), y = __builtin_bit_cast(u16x2, m);
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(x, y));
}

__device__ __forceinline__ void load_bounds16(const uint16_t* row, int lrow, uint4 (&w)[8]) {
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    w[s] = *(const uint4*)(row + 8 * (4 * s + lrow));
    w[4 + s] = *(const uint4*)(row + kD + 8 * (4 * s + lrow));
  }
}

// Step s of the queries of `heads` heads from head0 on (of which the column's is column % GP), or of the sum of all of them
// (`sum`), by one wave.
template <int GP>
__device__ __forceinline__ void make_query_step(const TopkArgs& a, int s, size_t head0, int heads, bool sum, bool write,
                                                typename MatrixQuery<GP>::Shared& sh) {
  const int lane = threadIdx.x & 63, col = lane & 15, lrow = lane >> 4;
  const bool active = sum ? col % GP == 0 : col % GP < heads;
  const int n = sum ? heads : 1, t = 8 * (4 * (s & 1) + lrow), half = s >> 1;
  float cs[8], sn[8], pos[8], neg[8];
  load8(a.cos_b + t, cs);
  load8(a.sin_b + t, sn);
#pragma unroll
  for (int e = 0; e < 8; ++e) pos[e] = neg[e] = 0.f;
  constexpr int AHEAD = 4;   // heads whose loads are requested together
  for (int g0 = 0; g0 < n; g0 += AHEAD) {
    uint4 own_raw[AHEAD], other_raw[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int h = sum ? min(g0 + k, n - 1) : min(col % GP, heads - 1);
      if (k == 0 || sum) {
        const uint16_t* row = (const uint16_t*)a.q + (head0 + h) * kD + t;
        own_raw[k] = *(const uint4*)(row + half * (kD / 2));
        other_raw[k] = *(const uint4*)(row + (half ^ 1) * (kD / 2));
      }
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (g0 + k >= n) continue;
      const int h = sum ? g0 + k : min(col % GP, heads - 1);
      float own[8], other[8], r[8];
      widen8(own_raw[k], own);
      widen8(other_raw[k], other);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double x = (double)own[e] * cs[e], y = (double)other[e] * sn[e];
        r[e] = (float)(half ? x + y : x - y);
        pos[e] += active ? fmaxf(r[e], 0.f) : 0.f;
        neg[e] += active ? fminf(r[e], 0.f) : 0.f;
      }
      if (write && (sum ? col == 0 : col < heads)) store8(a.q_rot + (head0 + h) * kD + half * (kD / 2) + t, r);
    }
  }
#pragma unroll
  for (int k = 0; k < MatrixQuery<GP>::SETS; ++k) {
    const int term = GP == 4 ? col / 4 : 2 * k + col / 8;
    const uint32_t c1 = term >= 1 ? 0xffff0000u : 0u, c2 = term >= 2 ? 0xffff0000u : 0u, c3 = term >= 3 ? 0xffff0000u : 0u;
    uint32_t p[4], m[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      p[e] = __builtin_amdgcn_perm(term_bits(pos[2 * e + 1], c1, c2, c3), term_bits(pos[2 * e], c1, c2, c3), 0x07060302u);
      m[e] = __builtin_amdgcn_perm(term_bits(neg[2 * e + 1], c1, c2, c3), term_bits(neg[2 * e], c1, c2, c3), 0x07060302u);
    }
    sh.op[s][k][0][lane] = make_uint4(p[0], p[1], p[2], p[3]);
    sh.op[s][k][1][lane] = make_uint4(m[0], m[1], m[2], m[3]);
  }
}

template <int GP>
__global__ __launch_bounds__(kScoreThreads) void score_blocks_kernel(TopkArgs a) {
  constexpr int NW = kScoreThreads / 64;
  static_assert(NW == 4, "a wave for each step of the queries");
  __shared__ uint32_t s_big[NW];
  __shared__ typename MatrixQuery<GP>::Shared s_query;
  int prob, part;
  xcd_map(blockIdx.x, a.chunks, a.problems, prob, part);
  const int b = prob / a.cache.n_kv_heads, kv = prob % a.cache.n_kv_heads, nh = a.shared ? 1 : a.group;
  const int lane = threadIdx.x & 63, col = lane & 15, lrow = lane >> 4;
  const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const SeqRange sr = seq_range(a.ctx_len, a.seq_lens, b, a.window, a.n_sink, 0);
  int first, last;
  candidate_blocks(sr, a.cache.shift, first, last);
  const int chunk = chunk_blocks(last - first, a.chunks), c0 = first + part * chunk, end = min(last, c0 + chunk);
  if (c0 >= end && part > 0) return;   // (uniform; the first part writes the rotated queries)
  const uint16_t* bounds = (const uint16_t*)a.cache.bounds;
  // Two tiles of 16 blocks are in flight.
  uint4 wa[8], wb[8];
  auto load = [&](int tile, uint4 (&w)[8]) {
    const int c = min(c0 + tile * 16 + col, end - 1);
    load_bounds16(bounds + block_at(a.cache, b, kv, c) * 2 * kD, lrow, w);
  };
  const int tiles = c0 < end ? (end - c0 + 15) / 16 : 0;
  if (wv < tiles) load(wv, wa);
  if (wv + NW < tiles) load(wv + NW, wb);
  make_query_step<GP>(a, wv, (size_t)prob * a.group, a.group, a.shared != 0, part == 0, s_query);
  __syncthreads();
  MatrixQuery<GP> mq;
  mq.load(s_query);
  uint32_t big = 0u;
  auto use = [&](int tile, const uint4 (&w)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      big = max_magnitudes(big, w[i].x);
      big = max_magnitudes(big, w[i].y);
      big = max_magnitudes(big, w[i].z);
      big = max_magnitudes(big, w[i].w);
    }
    const f32x4 sc = mq.scores(w);
    if (col < nh) {
      float* out = a.scores + ((size_t)prob * nh + col) * a.total_blocks;
      const int c = c0 + tile * 16 + 4 * lrow;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (c + i < end) out[c + i] = sc[i];
    }
  };
#pragma unroll 1
  for (int tile = wv; tile < tiles; tile += 2 * NW) {
    use(tile, wa);
    if (tile + 2 * NW < tiles) load(tile + 2 * NW, wa);
    if (tile + NW < tiles) use(tile + NW, wb);
    if (tile + 3 * NW < tiles) load(tile + 3 * NW, wb);
  }
  big = wave_max_to_last_lane(max(big & 0xffffu, big >> 16));
  if (lane == 63) s_big[wv] = big;
  __syncthreads();
  if (threadIdx.x == 0) {
    uint32_t m = s_big[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) m = max(m, s_big[w]);
    a.largest[(size_t)prob * a.chunks + part] = m << 16;
  }
}

// ------------------------------------------------------------------------------------------
// The selection of a head
// ------------------------------------------------------------------------------------------

// MATRIX: the scores are those of the matrix cores.  PER: scores of a thread, in registers; 0: they are read again in every
// pass.
template <typename T, bool MATRIX, int NT, int PER>
__global__ __launch_bounds__(NT) void pick_blocks_kernel(TopkArgs a) {
  constexpr int NW = NT / 64, KEEP = PER > 0 ? PER : 1;
  __shared__ uint32_t s_hist[kPickBins], s_a[NW], s_b[NW], s_res[2], s_lo, s_hi, s_band, s_big;
  __shared__ uint32_t s_band_key[kBandMost];
  __shared__ uint16_t s_band_at[kBandMost];
  __shared__ double2 s_query[MATRIX ? kD : 1];   // of several heads: the sums of their queries and of the magnitudes
  extern __shared__ __align__(8) uint32_t s_dyn[];   // a bit for each block that is taken out of the band; then the selection
  // (on the XCD where the head's scores have been written)
  const int of = a.shared ? 1 : a.group;
  int prob, head_of;
  xcd_map(blockIdx.x, of, a.problems, prob, head_of);
  const int bh = prob * of + head_of, b = bh / a.heads, tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int shift = a.cache.shift, kv = a.shared ? bh % a.heads : bh % a.heads / a.group;
  const int n_sum = a.shared ? a.group : 1;                                   // query heads of the score
  const size_t q_first = a.shared ? (size_t)bh * a.group : (size_t)bh;        // the first of them
  // Thread t has the blocks t, t + NT, ..: their scores are requested before it is known which of them are candidates.
  float raw[KEEP];
#pragma unroll
  for (int i = 0; i < PER; ++i) raw[i] = a.scores[(size_t)bh * a.total_blocks + min(tid + i * NT, max(a.total_blocks - 1, 0))];
  // ... and so are the queries (of one head: this lane's eight dimensions; of several: a dimension of each for a thread) and the
  // chunks' magnitudes (two chunks a thread hold all of them).
  const int d0 = (lane & 15) * 8, group = tid >> 4;
  const uint32_t* largest = a.largest + ((size_t)b * a.cache.n_kv_heads + kv) * a.chunks;
  float q_raw[8];
  uint32_t large_raw[2] = {0u, 0u};
  if constexpr (MATRIX) {
    if (n_sum == 1) {
      load8(a.q_rot + q_first * kD + d0, q_raw);
    } else if (tid < kD) {
#pragma unroll
      for (int g = 0; g < 8; ++g) q_raw[g] = a.q_rot[(q_first + min(g, n_sum - 1)) * kD + tid];
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) large_raw[i] = largest[min(tid + i * NT, a.chunks - 1)];
  }
  const SeqRange sr = seq_range(a.ctx_len, a.seq_lens, b, a.window, a.n_sink, 0);
  int first, last;
  candidate_blocks(sr, shift, first, last);
  const int n = last - first, kk = min(a.top_blocks, n);
  const int words = (a.total_blocks + NT - 1) / NT * (NT / 32);   // whole rounds
  uint32_t* s_taken = s_dyn;
  int32_t* s_sel = (int32_t*)(s_dyn + words);
  int32_t* idx = a.block_idx + (size_t)bh * a.top_blocks;
  float* score = a.block_score ? a.block_score + (size_t)bh * a.top_blocks : nullptr;
  const T* bounds = (const T*)a.cache.bounds;
  float* src = a.scores + (size_t)bh * a.total_blocks;

  if (tid == 0) {
    a.block_count[bh] = kk;
    s_lo = ~0u;
    s_hi = 0u;
    s_band = 0u;
    s_big = 0u;
  }
  for (int i = tid; i < kPickBins; i += NT) s_hist[i] = 0u;
  for (int i = tid; i < words; i += NT) s_taken[i] = 0u;
  for (int i = kk + tid; i < a.top_blocks; i += NT) {
    idx[i] = -1;
    if (score) score[i] = 0.f;
  }
  if constexpr (MATRIX) {
    __syncthreads();
    const int chunk = chunk_blocks(n, a.chunks);
    uint32_t big = 0u;   // (as bits: what is not a number is the largest)
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (tid + i * NT < a.chunks && (tid + i * NT) * chunk < n) big = max(big, large_raw[i]);
    big = wave_max_to_last_lane(big);
    if (lane == 63 && wv < (a.chunks + 63) / 64) atomicMax(&s_big, big);
    if (n_sum > 1 && tid < kD) {
      double q = 0.0, mag = 0.0;
#pragma unroll
      for (int g = 0; g < 8; ++g) {
        q += g < n_sum ? (double)q_raw[g] : 0.0;
        mag += g < n_sum ? (double)fabsf(q_raw[g]) : 0.0;
      }
      s_query[tid] = make_double2(q, mag);
    }
  }
  __syncthreads();

  // This group of 16 lanes' part of the head's query, for float64 scores.
  ExactQuery<1, true> eq;
  if constexpr (MATRIX) {
    if (n_sum == 1) {
      eq.add(0, true, q_raw);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        eq.q[0][e] = s_query[d0 + e].x;
        eq.mag[0][e] = s_query[d0 + e].y;
      }
    }
  }
  auto exact_score = [&](int c) {   // of block c, by 16 lanes
    float lo[8], hi[8], f[1];
    const T* p = bounds + block_at(a.cache, b, kv, c) * 2 * kD + d0;
    load8(p, lo);
    load8(p + kD, hi);
    eq.scores(lo, hi, f);
    return f[0];
  };

  // Keys in the order of the scores; 0 (which no score has) for what is not a candidate.
  uint32_t key[KEEP];
  auto key_of = [&](int c, float x) { return c >= first && c < last ? order_key(x != x ? INFINITY : x) : 0u; };
#pragma unroll
  for (int i = 0; i < PER; ++i) key[i] = key_of(tid + i * NT, raw[i]);
  const int round_first = first / NT, round_end = n > 0 ? (last - 1) / NT + 1 : round_first;
  // f(round, block, key) for all rounds of NT blocks with candidates, by whole waves
  auto for_rounds = [&](auto f) {
    if constexpr (PER > 0) {
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (i >= round_first && i < round_end) f(i, tid + i * NT, key[i]);
    } else {
      for (int i = round_first; i < round_end; ++i) {
        const int c = tid + i * NT;
        f(i, c, key_of(c, src[min(c, max(a.total_blocks - 1, 0))]));
      }
    }
  };
  // The selection is a bit for each block, two words for a wave's blocks of a round.
  auto put_mask = [&](int i, uint64_t mask) {
    if (lane == 0) *(uint2*)&s_taken[(i * NW + wv) * 2] = make_uint2((uint32_t)mask, (uint32_t)(mask >> 32));
  };
  auto find_range = [&]() {
    uint32_t k_min = ~0u, k_max = 0u;
    for_rounds([&](int, int, uint32_t k) {
      k_min = min(k_min, k - 1u);   // (no candidate: the largest number)
      k_max = max(k_max, k);
    });
    k_max = wave_max_to_last_lane(k_max);
    k_min = ~wave_max_to_last_lane(~k_min);
    if (lane == 63) {
      atomicMax(&s_hi, k_max);
      atomicMin(&s_lo, k_min);
    }
    __syncthreads();
  };

  if (kk > 0 && kk < n) {   // (uniform)
    uint32_t above, low_key;   // selected: keys above `above`, and some of those from low_key on
    find_range();
    // One digit: the bin of the kk-th largest.
    const uint32_t base = s_lo + 1u, range = s_hi - base;
    const int bits = 32 - (range ? __clz(range) : 32), cut = max(bits - 11, 0);
    for_rounds([&](int, int, uint32_t k) {
      if (k) atomicAdd(&s_hist[(k - base) >> cut], 1u);
    });
    // (|q|_1 for the error: the first wave's four groups have the same sums)
    float e2 = 0.f;
    if constexpr (MATRIX) {
      double l1 = 0.0;
#pragma unroll
      for (int e = 0; e < 8; ++e) l1 += eq.mag[0][e];
      l1 = row16_sum(l1);
      const float big = __uint_as_float(s_big);
      e2 = 2.f * ((float)l1 * 0x1.02p-12f + 0x1p-100f) * big;
    }
    __syncthreads();
    block_find_rank_desc<NT, kPickBins>([&](int bin) { return s_hist[bin]; }, (uint32_t)kk, s_a, s_res);
    const uint32_t bin_low = base + (s_res[0] << cut), bin_high = min(bin_low + ((1u << cut) - 1u), s_hi);
    low_key = bin_low;
    above = bin_high;
    bool all = false;   // the band is all of the head, or too large
    if constexpr (MATRIX) {
      const float lv = key_value(bin_low) - e2, hv = key_value(bin_high) + e2;
      all = !(e2 < 0x1p110f);   // (2^17 below what float32 holds, so that no sum has overflowed)
      low_key = order_key(lv);
      above = order_key(hv);
    }
    if (!all) {
      uint32_t more = 0;
      for_rounds([&](int i, int c, uint32_t k) {
        const uint64_t mask = __builtin_amdgcn_ballot_w64(k > above);
        put_mask(i, mask);
        more += (uint32_t)__popcll(mask);
        if (k >= low_key && k <= above) {
          const uint32_t at = atomicAdd(&s_band, 1u);
          if (at < kBandMost) {
            s_band_key[at] = k;
            s_band_at[at] = (uint16_t)c;
          }
        }
      });
      // how many of the band are still to be taken
      if (lane == 0) s_b[wv] = more;
      __syncthreads();
      uint32_t surely = 0;
#pragma unroll
      for (int w = 0; w < NW; ++w) surely += s_b[w];
      const uint32_t band = s_band, left = (uint32_t)kk - surely;
      if (band <= kBandMost) {
        if constexpr (MATRIX) {
          for (uint32_t i = group; i - (group & 3) < band; i += NT / 16) {   // (waves stay together)
            const uint32_t j = min(i, band - 1);
            const float f = exact_score(s_band_at[j]);
            if ((lane & 15) == 0 && i < band) s_band_key[i] = order_key(f);
          }
          __syncthreads();
        }
        // Rank by counting; the lower block goes first among equal scores.
        for (uint32_t i = tid >> 3; i - ((uint32_t)lane >> 3) < band; i += NT / 8) {   // eight lanes a block
          const uint32_t k = s_band_key[min(i, band - 1)], c = s_band_at[min(i, band - 1)];
          int32_t better = 0;
          for (uint32_t j = lane & 7; j < band; j += 8) better += s_band_key[j] > k || (s_band_key[j] == k && s_band_at[j] < c);
          better = group8_sum(better);
          if ((lane & 7) == 0 && i < band && (uint32_t)better < left) atomicOr(&s_taken[c >> 5], 1u << (c & 31));
        }
      } else {
        all = true;
      }
    }
    if (all) {   // (uniform)
      if constexpr (MATRIX) {
        for (int c = first + group; c - (group & 3) < last; c += NT / 16) {
          const float f = exact_score(min(c, last - 1));
          if ((lane & 15) == 0 && c < last) src[c] = f;
        }
        __threadfence_block();
      }
      __syncthreads();
      if (tid == 0) {
        s_lo = ~0u;
        s_hi = 0u;
      }
      __syncthreads();
      if constexpr (MATRIX) {
#pragma unroll
        for (int i = 0; i < PER; ++i) key[i] = key_of(tid + i * NT, src[min(tid + i * NT, max(a.total_blocks - 1, 0))]);
      }
      find_range();
      // The kk-th largest key by digits of 11 bits from the highest bit in which the keys differ; `equal` of those that have it
      // are taken, the lowest blocks first.
      const uint32_t base2 = s_lo + 1u, range2 = s_hi - base2;
      uint32_t left = (uint32_t)kk, prefix = 0;
      int now = 32 - (range2 ? __clz(range2) : 32);
      while (now > 0) {
        const int width = min(now, 11), over = now;
        now -= width;
        for (int i = tid; i < kPickBins; i += NT) s_hist[i] = 0u;
        __syncthreads();
        for_rounds([&](int, int, uint32_t k) {
          const uint32_t rel = k - base2;
          if (k && (over >= 32 || rel >> over == prefix)) atomicAdd(&s_hist[(rel >> now) & ((1u << width) - 1u)], 1u);
        });
        __syncthreads();
        block_find_rank_desc<NT, kPickBins>([&](int bin) { return s_hist[bin]; }, left, s_a, s_res);
        prefix = (prefix << width) | s_res[0];
        left -= s_res[1];
        __syncthreads();
      }
      above = base2 + prefix;
      // Equal keys in the order of the blocks: round by round.
      uint32_t before = 0;
      for_rounds([&](int i, int, uint32_t k) {
        const uint64_t mask = __builtin_amdgcn_ballot_w64(k == above);
        __syncthreads();
        if (lane == 0) s_b[wv] = (uint32_t)__popcll(mask);
        __syncthreads();
        uint32_t at = before;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
          at += w < wv ? s_b[w] : 0u;
          before += s_b[w];
        }
        const bool take = (mask >> lane & 1u) && at + (uint32_t)lanes_below(mask) < left;
        put_mask(i, __builtin_amdgcn_ballot_w64(k > above || take));
      });
    }
  } else if (kk > 0) {
    for_rounds([&](int i, int, uint32_t k) { put_mask(i, __builtin_amdgcn_ballot_w64(k != 0u)); });
  }
  __syncthreads();
  // The selection in ascending order: how many there are before each wave's blocks of a round.
  uint32_t* s_before = s_hist;   // [round][wave], at most 1024
  if (wv == 0) {
    uint32_t run = 0;
    for (int i = round_first * NW; i < round_end * NW; i += 64) {
      const int w = min(i + lane, round_end * NW - 1);
      const uint2 m = *(const uint2*)&s_taken[w * 2];
      const uint32_t v = i + lane < round_end * NW ? (uint32_t)(__popc(m.x) + __popc(m.y)) : 0u;
      const uint32_t inc = wave_inclusive_scan(v);
      if (i + lane < round_end * NW) s_before[i + lane] = run + inc - v;
      run += (uint32_t)__builtin_amdgcn_readlane((int)inc, 63);
    }
  }
  __syncthreads();
  for (int i = round_first; i < round_end; ++i) {
    const uint2 m = *(const uint2*)&s_taken[(i * NW + wv) * 2];
    const uint64_t mask = (uint64_t)m.y << 32 | m.x;
    if (mask >> lane & 1u) {
      const uint32_t at = s_before[i * NW + wv] + (uint32_t)lanes_below(mask);
      const int c = tid + i * NT;
      idx[at] = c;
      s_sel[at] = c;
      if (!MATRIX && score) score[at] = src[c];
    }
  }
  __syncthreads();
  if constexpr (MATRIX) {
    if (score) {
      for (int i = group; i - (group & 3) < kk; i += NT / 16) {
        const float f = exact_score(s_sel[min(i, kk - 1)]);
        if ((lane & 15) == 0 && i < kk) score[i] = f;
      }
    }
  }
  if (a.token_count == nullptr) return;   // (uniform)
  // The tokens: whole blocks but for the first and the last candidate block, of which the candidates are taken.
  const int blk = 1 << shift, slots = a.top_blocks << shift;
  const int skip = kk > 0 && s_sel[0] == first ? sr.sink_end - (first << shift) : 0;
  const int over = kk > 0 && s_sel[kk - 1] == last - 1 ? (last << shift) - sr.win_start : 0;
  const int count = (kk << shift) - skip - over;
  if (tid == 0) a.token_count[bh] = count;
  int32_t* tokens = a.token_idx + (size_t)bh * slots;
  for (int i = tid; i < slots; i += NT) {
    const int t = i + skip;
    tokens[i] = i < count ? (s_sel[t >> shift] << shift) + (t & (blk - 1)) : -1;
  }
}

}  // namespace

BlockTopkPlan make_block_topk_plan(const a2ats_dims& d, int block, bool shared) {
  BlockTopkPlan p;
  const long problems = (long)d.batch * d.n_kv_heads;
  p.total_blocks = (int)(((long)d.ctx_len + block - 1) / block);
  // Two workgroups a CU, each with 64 blocks at least (a tile for every wave).
  long chunks = problems > 0 ? (512 + problems - 1) / problems : 1;
  chunks = std::max(1l, std::min(chunks, (long)p.total_blocks / 64));
  p.chunks = (int)chunks;
  const size_t scores = (size_t)d.batch * (shared ? d.n_kv_heads : d.n_q_heads) * p.total_blocks * sizeof(float);
  p.off_largest = (scores + 255) / 256 * 256;
  p.bytes = p.off_largest + (size_t)problems * p.chunks * sizeof(uint32_t);
  return p;
}

template <int G>
static void launch_f64(const TopkArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)(a.problems * a.chunks)), block(kScoreThreads);
  if (a.shared) hipLaunchKernelGGL((score_blocks_f64_kernel<G, true>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((score_blocks_f64_kernel<G, false>), grid, block, 0, stream, a);
}

template <typename T, bool MATRIX, int NT, int PER>
static hipError_t launch_pick_as(const TopkArgs& a, int batch, hipStream_t stream) {
  const size_t lds = ((size_t)(a.total_blocks + NT - 1) / NT * (NT / 32) + a.top_blocks) * sizeof(uint32_t);
  hipLaunchKernelGGL((pick_blocks_kernel<T, MATRIX, NT, PER>), dim3((unsigned)(batch * a.heads)), dim3(NT), lds, stream, a);
  return hipGetLastError();
}
// Threads of a head's workgroup: it is a chain of short phases, each of which a small workgroup ends sooner and leaves room for
// others on its CU.  Both launches of a call (bfloat16, 4 heads a KV head, an eighth of the blocks selected, at most 128), us, with the
// threads taken and with 1024:
//   blocks   256: 128 heads  9.8 (11.1), 896 heads 20.0 (36.6)       2048: 128 heads 17.5 (17.9), 896 heads  68.3 (79.7)
//   blocks  1024: 128 heads 13.4 (13.8), 512 heads 22.1 (27.6),      4096: 128 heads 23.3 (23.0), 896 heads 121.4 (132.9)
//                 896 heads 33.8 with 256 threads, 38.8 with 512, 49.6
//   blocks  8192: 128 heads 35.1 with 1024, 37.3 with 512; 512 heads 131.5 and 126.3
template <typename T, bool MATRIX>
static hipError_t launch_pick(const TopkArgs& a, int batch, hipStream_t stream) {
  const long heads = (long)batch * a.heads;
  if (a.total_blocks <= 256) return launch_pick_as<T, MATRIX, 256, 1>(a, batch, stream);
  if (a.total_blocks <= 1024)
    return heads > 512 ? launch_pick_as<T, MATRIX, 256, 4>(a, batch, stream) : launch_pick_as<T, MATRIX, 512, 2>(a, batch, stream);
  if (a.total_blocks <= 2048) return launch_pick_as<T, MATRIX, 512, 4>(a, batch, stream);
  if (a.total_blocks <= 4096) return launch_pick_as<T, MATRIX, 512, 8>(a, batch, stream);
  if (a.total_blocks <= 8192)
    return heads > 256 ? launch_pick_as<T, MATRIX, 512, 16>(a, batch, stream) : launch_pick_as<T, MATRIX, 1024, 8>(a, batch, stream);
  return launch_pick_as<T, MATRIX, 1024, 0>(a, batch, stream);
}

hipError_t launch_block_topk(const a2ats_dims& d, const BlockCache& m, int kv_dtype, const void* q, const float* cos_b,
                             const float* sin_b, float* q_rot, bool shared, int top_blocks, int window, int n_sink,
                             const int32_t* seq_lens, int32_t* block_idx, int32_t* block_count, float* block_score,
                             int32_t* token_idx, int32_t* token_count, void* ws, hipStream_t stream) {
  if (d.batch == 0) return hipSuccess;
  const BlockTopkPlan p = make_block_topk_plan(d, 1 << m.shift, shared);
  TopkArgs a;
  a.cache = m;
  a.q = q;
  a.cos_b = cos_b;
  a.sin_b = sin_b;
  a.q_rot = q_rot;
  a.scores = (float*)ws;
  a.largest = (uint32_t*)((char*)ws + p.off_largest);
  a.seq_lens = seq_lens;
  a.block_idx = block_idx;
  a.block_count = block_count;
  a.block_score = block_score;
  a.token_idx = token_idx;
  a.token_count = token_count;
  a.total_blocks = p.total_blocks;
  a.chunks = p.chunks;
  a.problems = d.batch * d.n_kv_heads;
  a.ctx_len = d.ctx_len;
  a.window = window;
  a.n_sink = n_sink;
  a.top_blocks = top_blocks;
  a.group = d.n_q_heads / d.n_kv_heads;
  a.shared = shared;
  a.heads = shared ? d.n_kv_heads : d.n_q_heads;
  const dim3 grid((unsigned)(a.problems * a.chunks)), block(kScoreThreads);
  if (kv_dtype == A2ATS_BF16) {
    if (shared || a.group <= 4) hipLaunchKernelGGL((score_blocks_kernel<4>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((score_blocks_kernel<8>), grid, block, 0, stream, a);
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : launch_pick<uint16_t, true>(a, d.batch, stream);
  }
  switch (a.group) {
    case 1: launch_f64<1>(a, stream); break;
    case 2: launch_f64<2>(a, stream); break;
    case 3: launch_f64<3>(a, stream); break;
    case 4: launch_f64<4>(a, stream); break;
    case 5: launch_f64<5>(a, stream); break;
    case 6: launch_f64<6>(a, stream); break;
    case 7: launch_f64<7>(a, stream); break;
    default: launch_f64<8>(a, stream); break;
  }
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : launch_pick<float, false>(a, d.batch, stream);
}

}  // namespace a2ats
