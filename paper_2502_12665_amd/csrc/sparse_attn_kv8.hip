// Attention of one query token over sinks U selected tokens (or blocks) U window, from a cache held in 8 bits with a
// scale for each block of tokens and KV head:
//     logit_j = (q~ . code_j) * k_scale / sqrt(128)  (window rows: q R_delta for q~),  out = sum softmax(logit)_j code_j v_scale.
// The scales are per row of a block, so they multiply the finished product and the weight, never the 128 elements.  Rows of
// the sequence's incomplete block are in the tail, in the type of q.
//
// A row is 128 bytes of keys and as many of values, 2 flop per byte and head: a gather, whose instructions per row are what
// has to stay below its bytes.  Both products are on the matrix cores, also for one head, with the 16 columns of a tile used for
// the precision of the float32 operand:
//   - keys (A, 16 rows x 128) times queries (B).  A column is (head, term): int8 keys go into v_mfma_i32_16x16x64_i8 as they
//     come from memory, the query as four signed digits to the base 256 of q * 2^(30 - e), |q| < 2^e, so that each digit's product
//     is an exact integer; e4m3 keys become float16 (exact) and the query three float16 terms (eight heads: two, to the
//     nearest each: off by at most 2^-23 of an element, as two roundings of float32, with no sign of its own).  The terms of a head
//     are added across the columns of a lane row.
//   - values (A, 16 dimensions x 32 rows) times weights (B).  Logits leave the first product with a head in each column and
//     four rows of each of two tiles in each lane, which is the B operand of the second as it stands: no exchange between lanes.
//     Weights are split into three bfloat16 terms by truncation, again a column each (eight heads have two columns each, and a
//     second product for the third term): the range of float32 stays (v_scale is in the weight), and its 24 bits.  A lane loads
//     8 bytes of each of its 8 rows; the dimensions of tile t are 8 n + t, so that the transposition is a choice of bytes within a lane.
// Window rows are turned back by their distance, (q R_delta) . k = q . (k R_-delta), and go in as two float16 terms (2^-23, as
// above; a third would be half as many products again).  What is left in the tail, at most a block, is done on the vector ALU.
// The statistics, all sums and the output are float32.  Logits are kept times log2 e, so that a weight is one exponential.
//
// Measured: 32 x 28 heads of 2176 rows, e4m3, 97 - 101 us for 497 MB of rows that heads ask for, of which 453 MB are different ones (the
// heads of a KV head share the rest in L2): 4.5 - 4.7 TB/s, a large copy has 4.9; the same rows of int8, in blocks of 16, 93 us; 4 x 32
// heads of 2304 rows, int8, in 4 parts 21 us = 3.4 TB/s, of which the merge is 4; one selection for 4 heads, 16 x 8 of
// 1152 rows in pages, in 2 parts 20.5 us = 1.9 TB/s, for 7 heads, 32 x 4 of 2176 rows in 4 parts, int8 24, e4m3 23 us = 3.1 TB/s (float32
// queries the same within 4 %): few rows, and requests that wait for each other (length and index, page, row), of which a wave has two
// pairs of rows in flight.  More in flight does not fit: 128 registers for four waves a SIMD spill, and a spill waits for all
// loads (three times slower), so there are two waves a SIMD with 256.
#include <algorithm>

#include "internal.hpp"
#include "kv_attn.hpp"

namespace a2ats {
namespace {

constexpr int kD = kRowBytes;
constexpr int kThreads = 256, kWaves = kThreads / 64;

// Sum over aligned groups of 8 lanes, in every lane.
__device__ __forceinline__ float group8_fsum(float v) {
  v += dpp<0xB1>(v);    // quad_perm [1,0,3,2]
  v += dpp<0x4E>(v);    // quad_perm [2,3,0,1]
  v += dpp<0x141>(v);   // row_half_mirror
  return v;
}

__device__ __forceinline__ float code_float(uint32_t w, int byte) {   // of int8
  return (float)(int8_t)((w >> (8 * byte)) & 255u);
}

struct AttnArgs {
  BlockCache cache;
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

// The rows of a pair of tiles as they come from memory: keys of row `column` of either tile, 32 elements; values of the rows
// 4 * lane row + 0 .. 3 of either, 8 elements.
struct PairRows {
  uint4 k[2][2];
  uint2 v[8];
};
// Where the rows of two pairs are in the cache, their scales, and 0 or, for a place without a row, all bits: of a wave, in LDS.
struct alignas(16) PairPlaces {
  uint32_t row[2 * kPair];
  float ks[2 * kPair], vs[2 * kPair];
  uint32_t none[2 * kPair];
};

// Eight rows of the incomplete block, one for each group of 8 lanes, and a head's query for them: elements 8 * (lane of the group)
// + 0 .. 7 of either half of keys and query, 16 * (lane of the group) + 0 .. 15 of the values.
struct TailRows {
  float q[16], k[16], v[16], cs[8], sn[8];
};
struct TailState {
  float m, l, o[16];
};

// A wave's running softmax: a head in each column (the same m in all lane rows, l of the lane's own rows), and its output,
// o[t][i] being dimension 8 * (4 * lane row + i) + t.
struct WaveState {
  float m, l;
  f32x4 o[8];
};

__device__ __forceinline__ void load_keys(const uint8_t* k, const uint32_t* rows, int col, int at, int step, PairRows& p) {
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const uint32_t r = rows[t * 16 + col];
    const uint8_t* from = k + (size_t)r * kRowBytes + at;
    p.k[t][0] = *(const uint4*)from;
    p.k[t][1] = *(const uint4*)(from + step);
  }
}
__device__ __forceinline__ void load_values(const uint8_t* v, const uint32_t* rows, int col, int lrow, PairRows& p) {
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const uint4 r4 = *(const uint4*)(rows + t * 16 + lrow * 4);
    const uint32_t r[4] = {r4.x, r4.y, r4.z, r4.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) p.v[4 * t + i] = *(const uint2*)(v + (size_t)r[i] * kRowBytes + col * 8);
  }
}

// The weights of the two tiles' rows of a lane, from their products with the queries (times log2 e / sqrt(128), without the keys'
// scales), times v_scale; the state's maximum and sum.
__device__ __forceinline__ void pair_weights(const f32x4 (&dot)[2], const PairPlaces& pl, int first, int lrow, WaveState& st,
                                             float (&w)[8]) {
  float lg[8], vsc[8];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int at = first + t * 16 + lrow * 4;
    const float4 k4 = *(const float4*)(pl.ks + at), v4 = *(const float4*)(pl.vs + at);
    const uint4 n4 = *(const uint4*)(pl.none + at);
    const float kk[4] = {k4.x, k4.y, k4.z, k4.w}, vv[4] = {v4.x, v4.y, v4.z, v4.w};
    const uint32_t nn[4] = {n4.x, n4.y, n4.z, n4.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      lg[4 * t + i] = __uint_as_float((nn[i] & 0xff800000u) | (~nn[i] & __float_as_uint(dot[t][i] * kk[i])));   // (-inf)
      vsc[4 * t + i] = vv[i];
    }
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
    const float p = power(lg[i] - mn);
    st.l += p;
    w[i] = p * vsc[i];
  }
}

// The pair's values times its weights.
template <bool E4M3, int GP>
__device__ __forceinline__ void absorb_values(const float (&weight)[8], int term, const PairRows& p, WaveState& st) {
  // The weights' terms: a column takes its own (eight heads have two columns each: the third term is a product of its own).
  const uint32_t cut1 = term >= 1 ? 0xffff0000u : 0u, cut2 = term >= 2 ? 0xffff0000u : 0u;
  float x[8], rest[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float y = weight[i];
    if (GP == 8) {
      const float y1 = y - __uint_as_float(__float_as_uint(y) & 0xffff0000u);
      rest[i] = y1 - __uint_as_float(__float_as_uint(y1) & 0xffff0000u);
    }
    y -= __uint_as_float(__float_as_uint(y) & cut1);
    if (GP == 4) y -= __uint_as_float(__float_as_uint(y) & cut2);
    x[i] = y;
  }
  uint32_t pw[4], rw[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    pw[i] = upper_halves(x[2 * i], x[2 * i + 1]);
    if (GP == 4) pw[i] = term == 3 ? 0u : pw[i];
    if (GP == 8) rw[i] = term == 0 ? upper_halves(rest[2 * i], rest[2 * i + 1]) : 0u;
  }
  const bf16x8 pb = __builtin_bit_cast(bf16x8, make_uint4(pw[0], pw[1], pw[2], pw[3]));
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    // tiles 4 h + t: byte t of word h of the eight rows
    uint32_t r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = h ? p.v[i].y : p.v[i].x;
    uint32_t quad[2][4];   // e4m3: byte t of four rows
    if (E4M3) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t u0 = __builtin_amdgcn_perm(r[4 * i + 1], r[4 * i], 0x05010400u);
        const uint32_t u1 = __builtin_amdgcn_perm(r[4 * i + 1], r[4 * i], 0x07030602u);
        const uint32_t u2 = __builtin_amdgcn_perm(r[4 * i + 3], r[4 * i + 2], 0x05010400u);
        const uint32_t u3 = __builtin_amdgcn_perm(r[4 * i + 3], r[4 * i + 2], 0x07030602u);
        quad[i][0] = __builtin_amdgcn_perm(u2, u0, 0x05040100u);
        quad[i][1] = __builtin_amdgcn_perm(u2, u0, 0x07060302u);
        quad[i][2] = __builtin_amdgcn_perm(u3, u1, 0x05040100u);
        quad[i][3] = __builtin_amdgcn_perm(u3, u1, 0x07060302u);
      }
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (E4M3) {
          w[i] = __builtin_bit_cast(uint32_t, (i & 1) ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(quad[i >> 1][t], 1.f, true)
                                                      : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(quad[i >> 1][t], 1.f, false));
        } else {
          w[i] = upper_halves(code_float(r[2 * i], t), code_float(r[2 * i + 1], t));   // (exact)
        }
      }
      const bf16x8 vt = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
      st.o[4 * h + t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, pb, st.o[4 * h + t], 0, 0, 0);
      if (GP == 8) {
        const bf16x8 rb = __builtin_bit_cast(bf16x8, make_uint4(rw[0], rw[1], rw[2], rw[3]));
        st.o[4 * h + t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, rb, st.o[4 * h + t], 0, 0, 0);
      }
    }
  }
}

// The queries of far rows as the second operand: int8 caches, four digits of eight bits; e4m3, float16 terms.
template <bool E4M3, int GP>
struct FarQuery {
  i32x4 d[E4M3 ? 1 : 2], d2[GP == 8 && !E4M3 ? 2 : 1];   // (eight heads: the third and the fourth digit)
  f16x8 f[E4M3 ? 4 : 1];
  float cw, cw2;   // what a column's product is worth
  // Elements 32 * lane row + 0 .. 31 of the column's head.
  __device__ __forceinline__ void set(const float (&x)[32], int term, bool active) {
    cw2 = 0.f;
    if constexpr (E4M3) {
      cw = query_terms<GP>(x, term, active, f);
    } else {
      bool ok;
      const int e = row_exponent(x, ok);
      // v = x 2^(30 - e), a whole number but for what is below 2^-30 of 2^e; v = ((d0 256 + d1) 256 + d2) 256 + d3 with signed
      // digits: d3 = v, d2 = (v + 0x80) >> 8, d1 = (v + 0x8080) >> 16, d0 = (v + 0x808080) >> 24, the low 8 bits of each.
      const float up = ldexpf(active ? 1.f : 0.f, 30 - e);
      const uint32_t shift = 24u - 8u * (uint32_t)term, shift2 = GP == 8 ? 8u - 8u * (uint32_t)term : 0u;
      const uint32_t bias = 0x808080u & ((1u << shift) - 1u), bias2 = 0x80u & ((1u << shift2) - 1u);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        uint32_t w = 0u, w2 = 0u;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t v = (uint32_t)(int)(x[4 * i + j] * up);
          w |= (((v + bias) >> shift) & 0xffu) << (8 * j);
          if (GP == 8) w2 |= (((v + bias2) >> shift2) & 0xffu) << (8 * j);
        }
        d[i / 4][i % 4] = (int)w;
        if constexpr (GP == 8) d2[i / 4][i % 4] = (int)w2;
      }
      cw = ok ? ldexpf(1.f, e - 30 + (int)shift) : __uint_as_float(0x7fc00000u);
      if (GP == 8) cw2 = ldexpf(1.f, e - 30 + (int)shift2);
    }
  }
  // Products of a tile's keys (32 elements of row `column`) with the queries: rows 4 * lane row + i.
  __device__ __forceinline__ f32x4 dot(const uint4 (&k)[2]) const {
    f32x4 r;
    if constexpr (E4M3) {
      const uint32_t w[8] = {k[0].x, k[0].y, k[0].z, k[0].w, k[1].x, k[1].y, k[1].z, k[1].w};
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint4 k4 = make_uint4(f16_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[2 * i], 1.f, false)),
                                    f16_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[2 * i], 1.f, true)),
                                    f16_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[2 * i + 1], 1.f, false)),
                                    f16_bits(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[2 * i + 1], 1.f, true)));
        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, k4), f[i], acc, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] = head_sum<GP>(acc[i]) * cw;
    } else {
      i32x4 acc = {0, 0, 0, 0};
      acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, k[0]), d[0], acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, k[1]), d[1], acc, 0, 0, 0);
      if constexpr (GP == 8) {
        i32x4 acc2 = {0, 0, 0, 0};
        acc2 = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, k[0]), d2[0], acc2, 0, 0, 0);
        acc2 = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, k[1]), d2[1], acc2, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = head_sum<GP>((float)acc[i] * cw + (float)acc2[i] * cw2);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = head_sum<GP>((float)acc[i] * cw);
      }
    }
    return r;
  }
};

// Products of a tile's window keys (elements 16 * lane row + 0 .. 15 of either half of row `column`), turned back by the row's
// angles, with the queries' float16 terms.
template <bool E4M3>
__device__ __forceinline__ f32x4 turned_dot(const uint4 (&k)[2], const float (&cs)[16], const float (&sn)[16], const f16x8 (&q)[4]) {
  const uint32_t lw[4] = {k[0].x, k[0].y, k[0].z, k[0].w}, uw[4] = {k[1].x, k[1].y, k[1].z, k[1].w};
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 2; ++i) {   // eight pairs of elements
    float lower[8], upper[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t wl = lw[2 * i + (j >> 2)], wu = uw[2 * i + (j >> 2)];
      float kl, ku;
      if (E4M3) {
        const auto dl = (j & 2) ? __builtin_amdgcn_cvt_pk_f32_fp8((int)wl, true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)wl, false);
        const auto du = (j & 2) ? __builtin_amdgcn_cvt_pk_f32_fp8((int)wu, true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)wu, false);
        kl = dl[j & 1];
        ku = du[j & 1];
      } else {
        kl = code_float(wl, j & 3);
        ku = code_float(wu, j & 3);
      }
      lower[j] = kl * cs[8 * i + j] + ku * sn[8 * i + j];
      upper[j] = ku * cs[8 * i + j] - kl * sn[8 * i + j];
    }
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

// E4M3: format of the codes.  GP: heads that attend the same rows (one, or the G of a KV head if the selection is shared), padded to
// 4 or 8: 16 / GP columns a head.
template <typename T, bool E4M3, int GP>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void attn_kv8_kernel(AttnArgs a) {
  __shared__ __align__(16) union {
    struct {
      PairPlaces far[kWaves][2], win[kWaves];
    } places;
    float o[kWaves][GP][kD];
  } s;
  __shared__ float s_m[kWaves][GP], s_l[kWaves][GP], s_tm[8], s_tl[8], s_to[8][kD];
  __shared__ uint32_t s_late[4];                   // selected rows of the incomplete block

  // All workgroups of a KV head run on one XCD, whose L2 then serves the rows that its heads have in common.
  const int G = a.group, nh = a.shared ? G : 1, per = a.shared ? a.parts : a.parts * G;
  int prob, pg;
  xcd_map(blockIdx.x, per, a.problems, prob, pg);
  const int Hkv = a.cache.n_kv_heads, b = prob / Hkv, kv = prob % Hkv;
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
  const int shift = a.cache.shift, blk = 1 << shift, tail0 = sr.n >> shift << shift;
  const int cnt = min(max(a.sel_count[sel], 0), a.n_sel);
  const int f1 = min(f0 + a.far_share, n_sink + (cnt << a.sel_shift));
  // ... and of the window's rows in 8 bits, [w0, w8).
  const int w0 = sr.win_start + part * a.win_share, w8 = max(w0, min(w0 + a.win_share, tail0));
  const int n_far = f1 > f0 ? (f1 - f0 + kPair - 1) / kPair : 0, n_win = (w8 - w0 + kPair - 1) / kPair;
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

  // This lane's column: a head, and which term of its query and weights.
  const int hd = col % GP, term = col / GP;
  const bool active = hd < nh;
  const size_t q_at = (size_t)(head + min(hd, nh - 1)) * kD;

  if (tid < 4) s_late[tid] = 0u;
  __syncthreads();
  if (tail0 == 0) {   // no row is in 8 bits yet
    for (int t = f0 + tid; t < f1; t += kThreads) {
      int j = t;
      if (t >= n_sink) {
        const int u = idx[(t - n_sink) >> a.sel_shift];
        j = u >= 0 && u <= (sr.n - 1) >> a.sel_shift ? (u << a.sel_shift) + ((t - n_sink) & ((1 << a.sel_shift) - 1)) : -1;
        if (j < sr.sink_end || j >= sr.win_start) continue;
      }
      if (j < sr.win_start) atomicOr(&s_late[j >> 5], 1u << (j & 31));
    }
  }

  // Where this lane's row is, and its scales, which are requested here and put beside it by put_scales.
  struct Place {
    size_t at;
    float ks, vs;
    bool in;
  };
  auto place = [&](PairPlaces& to, int j, bool in) {   // row j of the sequence
    Place pc;
    pc.in = in;
    j = in ? j : 0;   // (a place without a row: the sequence's first one, which has been written and counts for nothing)
    pc.at = block_at(a.cache, b, kv, j >> shift);
    wave_exchange();
    to.row[lane] = (uint32_t)((pc.at << shift) + (size_t)(j & (blk - 1)));
    wave_exchange();
    return pc;
  };
  auto get_scales = [&](Place& pc) {
    pc.ks = a.cache.k_scale[pc.at];
    pc.vs = a.cache.v_scale[pc.at];
  };
  auto put_scales = [&](PairPlaces& to, const Place& pc) {
    wave_exchange();
    to.ks[lane] = pc.in ? pc.ks : 0.f;
    to.vs[lane] = pc.in ? pc.vs : 0.f;
    to.none[lane] = pc.in ? 0u : ~0u;
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
    if (in && j >= tail0) {
      atomicOr(&s_late[(j - tail0) >> 5], 1u << ((j - tail0) & 31));
      in = false;
    }
    return place(to, j, in);
  };
  auto place_win = [&](int pair) {
    const int j = w0 + pair * kPair + lane;
    return place(wp, j, lane < kPair && j < w8);
  };

  // The rows of the incomplete block are done on the vector ALU, eight at a time.  Up to four heads share out the waves, eight
  // heads go to the four in turn; the window's rows are dealt out to the parts.
  const int wph = nh > 2 ? 1 : kWaves / nh, tail_head = wv / wph;
  const int slot = lane >> 3, sub = lane & 7;
  const int tail_first = max(sr.win_start - tail0, 0) >> 3, tail_chunks = (sr.n - tail0 + 7) >> 3;   // the window's
  const int tail_begin = tail_first + part;
  const bool tail_part = tail_begin < tail_chunks && a.window > 0;
  auto load_tail = [&](int g, int c, bool selected, TailRows& t) {
    const int r = min(8 * c + slot, sr.n - tail0 - 1);
    const size_t at = (size_t)(head + g) * kD + sub * 8;
    const size_t row = (((size_t)prob << shift) + r) * kD;
    load_elems<8>((const T*)a.cache.k_tail + row + sub * 8, t.k);
    load_elems<8>((const T*)a.cache.k_tail + row + kD / 2 + sub * 8, t.k + 8);
    load_elems<16>((const T*)a.cache.v_tail + row + sub * 16, t.v);
    if (selected) {
      load_elems<8>(a.q_rot + at, t.q);
      load_elems<8>(a.q_rot + at + kD / 2, t.q + 8);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        t.cs[e] = 1.f;
        t.sn[e] = 0.f;
      }
    } else {
      load_elems<8>((const T*)a.q + at, t.q);
      load_elems<8>((const T*)a.q + at + kD / 2, t.q + 8);
      const int delta = min(sr.n - 1 - tail0 - r, a.window - 1);
      load8(a.cos_win + (size_t)delta * (kD / 2) + sub * 8, t.cs);
      load8(a.sin_win + (size_t)delta * (kD / 2) + sub * 8, t.sn);
    }
  };
  auto use_tail = [&](int c, bool selected, const TailRows& t, TailState& ts) {
    const int r = 8 * c + slot;
    const bool in = r < sr.n - tail0 && (selected ? (s_late[r >> 5] >> (r & 31) & 1u) != 0u : tail0 + r >= sr.win_start);
    float dot = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      dot += t.q[e] * (t.k[e] * t.cs[e] + t.k[8 + e] * t.sn[e]);
      dot += t.q[8 + e] * (t.k[8 + e] * t.cs[e] - t.k[e] * t.sn[e]);
    }
    dot = group8_fsum(dot);
    const float lg = in ? dot * kLogit : -INFINITY;
    const float mn = fmaxf(ts.m, lg), alpha = power(ts.m - mn), pr = power(lg - mn);
    ts.l = ts.l * alpha + pr;
#pragma unroll
    for (int e = 0; e < 16; ++e) ts.o[e] = ts.o[e] * alpha + (in ? pr * t.v[e] : 0.f);
    ts.m = mn;
  };
  // The groups of 8 lanes are merged; again: with what the wave has stored for the head before.
  auto store_tail = [&](int g, TailState& ts, bool again) {
    const int to = GP == 8 ? g : wv;
    float m = rows_max(fmaxf(ts.m, dpp<0x128>(ts.m)));
    const float m_old = again ? s_tm[to] : kNone;
    m = fmaxf(m, m_old);
    const float f = power(ts.m - m), f_old = power(m_old - m);
    float l = ts.l * f;
    l = rows_sum(l + dpp<0x128>(l)) + (again ? s_tl[to] * f_old : 0.f);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      float o = ts.o[e] * f;
      o = rows_sum(o + dpp<0x128>(o));
      if (slot == 0) s_to[to][sub * 16 + e] = o + (again ? s_to[to][sub * 16 + e] * f_old : 0.f);
    }
    wave_exchange();   // (all lanes have read what the wave stored before)
    if (lane == 0) {
      s_tm[to] = m;
      s_tl[to] = l;
    }
  };

  // A wave takes its pairs of the window, then those of the far rows, two of which are in flight at a time: a pair's keys and
  // values are requested when those of the pair two before it have been used.  What does not depend on other loads comes first.
  const int far_n = tail0 > 0 ? far_end - far_first : 0;
  const bool has_win = win_first < n_win;
  const int tail_c = tail_begin + a.parts * (wv % wph);
  WaveState st;
  PairRows pa, pc;
  Place far_place;
  st.m = kNone;
  st.l = 0.f;
#pragma unroll
  for (int t = 0; t < 8; ++t) st.o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto load_far = [&](const uint32_t* rows, PairRows& p) {
    load_keys(a.cache.k, rows, col, lrow * 32, 16, p);
    load_values(a.cache.v, rows, col, lrow, p);
  };
  if (has_win) {
    float x[32];
    load_elems<16>((const T*)a.q + q_at + lrow * 16, x);
    load_elems<16>((const T*)a.q + q_at + kD / 2 + lrow * 16, x + 16);
    Place win_place = place_win(win_first);
    if (far_n > 0) far_place = place_far(fp[0], far_first);
    get_scales(win_place);
    if (far_n > 0) get_scales(far_place);
    load_keys(a.cache.k, wp.row, col, lrow * 16, kD / 2, pc);
    load_values(a.cache.v, wp.row, col, lrow, pc);
    if (far_n > 0) load_far(fp[0].row, pa);
    f16x8 qw[4];
    to_logits(x);
    const float ww = query_terms<GP>(x, term, active, qw);
    if (far_n > 0) put_scales(fp[0], far_place);
#pragma unroll 1
    for (int pair = win_first; pair < n_win; pair += kWaves) {
      f32x4 dot[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int delta = min(max(sr.n - 1 - (w0 + pair * kPair + t * 16 + col), 0), a.window - 1);
        float cs[16], sn[16];
        load_elems<16>(a.cos_win + (size_t)delta * (kD / 2) + lrow * 16, cs);
        load_elems<16>(a.sin_win + (size_t)delta * (kD / 2) + lrow * 16, sn);
        const f32x4 acc = turned_dot<E4M3>(pc.k[t], cs, sn, qw);
#pragma unroll
        for (int i = 0; i < 4; ++i) dot[t][i] = head_sum<GP>(acc[i]) * ww;
      }
      put_scales(wp, win_place);
      float w[8];
      pair_weights(dot, wp, 0, lrow, st, w);
      absorb_values<E4M3, GP>(w, term, pc, st);
      if (pair + kWaves < n_win) {
        win_place = place_win(pair + kWaves);
        get_scales(win_place);
        load_keys(a.cache.k, wp.row, col, lrow * 16, kD / 2, pc);
        load_values(a.cache.v, wp.row, col, lrow, pc);
      }
    }
    if (far_n > 1) load_far(fp[0].row + kPair, pc);
  }
  if (far_n > 0) {
    FarQuery<E4M3, GP> fq;
    float x[32];
    load_elems<32>(a.q_rot + q_at + lrow * 32, x);
    if (!has_win) {
      far_place = place_far(fp[0], far_first);
      get_scales(far_place);
      load_far(fp[0].row, pa);
      if (far_n > 1) load_far(fp[0].row + kPair, pc);
      put_scales(fp[0], far_place);
    }
    if (far_n > 2) unit = unit_of(far_row(far_first + 2));
    to_logits(x);
    fq.set(x, term, active);
    auto use = [&](PairRows& p, const PairPlaces& pl, int first) {
      f32x4 dot[2];
      dot[0] = fq.dot(p.k[0]);
      dot[1] = fq.dot(p.k[1]);
      float w[8];
      pair_weights(dot, pl, first, lrow, st, w);
      absorb_values<E4M3, GP>(w, term, p, st);
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
      if (more) load_far(next.row, pa);
      if (i + 1 < far_n) use(pc, pl, kPair);
      if (i + 3 < far_n) load_far(next.row + kPair, pc);
      if (more) put_scales(next, far_place);
      buf ^= 1;
    }
  }
  if (tail_part) {
#pragma unroll 1
    for (int g = tail_head; g < (GP == 8 ? 8 : kWaves / wph); g += kWaves) {
      TailState ts;
      ts.m = kNone;
      ts.l = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) ts.o[e] = 0.f;
      if (g < nh) {
#pragma unroll 1
        for (int c = tail_c; c < tail_chunks; c += a.parts * wph) {
          TailRows tr;
          load_tail(g, c, false, tr);
          use_tail(c, false, tr, ts);
        }
      }
      store_tail(g, ts, false);
    }
  }
  __syncthreads();   // (the places are written again, with the outputs)

  // Selected rows of the incomplete block (only where the window is shorter than that block).
  const bool late = (s_late[0] | s_late[1] | s_late[2] | s_late[3]) != 0u, has_tail = late || tail_part;
  if (late) {
#pragma unroll 1
    for (int g = tail_head; g < (GP == 8 ? 8 : kWaves / wph); g += kWaves) {
      if (g >= nh) continue;
      TailState ts;
      ts.m = kNone;
      ts.l = 0.f;
#pragma unroll
      for (int e = 0; e < 16; ++e) ts.o[e] = 0.f;
#pragma unroll 1
      for (int c = wv % wph; 8 * c < sr.n - tail0; c += wph) {
        TailRows tr;
        load_tail(g, c, true, tr);
        use_tail(c, true, tr, ts);
      }
      store_tail(g, ts, tail_part);
    }
  }

  // The terms of a head are added up, and the waves merged.
  const float l_all = rows_sum(st.l);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float o[8];
#pragma unroll
    for (int t = 0; t < 8; ++t) o[t] = head_sum<GP>(st.o[t][i]);
    if (term == 0) {
      float* to = &s.o[wv][hd][8 * (4 * lrow + i)];
      *(float4*)to = make_float4(o[0], o[1], o[2], o[3]);
      *(float4*)(to + 4) = make_float4(o[4], o[5], o[6], o[7]);
    }
  }
  if (lane < GP) {
    s_m[wv][lane] = st.m;
    s_l[wv][lane] = l_all;
  }
  __syncthreads();
  for (int i = tid; i < nh * kD; i += kThreads) {
    const int g = i / kD, d = i % kD;
    float m = kNone, l = 0.f, o = 0.f;
    if (has_tail) {
      const int t0 = GP == 8 ? g : g * wph, tn = GP == 8 ? 1 : wph;
      for (int w = t0; w < t0 + tn; ++w) m = fmaxf(m, s_tm[w]);
      for (int w = t0; w < t0 + tn; ++w) {
        const float f = power(s_tm[w] - m);
        l += s_tl[w] * f;
        o += s_to[w][d] * f;
      }
    }
    float mn = m;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) mn = fmaxf(mn, s_m[w][g]);
    const float f = power(m - mn);
    l *= f;
    o *= f;
    m = mn;
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

// Merges the parts of a head, at most 32, a thread per output element.
template <typename T>
__global__ __launch_bounds__(kD) void attn_kv8_merge_kernel(const float* __restrict__ partial, T* __restrict__ out, int parts) {
  const float* p = partial + (size_t)blockIdx.x * parts * (kD + 2);
  const int d = threadIdx.x, lane = d & 63;
  const float* mine = p + (size_t)min(lane, parts - 1) * (kD + 2) + kD;
  const float mp = mine[0], lp = mine[1];
  float o8[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) o8[i] = p[(size_t)min(i, parts - 1) * (kD + 2) + d];
  float m = mp;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) m = fmaxf(m, __shfl_xor(m, off));
  const float f = lane < parts ? power(mp - m) : 0.f;
  float l = f * (lane < parts ? lp : 0.f), o = 0.f;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) l += __shfl_xor(l, off);
#pragma unroll
  for (int i = 0; i < 8; ++i) o += i < parts ? __shfl(f, i) * o8[i] : 0.f;
  for (int i = 8; i < parts; ++i) o += __shfl(f, i) * p[(size_t)i * (kD + 2) + d];
  l = __shfl(l, 0);
  store_elem(out + (size_t)blockIdx.x * kD + d, l == 0.f ? 0.f : o / l);
}

}  // namespace

// Parts: a second launch (3 to 4.6 us in whole steps, 2 at least) and as many more first requests to wait for, against rows that wait for each other.  From all
// counts of parts up to 32 of 2 to 896 problems with 160 to 2304 rows (bfloat16, int8, selections of one head and shared by four), us
// with one part -> with the parts taken:
//   - a workgroup for every CU where there are few problems: 4 problems, 576 rows 10.4 -> 8.4 (8 parts), 2304 rows 27.0 -> 9.9
//     (12); 32 problems, 1152 rows 17.1 -> 9.7 (8); 64 problems, 576 rows 11.2 -> 9.7 (4); but 160 rows of any number of problems
//     are faster in one part (6.5 -> 8.1 for two);
//   - up to 128 problems, 1152 rows 17.9 -> 15.2 (2), 576 rows would be 11.9 -> 12.6; 2304 rows 31.2 -> 20.6 (4);
//   - many rows of up to 511 problems in two: 256 problems, 2304 rows 39.1 -> 37.0, 384 problems 56.5 -> 53.0, but 512 problems
//     62.4 -> 66.2, and 1152 rows of 256 problems 20.1 -> 20.7.
Kv8Plan make_kv8_plan(const a2ats_dims& d, long sel_rows, int window, bool shared) {
  Kv8Plan p;
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

template <typename T, bool E4M3>
static void launch_heads(const AttnArgs& a, long workgroups, hipStream_t stream) {
  const dim3 grid((unsigned)workgroups), block(kThreads);
  if (a.shared && a.group > 4) hipLaunchKernelGGL((attn_kv8_kernel<T, E4M3, 8>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((attn_kv8_kernel<T, E4M3, 4>), grid, block, 0, stream, a);
}

hipError_t launch_sparse_attn_kv8(const a2ats_dims& d, const BlockCache& m, int kv_dtype, int format, const void* q,
                                  const float* q_rot, const int32_t* sel_idx, const int32_t* sel_count, int n_sel, int sel_shift,
                                  bool shared, int window, int n_sink, const float* cos_win, const float* sin_win,
                                  const int32_t* seq_lens, void* out, void* ws, hipStream_t stream) {
  if (d.batch == 0) return hipSuccess;
  const Kv8Plan p = make_kv8_plan(d, (long)n_sel << sel_shift, window, shared);
  AttnArgs a;
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
  const bool e4m3 = format == A2ATS_E4M3;
  if (kv_dtype == A2ATS_BF16) {
    if (e4m3) launch_heads<uint16_t, true>(a, workgroups, stream);
    else launch_heads<uint16_t, false>(a, workgroups, stream);
  } else {
    if (e4m3) launch_heads<float, true>(a, workgroups, stream);
    else launch_heads<float, false>(a, workgroups, stream);
  }
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || p.parts == 1 ? e : launch_attn_merge(kv_dtype, (const float*)ws, out, d.batch * d.n_q_heads, p.parts, stream);
}

hipError_t launch_attn_merge(int kv_dtype, const float* partial, void* out, int heads, int parts, hipStream_t stream) {
  if (kv_dtype == A2ATS_BF16)
    hipLaunchKernelGGL((attn_kv8_merge_kernel<uint16_t>), dim3(heads), dim3(kD), 0, stream, partial, (uint16_t*)out, parts);
  else
    hipLaunchKernelGGL((attn_kv8_merge_kernel<float>), dim3(heads), dim3(kD), 0, stream, partial, (float*)out, parts);
  return hipGetLastError();
}

}  // namespace a2ats
