// Selection of blocks: every block of a cache has an upper bound of its tokens' logits, and the top-K blocks of each
// query head (or of each KV head) are selected.
//
// Under WRoPE all tokens outside the window see the query at one offset, q~ = q R_b, so a bound over pre-RoPE keys holds:
//     q~ . k_j  <=  s = sum_d max(q~_d lo_d, q~_d hi_d)        (lo, hi: the block's bounds per dimension)
//               =  1/2 sum_d q~_d (lo_d + hi_d) + |q~_d| (hi_d - lo_d) ,
// two products per dimension and head without a choice between lo and hi.  Shared selection: the sum over the G heads of a
// KV head is the same form with sum_g q~_g and sum_g |q~_g|, so it costs one head.  Sums are float64 (the products of
// float32 numbers are exact), rounded once to float32: the order of the blocks does not depend on how a sum is cut up.
//
// The scores are a stream over the bounds (2 * 128 * e bytes per block and KV head, read once for all G heads): 16 lanes
// take a block, 8 dimensions each.  Then a workgroup per head finds the K-th score by radix digits and writes the
// selection in ascending order.
#include "internal.hpp"
#include "kv_blocks.hpp"

namespace a2ats {
namespace {

constexpr int kScoreThreads = 256;
constexpr int kPickThreads = 1024;
constexpr int kPickBins = 2048;
constexpr int kD = kRowBytes;

// Sum over the 16 lanes of a DPP row, in every lane.
template <int CTRL>
__device__ __forceinline__ double dpp_move(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, 0xf, 0xf, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, 0xf, 0xf, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double row16_sum(double v) {
  v += dpp_move<0xB1>(v);    // quad_perm [1,0,3,2]
  v += dpp_move<0x4E>(v);    // quad_perm [2,3,0,1]
  v += dpp_move<0x141>(v);   // row_half_mirror
  v += dpp_move<0x140>(v);   // row_mirror
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

// G: query heads of a KV head.  NH: scores of a block (G, or 1 if the selection is shared).
template <typename T, int G, bool SHARED>
__global__ __launch_bounds__(kScoreThreads) void score_blocks_kernel(
    BlockCache m, const T* __restrict__ q, const float* __restrict__ cos_b, const float* __restrict__ sin_b,
    float* __restrict__ q_rot, float* __restrict__ scores, int total_blocks, int chunk, int chunks, int problems, int ctx_len,
    const int32_t* __restrict__ seq_lens, int window, int n_sink) {
  constexpr int NH = SHARED ? 1 : G;
  constexpr int U = 2;   // blocks of a group of 16 lanes whose bounds are requested together
  int prob, part;
  xcd_map(blockIdx.x, chunks, problems, prob, part);
  const int b = prob / m.n_kv_heads, kv = prob % m.n_kv_heads;
  const int lane = threadIdx.x & 63, d0 = (lane & 15) * 8;
  const SeqRange sr = seq_range(ctx_len, seq_lens, b, window, n_sink, 0);
  int first, last;
  candidate_blocks(sr, m.shift, first, last);

  double q1[NH][8], q2[SHARED ? 1 : 1][SHARED ? 8 : 1];
  {
    const bool lower = d0 < kD / 2;
    const int t = d0 & (kD / 2 - 1);
    float cs[8], sn[8];
    load8(cos_b + t, cs);
    load8(sin_b + t, sn);
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const T* row = q + ((size_t)prob * G + g) * kD;
      float own[8], other[8];
      load8(row + d0, own);
      load8(row + (d0 ^ (kD / 2)), other);
      float* out = q_rot + ((size_t)prob * G + g) * kD + d0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double x = (double)own[e] * cs[e], y = (double)other[e] * sn[e];
        const float r = (float)(lower ? x - y : x + y);
        if (part == 0 && threadIdx.x < 16) out[e] = r;
        if constexpr (SHARED) {
          q1[0][e] = (g ? q1[0][e] : 0.0) + (double)r;
          q2[0][e] = (g ? q2[0][e] : 0.0) + (double)fabsf(r);
        } else {
          q1[g][e] = (double)r;
        }
      }
    }
  }
  const int end = min(last, first + (part + 1) * chunk);
  const T* bounds = (const T*)m.bounds;
  for (int c0 = first + part * chunk + (int)(threadIdx.x >> 4); c0 - (int)((threadIdx.x >> 4) & 3) < end;
       c0 += U * (kScoreThreads / 16)) {
    float lo[U][8], hi[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = min(c0 + u * (kScoreThreads / 16), end - 1);
      const T* p = bounds + block_at(m, b, kv, c) * 2 * kD + d0;
      load8(p, lo[u]);
      load8(p + kD, hi[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      double s[NH];
#pragma unroll
      for (int g = 0; g < NH; ++g) s[g] = 0.0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double l = lo[u][e], h = hi[u][e], mid = l + h, half = h - l;
#pragma unroll
        for (int g = 0; g < NH; ++g) {
          s[g] = __builtin_fma(q1[g][e], mid, s[g]);
          s[g] = __builtin_fma(SHARED ? q2[0][e] : __builtin_fabs(q1[g][e]), half, s[g]);
        }
      }
      const int c = c0 + u * (kScoreThreads / 16);
#pragma unroll
      for (int g = 0; g < NH; ++g) {
        const double sum = row16_sum(s[g]) * 0.5;
        float f = (float)sum + 0.f;   // (one zero)
        f = f != f ? INFINITY : f;
        if ((lane & 15) == 0 && c < end) scores[((size_t)prob * NH + g) * total_blocks + c] = f;
      }
    }
  }
}

// PER: scores of a thread, in registers.
template <int PER>
__global__ __launch_bounds__(kPickThreads) void pick_blocks_kernel(
    const float* __restrict__ scores, int total_blocks, int shift, int heads, int ctx_len, const int32_t* __restrict__ seq_lens,
    int window, int n_sink, int top_blocks, int32_t* __restrict__ block_idx, int32_t* __restrict__ block_count,
    float* __restrict__ block_score, int32_t* __restrict__ token_idx, int32_t* __restrict__ token_count) {
  constexpr int NT = kPickThreads;
  __shared__ uint32_t s_hist[kPickBins];
  __shared__ uint32_t s_a[NT / 64], s_b[NT / 64], s_c[NT / 64], s_res[2], s_lo, s_hi;
  extern __shared__ int32_t s_sel[];   // the selection, if tokens are asked for
  const int bh = blockIdx.x, b = bh / heads, tid = threadIdx.x, lane = tid & 63;
  const SeqRange sr = seq_range(ctx_len, seq_lens, b, window, n_sink, 0);
  int first, last;
  candidate_blocks(sr, shift, first, last);
  const int n = last - first, kk = min(top_blocks, n);
  if (tid == 0) {
    block_count[bh] = kk;
    s_lo = ~0u;
    s_hi = 0u;
  }
  int32_t* idx = block_idx + (size_t)bh * top_blocks;
  float* score = block_score ? block_score + (size_t)bh * top_blocks : nullptr;
  for (int i = kk + tid; i < top_blocks; i += NT) {
    idx[i] = -1;
    if (score) score[i] = 0.f;
  }
  __syncthreads();
  // Thread t has the blocks [t PER, (t + 1) PER) of the candidates.
  const float* src = scores + (size_t)bh * total_blocks + first;
  uint32_t key[PER];
  uint32_t k_min = ~0u, k_max = 0u;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int c = tid * PER + i;
    key[i] = c < n ? order_key(src[c]) : 0u;
    if (c < n) {
      k_min = min(k_min, key[i]);
      k_max = max(k_max, key[i]);
    }
  }
  k_max = wave_max_to_last_lane(k_max);
  k_min = ~wave_max_to_last_lane(~k_min);
  if (lane == 63) {
    atomicMax(&s_hi, k_max);
    atomicMin(&s_lo, k_min);
  }
  __syncthreads();
  // The kk-th largest key by digits of 11 bits from the highest bit in which the keys differ, so that they spread over the
  // bins; `equal` of the keys that have it are selected, the lowest blocks first.
  uint32_t kth = 0, equal = 0;
  if (kk > 0 && kk < n) {
    const uint32_t base = s_lo, range = s_hi - base;
    uint32_t left = (uint32_t)kk, prefix = 0;
    int shift_now = 32 - (range ? __clz(range) : 32);
    while (shift_now > 0) {
      const int width = min(shift_now, 11), above = shift_now;
      shift_now -= width;
      for (int i = tid; i < kPickBins; i += NT) s_hist[i] = 0;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const uint32_t rel = key[i] - base;
        if (tid * PER + i < n && (above >= 32 || rel >> above == prefix)) atomicAdd(&s_hist[(rel >> shift_now) & ((1u << width) - 1u)], 1u);
      }
      __syncthreads();
      block_find_rank_desc<NT, kPickBins>([&](int bin) { return s_hist[bin]; }, left, s_a, s_res);
      prefix = (prefix << width) | s_res[0];
      left -= s_res[1];
      __syncthreads();
    }
    kth = base + prefix;
    equal = left;
  } else if (kk > 0) {
    kth = 0;   // all: every key is larger (no score maps to 0, which would be a NaN)
    equal = 0;
  }
  uint32_t n_above = 0, n_equal = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const bool in = tid * PER + i < n && kk > 0;
    n_above += in && key[i] > kth;
    n_equal += in && key[i] == kth;
  }
  uint32_t total;
  uint32_t equal_at = block_exclusive_scan<NT>(n_equal, s_b, total);
  const uint32_t taken = min(n_equal, equal > equal_at ? equal - equal_at : 0u);
  uint32_t at = block_exclusive_scan<NT>(n_above + taken, s_c, total);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int c = tid * PER + i;
    if (c >= n || kk == 0) continue;
    bool take = key[i] > kth;
    if (key[i] == kth) take = equal_at++ < equal;
    if (take) {
      idx[at] = first + c;
      if (score) score[at] = key_value(key[i]);
      if (token_idx) s_sel[at] = first + c;
      ++at;
    }
  }
  if (token_idx == nullptr) return;   // (uniform)
  __syncthreads();
  // The tokens: whole blocks but for the first and the last candidate block, of which the candidates are taken.
  const int blk = 1 << shift, all = top_blocks << shift;
  const int skip = kk > 0 && s_sel[0] == first ? sr.sink_end - (first << shift) : 0;
  const int cut = kk > 0 && s_sel[kk - 1] == last - 1 ? (last << shift) - sr.win_start : 0;
  const int count = (kk << shift) - skip - cut;
  if (tid == 0) token_count[bh] = count;
  int32_t* tokens = token_idx + (size_t)bh * all;
  for (int i = tid; i < all; i += NT) {
    const int t = i + skip;
    tokens[i] = i < count ? (s_sel[t >> shift] << shift) + (t & (blk - 1)) : -1;
  }
}

}  // namespace

BlockTopkPlan make_block_topk_plan(const a2ats_dims& d, int block, bool shared) {
  BlockTopkPlan p;
  const long problems = (long)d.batch * d.n_kv_heads;
  p.total_blocks = (int)(((long)d.ctx_len + block - 1) / block);
  // Four rounds of workgroups over the CUs, each with 32 blocks at least (two steps of its groups of 16 lanes).
  long chunks = problems > 0 ? (2048 + problems - 1) / problems : 1;
  chunks = std::max(1l, std::min(chunks, (long)p.total_blocks / 32));
  p.chunk = std::max(1, (int)((p.total_blocks + chunks - 1) / chunks));
  p.chunks = std::max(1, (p.total_blocks + p.chunk - 1) / p.chunk);
  p.bytes = (size_t)d.batch * (shared ? d.n_kv_heads : d.n_q_heads) * p.total_blocks * sizeof(float);
  return p;
}

template <typename T, int G>
static void launch_score(const a2ats_dims& d, const BlockCache& m, const BlockTopkPlan& p, const void* q, const float* cos_b,
                         const float* sin_b, float* q_rot, bool shared, int window, int n_sink, const int32_t* seq_lens,
                         void* ws, hipStream_t stream) {
  const int problems = d.batch * d.n_kv_heads;
  const dim3 grid((unsigned)(problems * p.chunks)), block(kScoreThreads);
  if (shared)
    hipLaunchKernelGGL((score_blocks_kernel<T, G, true>), grid, block, 0, stream, m, (const T*)q, cos_b, sin_b, q_rot, (float*)ws,
                       p.total_blocks, p.chunk, p.chunks, problems, d.ctx_len, seq_lens, window, n_sink);
  else
    hipLaunchKernelGGL((score_blocks_kernel<T, G, false>), grid, block, 0, stream, m, (const T*)q, cos_b, sin_b, q_rot, (float*)ws,
                       p.total_blocks, p.chunk, p.chunks, problems, d.ctx_len, seq_lens, window, n_sink);
}

template <typename T, typename... A>
static void launch_score_g(int G, A... a) {
  switch (G) {
    case 1: return launch_score<T, 1>(a...);
    case 2: return launch_score<T, 2>(a...);
    case 3: return launch_score<T, 3>(a...);
    case 4: return launch_score<T, 4>(a...);
    case 5: return launch_score<T, 5>(a...);
    case 6: return launch_score<T, 6>(a...);
    case 7: return launch_score<T, 7>(a...);
    default: return launch_score<T, 8>(a...);
  }
}

hipError_t launch_block_topk(const a2ats_dims& d, const BlockCache& m, int kv_dtype, const void* q, const float* cos_b,
                             const float* sin_b, float* q_rot, bool shared, int top_blocks, int window, int n_sink,
                             const int32_t* seq_lens, int32_t* block_idx, int32_t* block_count, float* block_score,
                             int32_t* token_idx, int32_t* token_count, void* ws, hipStream_t stream) {
  if (d.batch == 0) return hipSuccess;
  const BlockTopkPlan p = make_block_topk_plan(d, 1 << m.shift, shared);
  const int G = d.n_q_heads / d.n_kv_heads;
  if (kv_dtype == A2ATS_BF16)
    launch_score_g<uint16_t>(G, d, m, p, q, cos_b, sin_b, q_rot, shared, window, n_sink, seq_lens, ws, stream);
  else
    launch_score_g<float>(G, d, m, p, q, cos_b, sin_b, q_rot, shared, window, n_sink, seq_lens, ws, stream);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int heads = shared ? d.n_kv_heads : d.n_q_heads;
  const size_t lds = token_idx ? (size_t)top_blocks * sizeof(int32_t) : 0;
#define A2ATS_PICK(PER)                                                                                                   \
  hipLaunchKernelGGL((pick_blocks_kernel<PER>), dim3(d.batch * heads), dim3(kPickThreads), lds, stream, (const float*)ws,  \
                     p.total_blocks, m.shift, heads, d.ctx_len, seq_lens, window, n_sink, top_blocks, block_idx,           \
                     block_count, block_score, token_idx, token_count)
  if (p.total_blocks <= kPickThreads) A2ATS_PICK(1);
  else if (p.total_blocks <= 4 * kPickThreads) A2ATS_PICK(4);
  else if (p.total_blocks <= 16 * kPickThreads) A2ATS_PICK(16);
  else A2ATS_PICK(64);
#undef A2ATS_PICK
  return hipGetLastError();
}

}  // namespace a2ats
