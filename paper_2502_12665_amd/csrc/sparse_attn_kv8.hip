// Attention of one query token over sinks U selected tokens (or blocks) U window, from a cache held in 8 bits with a
// scale for each block of tokens and KV head:
//     logit_j = (q~ . code_j) * k_scale / sqrt(128)  (window rows: q R_delta for q~),  out = sum softmax(logit)_j code_j v_scale.
// The scales are per row of a block, so they multiply the finished product and the weight, never the 128 elements.  Rows of
// the sequence's incomplete block are in the tail, in the type of q.
//
// A row is 128 bytes of keys and as many of values, 2 flop per byte and head: a gather.  LPR lanes take a row, 128 / LPR
// elements each; a wave works on 64 / LPR rows at once and has two sets of U of them, one requested while the other is used.
// Each group of LPR lanes keeps its own running maximum, sum and accumulator, and one rescaling serves the U rows
// of a set; the groups, then the waves, then (where a head's rows are shared out among workgroups) the workgroups are merged.
// Logits are kept times log2 e, so that a weight is one exponential of a difference.
#include <algorithm>
#include <cfloat>

#include "internal.hpp"
#include "kv_blocks.hpp"

namespace a2ats {
namespace {

constexpr int kD = kRowBytes;
constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr int kTile = 2048;            // far rows staged in LDS at a time
constexpr float kNone = -FLT_MAX;      // the maximum of no rows
constexpr float kLogit = 0.12751743f;  // log2(e) / sqrt(128)

__device__ __forceinline__ float power(float x) { return __builtin_amdgcn_exp2f(x); }

// Sum over aligned groups of 8 or 16 lanes, in every lane.
template <int LPR>
__device__ __forceinline__ float group_sum(float v) {
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xB1, 0xf, 0xf, false));    // quad_perm [1,0,3,2]
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4E, 0xf, 0xf, false));    // quad_perm [2,3,0,1]
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x141, 0xf, 0xf, false));   // row_half_mirror
  if (LPR == 16) v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x140, 0xf, 0xf, false));   // row_mirror
  return v;
}

// The four codes of a word as floats.
template <bool E4M3>
__device__ __forceinline__ void widen4(uint32_t w, float* x) {
  if (E4M3) {
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1];
  } else {
    x[0] = (float)(int8_t)(w & 255u);
    x[1] = (float)(int8_t)((w >> 8) & 255u);
    x[2] = (float)(int8_t)((w >> 16) & 255u);
    x[3] = (float)(int8_t)(w >> 24);
  }
}
template <bool E4M3, int W>
__device__ __forceinline__ void widen_words(const uint32_t (&w)[W], float (&x)[4 * W]) {
#pragma unroll
  for (int i = 0; i < W; ++i) widen4<E4M3>(w[i], x + 4 * i);
}
template <int W>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t (&w)[W]) {
  if constexpr (W == 4) {
    const uint4 v = *(const uint4*)p;
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
  } else {
    const uint2 v = *(const uint2*)p;
    w[0] = v.x; w[1] = v.y;
  }
}
// Half of DPL consecutive elements of a row in the type of q.
template <int N>
__device__ __forceinline__ void load_elems(const float* p, float* x) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const float4 v = *(const float4*)(p + i);
    x[i] = v.x; x[i + 1] = v.y; x[i + 2] = v.z; x[i + 3] = v.w;
  }
}
template <int N>
__device__ __forceinline__ void load_elems(const uint16_t* p, float* x) {
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const uint2 v = *(const uint2*)(p + i);
    x[i] = __uint_as_float(v.x << 16); x[i + 1] = __uint_as_float(v.x & 0xffff0000u);
    x[i + 2] = __uint_as_float(v.y << 16); x[i + 3] = __uint_as_float(v.y & 0xffff0000u);
  }
}
__device__ __forceinline__ void store_elem(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_elem(uint16_t* p, float v) { *p = f32_to_bf16(v); }

// Running softmax of GH heads over the rows of a group of lanes; DPL output elements a lane.
template <int GH, int DPL>
struct State {
  float m[GH], l[GH], o[GH][DPL];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int g = 0; g < GH; ++g) {
      m[g] = kNone;
      l[g] = 0.f;
#pragma unroll
      for (int e = 0; e < DPL; ++e) o[g][e] = 0.f;
    }
  }
};

// One row more for every head: `x` its values, `logit` (times log2 e) for each head.
template <int GH, int DPL>
__device__ __forceinline__ void absorb(State<GH, DPL>& st, const float (&logit)[GH], bool in, float scale, const float (&x)[DPL]) {
#pragma unroll
  for (int g = 0; g < GH; ++g) {
    const float lg = in ? logit[g] : kNone;
    const float mn = fmaxf(st.m[g], lg);
    const float alpha = power(st.m[g] - mn), p = in ? power(lg - mn) : 0.f;
    st.l[g] = st.l[g] * alpha + p;
    const float pv = p * scale;
#pragma unroll
    for (int e = 0; e < DPL; ++e) st.o[g][e] = st.o[g][e] * alpha + pv * x[e];
    st.m[g] = mn;
  }
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
  int32_t ctx_len, n_sel, sel_shift, window, n_sink, group, parts, win_waves, problems;
};

// E4M3: format of the codes.  GH: heads that attend the same rows, G of a KV head padded to 1, 2, 4 or 8 (shared selection),
// or 1.  LPR: lanes of a row.
template <typename T, bool E4M3, int GH, bool SHARED>
__global__ __launch_bounds__(kThreads) void attn_kv8_kernel(AttnArgs a) {
  constexpr int LPR = GH > 4 ? 16 : 8, DPL = kD / LPR, W = DPL / 4, SLOTS = 64 / LPR;
  constexpr int U = GH == 1 ? 4 : 2;
  __shared__ uint32_t s_row[kTile];   // row of the cache, from the first one of the base block up (or kNoRow)
  __shared__ float s_ks[kTile], s_vs[kTile];
  __shared__ uint32_t s_late[4];      // selected rows of the incomplete block
  __shared__ float s_m[kWaves][GH], s_l[kWaves][GH], s_o[kWaves][GH][kD];
  constexpr uint32_t kNoRow = 0xffffffffu;

  // All workgroups of a KV head run on one XCD, whose L2 then serves the rows that its heads have in common.
  const int G = a.group, per = SHARED ? a.parts : a.parts * G;
  int prob, pg;
  xcd_map(blockIdx.x, per, a.problems, prob, pg);
  const int Hkv = a.cache.n_kv_heads, b = prob / Hkv, kv = prob % Hkv;
  const int part = SHARED ? pg : pg / G, h0 = SHARED ? 0 : pg % G;
  const int head = prob * G + h0;                 // the first of the workgroup's heads
  const int sel = SHARED ? prob : head;           // whose selection it reads
  const int tid = threadIdx.x, lane = tid & 63, slot = lane / LPR, sub = lane % LPR;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const SeqRange sr = seq_range(a.ctx_len, a.seq_lens, b, a.window, a.n_sink, 0);
  const int shift = a.cache.shift, blk = 1 << shift, tail0 = sr.n >> shift << shift;
  const int cnt = min(max(a.sel_count[sel], 0), a.n_sel);
  const int32_t* idx = a.sel_idx + (size_t)sel * a.n_sel;
  const T* kt = (const T*)a.cache.k_tail + ((size_t)prob << shift) * kD;
  const T* vt = (const T*)a.cache.v_tail + ((size_t)prob << shift) * kD;

  // This part's share of the far rows (sinks, then the selected ones) and of the window.
  const int far_all = sr.sink_end + (cnt << a.sel_shift), win_all = sr.n - sr.win_start;
  const int f0 = (int)((long)far_all * part / a.parts), f1 = (int)((long)far_all * (part + 1) / a.parts);
  const int w0 = sr.win_start + (int)((long)win_all * part / a.parts);
  const int w1 = sr.win_start + (int)((long)win_all * (part + 1) / a.parts);

  State<GH, DPL> st;
  st.clear();
  const int far_waves = kWaves - a.win_waves;
  const bool far_role = wv < far_waves;
  // Elements of this lane: far rows DPL consecutive ones; window rows DPL / 2 of each half, which are turned together.
  constexpr int HD = DPL / 2;
  const int d_far = sub * DPL, d_win = sub * HD;
  float qv[GH][DPL];
#pragma unroll
  for (int g = 0; g < GH; ++g) {
    const int hg = head + (GH > 1 ? min(g, G - 1) : 0);
    if (far_role) {
      load_elems<DPL>(a.q_rot + (size_t)hg * kD + d_far, qv[g]);
    } else {
      load_elems<HD>((const T*)a.q + (size_t)hg * kD + d_win, qv[g]);
      load_elems<HD>((const T*)a.q + (size_t)hg * kD + kD / 2 + d_win, qv[g] + HD);
    }
  }
  if (tid < 4) s_late[tid] = 0u;

  const int tiles = max(1, (f1 - f0 + kTile - 1) / kTile);
  for (int tile = 0; tile < tiles; ++tile) {
    const int t0 = f0 + tile * kTile, tn = min(kTile, f1 - t0);
    __syncthreads();
    for (int i = tid; i < tn; i += kThreads) {
      const int t = t0 + i;
      int j = t;
      bool in = true;
      if (t >= sr.sink_end) {
        const int s = t - sr.sink_end;
        const int unit = idx[s >> a.sel_shift];
        in = unit >= 0 && unit <= (sr.n - 1) >> a.sel_shift;   // (an index from elsewhere must not leave the cache)
        j = in ? (unit << a.sel_shift) + (s & ((1 << a.sel_shift) - 1)) : 0;
        in = in && j >= sr.sink_end && j < sr.win_start;
      }
      if (in && j >= tail0) {
        atomicOr(&s_late[(j - tail0) >> 5], 1u << ((j - tail0) & 31));
        in = false;
      }
      uint32_t row = kNoRow;
      float ks = 0.f, vs = 0.f;
      if (in) {
        const size_t at = block_at(a.cache, b, kv, j >> shift);
        row = (uint32_t)((at << shift) + (size_t)(j & (blk - 1)));
        ks = a.cache.k_scale[at] * kLogit;
        vs = a.cache.v_scale[at];
      }
      s_row[i] = row;
      s_ks[i] = ks;
      s_vs[i] = vs;
    }
    __syncthreads();
    if (far_role && tn > 0) {
      const int rb = far_waves * SLOTS, step = rb * U, first = wv * SLOTS + slot;
      uint32_t ka[U][W], va[U][W], kc[U][W], vc[U][W];
      auto load_set = [&](int i0, uint32_t (&kr)[U][W], uint32_t (&vr)[U][W]) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const uint32_t row = s_row[min(i0 + u * rb, tn - 1)];
          const size_t off = (size_t)(row == kNoRow ? 0u : row) * kRowBytes + d_far;
          load_words<W>(a.cache.k + off, kr[u]);
          load_words<W>(a.cache.v + off, vr[u]);
        }
      };
      auto use_set = [&](int i0, const uint32_t (&kr)[U][W], uint32_t (&vr)[U][W]) {
        float lg[U][GH], vs[U];
        bool in[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int i = min(i0 + u * rb, tn - 1);
          in[u] = i0 + u * rb < tn && s_row[i] != kNoRow;
          vs[u] = s_vs[i];
          const float ks = s_ks[i];
          float kf[DPL];
          widen_words<E4M3, W>(kr[u], kf);
#pragma unroll
          for (int g = 0; g < GH; ++g) {
            float dot = 0.f;
#pragma unroll
            for (int e = 0; e < DPL; ++e) dot += qv[g][e] * kf[e];
            dot = group_sum<LPR>(dot) * ks;
            lg[u][g] = in[u] ? dot : kNone;
          }
        }
        float pv[U][GH];
#pragma unroll
        for (int g = 0; g < GH; ++g) {
          float mn = st.m[g];
#pragma unroll
          for (int u = 0; u < U; ++u) mn = fmaxf(mn, lg[u][g]);
          const float alpha = power(st.m[g] - mn);
          st.m[g] = mn;
          float l = st.l[g] * alpha;
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const float p = in[u] ? power(lg[u][g] - mn) : 0.f;
            l += p;
            pv[u][g] = in[u] ? p * vs[u] : 0.f;
          }
          st.l[g] = l;
#pragma unroll
          for (int e = 0; e < DPL; ++e) st.o[g][e] *= alpha;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float vf[DPL];
          if (E4M3) {   // (what is read for no row may be a NaN)
#pragma unroll
            for (int i = 0; i < W; ++i) vr[u][i] = in[u] ? vr[u][i] : 0u;
          }
          widen_words<E4M3, W>(vr[u], vf);
#pragma unroll
          for (int g = 0; g < GH; ++g)
#pragma unroll
            for (int e = 0; e < DPL; ++e) st.o[g][e] += pv[u][g] * vf[e];
        }
      };
      load_set(first, ka, va);
#pragma unroll 1
      for (int base = 0; base < tn; base += 2 * step) {
        load_set(base + step + first, kc, vc);
        use_set(base + first, ka, va);
        load_set(base + 2 * step + first, ka, va);
        use_set(base + step + first, kc, vc);
      }
    }
    if (!far_role && tile == 0) {
      // Window rows: the key is turned back by the row's distance, once for all heads:  (q R_delta) . k = q . (k R_-delta).
      const int rb = a.win_waves * SLOTS;
      auto turned = [&](int j, const float (&kf)[DPL], float (&lg)[GH], float ks) {
        const int delta = min(max(sr.n - 1 - j, 0), a.window - 1);
        const float* cp = a.cos_win + (size_t)delta * (kD / 2) + d_win;
        const float* sp = a.sin_win + (size_t)delta * (kD / 2) + d_win;
        float cs[HD], sn[HD], kr[DPL];
        load_elems<HD>(cp, cs);
        load_elems<HD>(sp, sn);
#pragma unroll
        for (int e = 0; e < HD; ++e) {
          kr[e] = kf[e] * cs[e] + kf[HD + e] * sn[e];
          kr[HD + e] = kf[HD + e] * cs[e] - kf[e] * sn[e];
        }
#pragma unroll
        for (int g = 0; g < GH; ++g) {
          float dot = 0.f;
#pragma unroll
          for (int e = 0; e < DPL; ++e) dot += qv[g][e] * kr[e];
          lg[g] = group_sum<LPR>(dot) * ks;
        }
      };
      const int w8 = min(w1, max(w0, tail0));   // [w0, w8) in 8 bits, [w8, w1) in the tail
      for (int j0 = w0 + (wv - far_waves) * SLOTS; j0 < w8; j0 += rb) {
        const int j = j0 + slot, jc = min(j, w8 - 1);
        const size_t at = block_at(a.cache, b, kv, jc >> shift);
        const size_t off = ((at << shift) + (size_t)(jc & (blk - 1))) * kRowBytes + d_win;
        uint32_t kw[2][W / 2], vw[2][W / 2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if constexpr (W == 4) {
            load_words<2>(a.cache.k + off + h * (kD / 2), kw[h]);
            load_words<2>(a.cache.v + off + h * (kD / 2), vw[h]);
          } else {
            kw[h][0] = *(const uint32_t*)(a.cache.k + off + h * (kD / 2));
            vw[h][0] = *(const uint32_t*)(a.cache.v + off + h * (kD / 2));
          }
        }
        float kf[DPL], vf[DPL], lg[GH];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < W / 2; ++i) {
            widen4<E4M3>(kw[h][i], kf + h * HD + 4 * i);
            widen4<E4M3>(vw[h][i], vf + h * HD + 4 * i);
          }
        turned(jc, kf, lg, a.cache.k_scale[at] * kLogit);
        absorb<GH, DPL>(st, lg, j < w8, a.cache.v_scale[at], vf);
      }
      for (int j0 = w8 + (wv - far_waves) * SLOTS; j0 < w1; j0 += rb) {
        const int j = j0 + slot, jc = min(j, w1 - 1);
        const size_t off = (size_t)(jc & (blk - 1)) * kD + d_win;
        float kf[DPL], vf[DPL], lg[GH];
        load_elems<HD>(kt + off, kf);
        load_elems<HD>(kt + off + kD / 2, kf + HD);
        load_elems<HD>(vt + off, vf);
        load_elems<HD>(vt + off + kD / 2, vf + HD);
        turned(jc, kf, lg, kLogit);
        absorb<GH, DPL>(st, lg, j < w1, 1.f, vf);
      }
    }
  }
  // Far rows of the incomplete block (only where the window is shorter than that block).
  __syncthreads();
  if (wv == 0 && (s_late[0] | s_late[1] | s_late[2] | s_late[3]) != 0u) {
    for (int r0 = 0; r0 < sr.n - tail0; r0 += SLOTS) {
      const int r = min(r0 + slot, sr.n - 1 - tail0);
      const bool in = r0 + slot < sr.n - tail0 && (s_late[r >> 5] >> (r & 31) & 1u);
      float kf[DPL], vf[DPL], lg[GH];
      load_elems<DPL>(kt + (size_t)r * kD + d_far, kf);
      load_elems<DPL>(vt + (size_t)r * kD + d_far, vf);
#pragma unroll
      for (int g = 0; g < GH; ++g) {
        float dot = 0.f;
#pragma unroll
        for (int e = 0; e < DPL; ++e) dot += qv[g][e] * kf[e];
        lg[g] = group_sum<LPR>(dot) * kLogit;
      }
      absorb<GH, DPL>(st, lg, in, 1.f, vf);
    }
  }

  // The groups of a wave take the wave's maximum and are added up.
#pragma unroll
  for (int g = 0; g < GH; ++g) {
    float m = st.m[g];
#pragma unroll
    for (int off = LPR; off < 64; off <<= 1) m = fmaxf(m, __shfl_xor(m, off));
    const float f = power(st.m[g] - m);
    float l = st.l[g] * f;
#pragma unroll
    for (int off = LPR; off < 64; off <<= 1) l += __shfl_xor(l, off);
#pragma unroll
    for (int e = 0; e < DPL; ++e) {
      float o = st.o[g][e] * f;
#pragma unroll
      for (int off = LPR; off < 64; off <<= 1) o += __shfl_xor(o, off);
      const int d = far_role ? d_far + e : (e < HD ? d_win + e : kD / 2 + d_win + e - HD);
      if (slot == 0) s_o[wv][g][d] = o;
    }
    if (lane == 0) {
      s_m[wv][g] = m;
      s_l[wv][g] = l;
    }
  }
  __syncthreads();
  for (int i = tid; i < GH * kD; i += kThreads) {
    const int g = i / kD, d = i % kD;
    if (GH > 1 && g >= G) break;
    float m = s_m[0][g];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) m = fmaxf(m, s_m[w][g]);
    float l = 0.f, o = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = power(s_m[w][g] - m);
      l += s_l[w][g] * f;
      o += s_o[w][g][d] * f;
    }
    if (a.parts == 1) {
      store_elem((T*)a.out + (size_t)(head + g) * kD + d, l == 0.f ? 0.f : o / l);
    } else {
      float* p = a.partial + ((size_t)(head + g) * a.parts + part) * (kD + 2);
      p[d] = o;
      if (d == 0) {
        p[kD] = m;
        p[kD + 1] = l;
      }
    }
  }
}

// Merges the parts of a head, a thread per output element.
template <typename T>
__global__ __launch_bounds__(kD) void attn_kv8_merge_kernel(const float* __restrict__ partial, T* __restrict__ out, int parts) {
  const float* p = partial + (size_t)blockIdx.x * parts * (kD + 2);
  const int d = threadIdx.x;
  float m = kNone;
  for (int i = 0; i < parts; ++i) m = fmaxf(m, p[(size_t)i * (kD + 2) + kD]);
  float l = 0.f, o = 0.f;
#pragma unroll 8
  for (int i = 0; i < parts; ++i) {
    const float* s = p + (size_t)i * (kD + 2);
    const float f = power(s[kD] - m);
    l += s[kD + 1] * f;
    o += s[d] * f;
  }
  store_elem(out + (size_t)blockIdx.x * kD + d, l == 0.f ? 0.f : o / l);
}

}  // namespace

Kv8Plan make_kv8_plan(const a2ats_dims& d, long sel_rows, int window, bool shared) {
  Kv8Plan p;
  const long problems = (long)d.batch * (shared ? d.n_kv_heads : d.n_q_heads);
  const long rows = std::min<long>(sel_rows, d.ctx_len) + std::min(window, d.ctx_len);
  // Two workgroups a CU, each with 128 rows at least (16 a wave).
  long parts = problems > 0 ? (512 + problems - 1) / problems : 1;
  parts = std::max(1l, std::min(std::min(parts, rows / 128), 32l));
  p.parts = (int)parts;
  p.bytes = parts > 1 ? (size_t)d.batch * d.n_q_heads * parts * (kD + 2) * sizeof(float) : 0;
  return p;
}

template <typename T, bool E4M3>
static void launch_heads(const AttnArgs& a, bool shared, long workgroups, hipStream_t stream) {
  const dim3 grid((unsigned)workgroups), block(kThreads);
  if (!shared) hipLaunchKernelGGL((attn_kv8_kernel<T, E4M3, 1, false>), grid, block, 0, stream, a);
  else if (a.group == 1) hipLaunchKernelGGL((attn_kv8_kernel<T, E4M3, 1, true>), grid, block, 0, stream, a);
  else if (a.group == 2) hipLaunchKernelGGL((attn_kv8_kernel<T, E4M3, 2, true>), grid, block, 0, stream, a);
  else if (a.group <= 4) hipLaunchKernelGGL((attn_kv8_kernel<T, E4M3, 4, true>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((attn_kv8_kernel<T, E4M3, 8, true>), grid, block, 0, stream, a);
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
  a.parts = p.parts;
  a.problems = d.batch * d.n_kv_heads;
  // Waves for the window in proportion to its rows, which cost about half as much again as others.
  const long far = std::min<long>(((long)n_sel << sel_shift) + n_sink, d.ctx_len), win = 3l * std::min(window, d.ctx_len);
  const long all = std::max(1l, 2 * far + win);
  a.win_waves = window == 0 ? 0 : std::min(kWaves - 1, std::max(1, (int)((kWaves * win + all / 2) / all)));
  const long workgroups = (long)a.problems * p.parts * (shared ? 1 : a.group);
  const bool e4m3 = format == A2ATS_E4M3;
  if (kv_dtype == A2ATS_BF16) {
    if (e4m3) launch_heads<uint16_t, true>(a, shared, workgroups, stream);
    else launch_heads<uint16_t, false>(a, shared, workgroups, stream);
  } else {
    if (e4m3) launch_heads<float, true>(a, shared, workgroups, stream);
    else launch_heads<float, false>(a, shared, workgroups, stream);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.parts == 1) return e;
  if (kv_dtype == A2ATS_BF16)
    hipLaunchKernelGGL((attn_kv8_merge_kernel<uint16_t>), dim3(d.batch * d.n_q_heads), dim3(kD), 0, stream, (const float*)ws,
                       (uint16_t*)out, p.parts);
  else
    hipLaunchKernelGGL((attn_kv8_merge_kernel<float>), dim3(d.batch * d.n_q_heads), dim3(kD), 0, stream, (const float*)ws,
                       (float*)out, p.parts);
  return hipGetLastError();
}

}  // namespace a2ats
