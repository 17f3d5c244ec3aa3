// A key/value cache cut into blocks of tokens (a2ats_kv_blocks): where its parts are, shared by the
// append, the block selection and the attention over it.
#pragma once
#include "common.hpp"

namespace a2ats {

constexpr int kRowBytes = 128;   // a cached row: 128 codes of 8 bits

struct BlockCache {
  uint8_t* k;
  uint8_t* v;
  float* k_scale;
  float* v_scale;
  void* k_tail;
  void* v_tail;
  void* bounds;
  const int32_t* pages;      // nullptr: contiguous
  int64_t blocks_per_seq;    // contiguous: blocks of a sequence's and KV head's rows
  int32_t pages_per_seq;
  int32_t shift;             // a block is 1 << shift tokens
  int32_t page_shift;        // paged: a page is 1 << page_shift blocks
  int32_t n_kv_heads;
};

// The number of block c of (sequence b, KV head kv) in the cache's memory: its rows begin at number << shift, its
// scales are at [number] and its bounds at [number][2][128].  64 bits: a pool may hold more than 2^32 bytes.
__device__ __forceinline__ size_t block_at(const BlockCache& m, int b, int kv, int c) {
  if (m.pages == nullptr) return ((size_t)b * m.n_kv_heads + kv) * (size_t)m.blocks_per_seq + (size_t)c;
  const int page = m.pages[(size_t)b * m.pages_per_seq + (c >> m.page_shift)];
  return (((size_t)page * m.n_kv_heads + kv) << m.page_shift) + (size_t)(c & ((1 << m.page_shift) - 1));
}

// Eight consecutive elements as floats.
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
  x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void widen8(const uint4& v, float (&x)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8(const uint16_t* p, float (&x)[8]) { widen8(*(const uint4*)p, x); }

// Candidate blocks of a sequence: those that hold a candidate token, [sink_end, win_start).
__device__ __forceinline__ void candidate_blocks(const SeqRange& sr, int shift, int& first, int& last) {
  first = sr.sink_end >> shift;
  last = sr.win_start > sr.sink_end ? ((sr.win_start - 1) >> shift) + 1 : first;
}

}  // namespace a2ats
