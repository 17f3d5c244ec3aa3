// A key/value cache held in 4 bits (a2ats_kv4): where its rows are, shared by the append, the read and the attention over it.
//
// A row is 128 bytes, one line of memory: 64 of the key's codes (byte i: dimensions 2 i and 2 i + 1, the first in the low half)
// and 64 of the value's (byte 4 n + g: dimensions 32 g + 2 n and 32 g + 2 n + 1, so that the four bytes from 4 n on are two
// dimensions of each of the four groups).  Beside it 8 bytes of scales, exponents + 127: the key's four groups of 32
// dimensions, then the value's.  255 stands for NaN.
#pragma once
#include "kv_blocks.hpp"

namespace a2ats {

constexpr int kKv4RowBytes = 128, kKv4Half = 64, kKv4ScaleBytes = 8;

struct Kv4Cache {
  uint8_t* rows;
  uint8_t* scales;
  BlockCache at;   // where blocks are (and the bounds); its own rows are not used
};

// The scale of a byte: a power of two; 0 for the byte 0, infinite for 255.
__device__ __forceinline__ float kv4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

}  // namespace a2ats
