// pack8.h -- the numbers of 8-bit checkpoints.
#pragma once

#include "load_frag.h"

namespace abcd {

constexpr int kPackBlock = ABCD_PACK8_BLOCK;  // elements that share an exponent
constexpr int kPackLeast = 7;                 // smallest exponent byte: of 2^-120

inline int64_t pack_blocks(int64_t d) { return (d + kPackBlock - 1) / kPackBlock; }

// 2^(e - 6) of the exponent byte e + 127 (at least kPackLeast).
__device__ __forceinline__ float packed_unit(uint32_t e) { return __uint_as_float((e - 6) << 23); }

// Number i of a word's four.
__device__ __forceinline__ float unpacked(uint32_t word, int i, float unit) {
  const int q = (int)(int8_t)(word >> (8 * i));
  return q == -128 ? __builtin_nanf("") : (float)q * unit;
}

}  // namespace abcd
