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

// Two words' eight. q + 128 is what an unsigned byte's conversion takes, and q unit =
// (q + 128) unit - 128 unit is exact; what is not finite is found for a wave's lanes together.
__device__ __forceinline__ Floats<8> unpack_8(uint32_t lo, uint32_t hi, float unit) {
  const uint32_t u[2] = {lo ^ 0x80808080u, hi ^ 0x80808080u};
  const float off = -128.0f * unit;
  Floats<8> v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = fmaf((float)(u[i / 4] >> (8 * (i % 4)) & 255u), unit, off);
  const uint32_t zero = ((u[0] - 0x01010101u) & ~u[0]) | ((u[1] - 0x01010101u) & ~u[1]);  // of a byte 0 the top bit
  if (__builtin_expect(__any((int)(zero & 0x80808080u)), 0)) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if ((u[i / 4] >> (8 * (i % 4)) & 255u) == 0) v[i] = __builtin_nanf("");
  }
  return v;
}

}  // namespace abcd
