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
// (q + 128) unit - 128 unit is exact, but of the largest exponent, where 128 unit is an
// infinity (kLargest: a type that has it, as float16 does not). That, and what is not finite,
// is found for a wave's lanes together.
template <bool kLargest>
__device__ __forceinline__ Floats<8> unpack_8(uint32_t lo, uint32_t hi, float unit) {
  const uint32_t u[2] = {lo ^ 0x80808080u, hi ^ 0x80808080u};
  const float off = -128.0f * unit;
  Floats<8> v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = fmaf((float)(u[i / 4] >> (8 * (i % 4)) & 255u), unit, off);
  const uint32_t zero = ((u[0] - 0x01010101u) & ~u[0]) | ((u[1] - 0x01010101u) & ~u[1]);  // of a byte 0 the top bit
  if (__builtin_expect(__any((zero & 0x80808080u) != 0 || (kLargest && unit >= 0x1p121f)), 0)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t b = u[i / 4] >> (8 * (i % 4)) & 255u;
      if (kLargest) v[i] = ((float)b - 128.0f) * unit;
      if (b == 0) v[i] = __builtin_nanf("");
    }
  }
  return v;
}

}  // namespace abcd
