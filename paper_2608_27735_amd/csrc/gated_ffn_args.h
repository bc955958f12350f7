// gated_ffn_args.h -- arguments of the gated feed-forward block's products, and
// their launchers by element type.
#pragma once

#include "rows.h"

namespace abcd {

// One side of a product. Aligned for 16-byte loads: p and ld * sizeof(T) are
// multiples of 16, 256 rows are less than 2^31 bytes, and, contracted along, the
// elements between the contraction's end and the next multiple of 16 bytes are zeros.
struct Side {
  const void* p[2];  // the second where there are two segments or two halves
  int64_t ld;
  int64_t len;  // of the index that is not contracted (of each half)
};

// How a product is dealt out: tiles, and (with few of them) parts of the contraction
// of `steps` steps each, whose sums go to part: [splits][halves][rows][columns up to a
// multiple of 8].
struct Tiling {
  float* part;
  int tiles_x, tiles_w, splits, steps;
};

// hidden and its derivatives by gate and up: [n][ldh], columns [h, ldh) zero;
// by_gate NULL: only hidden
struct FfnIn {
  Side x, w;
  const void* bg;
  const void* bu;
  void* hidden;
  void* by_gate;
  void* by_up;
  int64_t d, h, ldh;
  int act;
  Tiling t;
};
struct FfnOut {
  Side hidden, w;
  const void* bias;
  const void* res;
  void* y;
  int64_t h, o, ldr, ldy;
  DropKey key;
  Tiling t;
};
// dgate and dup may be by_gate and by_up themselves
struct FfnDHidden {
  Side dz, w;
  const void* by_gate;
  const void* by_up;
  void* dgate;
  void* dup;
  int64_t o, h, ldh;
  float scale;  // of dz
  Tiling t;
};
struct FfnDX {
  Side dgu, w;
  void* dx;
  int64_t h, d, lddx;
  Tiling t;
};
// The weights' gradients, out = scale X' W over n rows each, their tiles one after the
// other. The first `whole` of these take a workgroup each, the others one for each of
// `splits` parts of the rows, whose sums go to part: [tiles - whole][splits][tile].
struct FfnDWeight {
  struct One {
    const void* x;
    const void* w;
    void* out;
    int64_t ldx, rows, ldw, cols;
    float scale;
    int tiles_x, tiles_w, first;
  } one[3];
  float* part;
  int64_t n;
  int count, tiles, whole, splits, steps;
};

// Workgroups that run at once with tiles of 256 x 256, one a CU, and of 128 x 128.
constexpr int kCUs = 256, kBigSlots = kCUs, kSmallSlots = 2 * kCUs;

// Floats of the parts that a product of rows x cols (of `halves` of them) over
// `steps` steps writes, 0 if its contraction is not split: it is where its tiles of
// 128 x 128 leave half of the workgroups that fit idle, into at least four steps each,
// and from 8 steps on in fp32, which take 1.9 us each, and 12 in 16-bit types, whose 1 us
// pays for the second launch later (forward and backward, bf16, 1,000 x 512 x 2,816 x 512:
// 99 us, from 8 on 109; fp32, 3,000 x 64 x 128 x 64: 76, from 12 on 80).
inline int64_t product_tiles(int64_t rows, int64_t cols, int halves) {
  return (rows + 127) / 128 * ((halves * cols + 127) / 128);
}
inline int product_splits(size_t item, int64_t rows, int64_t cols, int halves, int64_t steps) {
  const int64_t tiles = product_tiles(rows, cols, halves);
  if (tiles == 0 || 2 * tiles > kSmallSlots || steps < (item == 2 ? 12 : 8)) return 1;
  int64_t s = kSmallSlots / tiles;
  s = s < steps / 4 ? s : steps / 4;
  return (int)(s < 32 ? s : 32);
}
inline size_t product_part(size_t item, int64_t rows, int64_t cols, int halves, int64_t steps) {
  const int s = product_splits(item, rows, cols, halves, steps);
  return s == 1 ? 0 : (size_t)s * halves * rows * ((cols + 7) & ~int64_t(7));
}

// Into how many parts the rows of a tile of the weights' gradients may be split: of four
// steps each, and from 16 on, as adding them up is a launch (fp32, 3,000 x 64 x 128 x 64:
// 15 and 7 us, of 512 rows each 37 and 6).
inline int64_t dweight_splits(int64_t steps) { return steps < 16 ? 1 : steps / 4; }

// The narrow block. Which of the forward's compiled shapes holds it, 0 if none: with
// its weights in 48, 144, 120 or 144 KB of LDS.
inline int narrow_shape(int64_t d, int64_t h, int64_t o) {
  if (d <= 64 && o <= 64 && h <= 384) return h <= 128 ? 1 : 2;
  if (d <= 128 && o <= 128 && h <= 192) return o <= 64 ? 3 : 4;
  return 0;
}
struct FfnNarrow {
  const void *x, *w_gate, *w_up, *w_down, *b_gate, *b_up, *b_down;
  const void* res;
  void* y;
  int64_t n, d, h, o, ldx, ldr, ldy;
  DropKey key;
  int act;
};
// The backward of columns first .. first + h - 1 of an h of ldd (whose pointers are moved
// to them; ldd is also w_down's row stride). part: [workgroups][narrow_groups][sums], the
// sums laid out as dWg, dWu, dWd, dbg, dbu, dbd of all of h. dx_part: dx so far, rows of
// ldp; the last columns' launch writes dx.
struct FfnNarrowBwd {
  const void *x, *dy, *w_gate, *w_up, *w_down, *b_gate, *b_up;
  void* dx;  // may be NULL
  float *part, *dx_part;
  int64_t n, d, h, o, ldd, first, ldx, lddy, lddx, ldp, sums;
  bool last;
  DropKey key;
  float scale;  // of what the forward kept
  int act;
};
// How many groups of its waves share a block's rows: with up to 64 columns of h half of
// the waves would have none (the backward of 300,000 rows of 64 x 64 x 64 in bf16: 48 us,
// in one group 65).
inline int narrow_groups(int64_t h) { return h <= 64 ? 2 : 1; }
int32_t ffn_narrow_f16(const FfnNarrow&, int64_t blocks, hipStream_t);
int32_t ffn_narrow_bf16(const FfnNarrow&, int64_t blocks, hipStream_t);
int32_t ffn_narrow_bwd_f16(const FfnNarrowBwd&, int64_t blocks, hipStream_t);
int32_t ffn_narrow_bwd_bf16(const FfnNarrowBwd&, int64_t blocks, hipStream_t);

#define ABCD_FFN_DECLARE(NAME)                                 \
  int32_t ffn_in_##NAME(const FfnIn&, hipStream_t);            \
  int32_t ffn_few_in_##NAME(const FfnIn&, hipStream_t);        \
  int32_t ffn_few_out_##NAME(const FfnOut&, hipStream_t);      \
  int32_t ffn_out_##NAME(const FfnOut&, hipStream_t);          \
  int32_t ffn_dhidden_##NAME(const FfnDHidden&, hipStream_t);  \
  int32_t ffn_dx_##NAME(const FfnDX&, hipStream_t);            \
  int32_t ffn_dweight_##NAME(const FfnDWeight&, hipStream_t);
ABCD_FFN_DECLARE(f32)
ABCD_FFN_DECLARE(f16)
ABCD_FFN_DECLARE(bf16)
#undef ABCD_FFN_DECLARE

}  // namespace abcd
