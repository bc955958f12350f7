// linear_args.h -- arguments of the linear layer's kernels, and their launchers by
// element type.
#pragma once

#include "gated_ffn_args.h"

namespace abcd {

// What a forward keeps of act's derivative: in 16-bit types float16 whatever these are, as it
// lies between -0.13 and 1.13 (below 2^-14 with fewer digits): kept in bfloat16 its rounding
// would be as large as dz's.
template <typename T>
using SlopeOf = std::conditional_t<sizeof(T) == 4, float, _Float16>;

// y = res + act(x w' + bias); slope: act's derivative, [n][ldslope], columns past o zeros.
struct LinearOut {
  Side x, w;
  const void* bias;
  const void* res;
  void* y;
  void* slope;  // NULL: not kept
  int64_t i, o, ldr, ldy, ldslope;
  int act;
  Tiling t;
};
// dz = dy act'(x w' + bias): [n][lddz], columns past o zeros.
struct LinearDz {
  Side x, w;
  const void* bias;
  const void* dy;
  void* dz;
  int64_t i, o, lddy, lddz;
  int act;
  Tiling t;
};
// dx = dz w
struct LinearDx {
  Side dz, w;
  void* dx;
  int64_t o, i, lddx;
  Tiling t;
};
// dz = dy slope, of n rows; part: [parts][o], the sums of dz's rows before it is rounded
// (NULL: not wanted)
struct LinearSlope {
  const void* dy;
  const void* slope;
  void* dz;
  float* part;
  int64_t n, o, lddy, ldslope, lddz;
  int lanes;  // threads along a row, 8 columns each
};

// Narrow rows, 16-bit types.
struct LinearNarrow {
  const void *x, *w, *bias, *res;
  void *y, *slope;
  int64_t n, i, o, ldx, ldr, ldy, ldslope;
  int act;
};
// x, or q and e; part: [workgroups][o i + o], the sums of dw and db, NULL: neither is wanted
struct LinearNarrowBwd {
  const void* x;
  const int8_t* q;
  const uint8_t* e;
  const void *dy, *slope, *w, *bias;
  void* dx;
  float* part;
  int64_t n, i, o, ldx, lddy, ldslope, lddx;
  int act;
};
inline bool narrow_layer(int64_t i, int64_t o) { return i <= 256 && o <= 256 && (i <= 128 || o <= 128); }
inline bool narrow_layer_bwd(int64_t i, int64_t o) { return i <= 128 && o <= 128 && (i <= 64 || o <= 64); }
int32_t linear_narrow_f16(const LinearNarrow&, int64_t blocks, hipStream_t);
int32_t linear_narrow_bf16(const LinearNarrow&, int64_t blocks, hipStream_t);
int32_t linear_narrow_bwd_f16(const LinearNarrowBwd&, int64_t blocks, hipStream_t);
int32_t linear_narrow_bwd_bf16(const LinearNarrowBwd&, int64_t blocks, hipStream_t);

#define ABCD_LINEAR_DECLARE(NAME)                               \
  int32_t linear_out_##NAME(const LinearOut&, hipStream_t);     \
  int32_t linear_few_##NAME(const LinearOut&, hipStream_t);     \
  int32_t linear_dz_##NAME(const LinearDz&, hipStream_t);       \
  int32_t linear_dx_##NAME(const LinearDx&, hipStream_t);       \
  int32_t linear_dw_##NAME(const FfnDWeight&, hipStream_t);     \
  int32_t linear_slope_##NAME(const LinearSlope&, int64_t parts, hipStream_t);
ABCD_LINEAR_DECLARE(f32)
ABCD_LINEAR_DECLARE(f16)
ABCD_LINEAR_DECLARE(bf16)
#undef ABCD_LINEAR_DECLARE

}  // namespace abcd
