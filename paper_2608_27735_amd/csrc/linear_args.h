// linear_args.h -- arguments of the linear layer's kernels, and their launchers by
// element type.
#pragma once

#include "gated_ffn_args.h"

namespace abcd {

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
// dz = dy slope, of n rows
struct LinearSlope {
  const void* dy;
  const void* slope;
  void* dz;
  int64_t n, o, lddy, ldslope, lddz;
};

#define ABCD_LINEAR_DECLARE(NAME)                               \
  int32_t linear_out_##NAME(const LinearOut&, hipStream_t);     \
  int32_t linear_few_##NAME(const LinearOut&, hipStream_t);     \
  int32_t linear_dz_##NAME(const LinearDz&, hipStream_t);       \
  int32_t linear_dx_##NAME(const LinearDx&, hipStream_t);       \
  int32_t linear_slope_##NAME(const LinearSlope&, hipStream_t);
ABCD_LINEAR_DECLARE(f32)
ABCD_LINEAR_DECLARE(f16)
ABCD_LINEAR_DECLARE(bf16)
#undef ABCD_LINEAR_DECLARE

}  // namespace abcd
