// residual_norm_args.h -- arguments of the joint's kernels, and their launchers by
// element type.
#pragma once

#include "rows.h"

namespace abcd {

struct JointArgs {
  const void *f, *x, *gate;
  const void *post_w, *post_b, *pre_w, *pre_b, *scale;  // each may be NULL
  void *y, *z;  // the backward reads y and takes no z
  float *post_mean, *post_rstd, *pre_mean, *pre_rstd;
  const void *dz, *dy;
  void *dx, *df, *dgate;  // each may be NULL, and so may the parameters' gradients
  void *dpost_w, *dpost_b, *dpre_w, *dpre_b, *dscale;
  float* part;  // [workgroups][4][pitch]: S1, S0, dwpre, dbpre; NULL: none is wanted
  int64_t ldf, ldx, ldg, ldy, ldz, lddz, lddy, lddx, lddf, lddg, n, pitch;
  int d, post, pre, gate_mode;  // gate_mode: 0 none, 1 one number a row, 2 one an element
  int wf32;                     // the parameters are fp32, the rows not
  float eps, inv_d;
};

#define ABCD_JOINT_DECLARE(NAME)                         \
  int32_t residual_norm_##NAME(const JointArgs&, hipStream_t); \
  int32_t residual_norm_bwd_##NAME(const JointArgs&, int64_t blocks, hipStream_t);
ABCD_JOINT_DECLARE(f32)
ABCD_JOINT_DECLARE(f16)
ABCD_JOINT_DECLARE(bf16)
#undef ABCD_JOINT_DECLARE

}  // namespace abcd
