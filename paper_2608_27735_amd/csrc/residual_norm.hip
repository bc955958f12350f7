// residual_norm.hip -- the joint between two blocks: how a call becomes launches
// (residual_norm.h).
#include <algorithm>

#include "gated_ffn_args.h"
#include "residual_norm_args.h"

namespace abcd {
namespace {

// Workgroups of the backward, each with its own column sums: one for every CU; of one or two
// long rows at a time two, where their parameters' LDS has room for that (16,384 x 2,048 in
// bf16 100 against 119 us, 8,192 x 4,096 140 against 150; 65,536 x 1,024 167 against 159, 1M x 64
// in fp32 308 against 292). A single one, which leaves out the second launch, where it takes all
// rows at once: two turns of it cost more than that launch saves (bf16, with parameters, two
// turns against two workgroups and the launch: 4 x 2,048 12.2 against 10.4 us, 2 x 20,000 40 against
// 22, 8 x 1,024 10.1 against 9.9, but 128 x 64 10.1 against 10.4 and 2 x 4,096 8.7 against 9.1).
int64_t joint_blocks(const abcd_joint& j, int64_t n) {
  const int64_t item = (int64_t)type_bytes(j.dtype), nvec = (j.d * item + 15) / 16;
  int64_t rows = 64;  // that a workgroup takes at a time: 512 threads, 8 or more a row
  while (rows > 1 && nvec * rows > 512) rows /= 2;
  const int64_t most = rows <= 2 && nvec <= 512 ? 2 * kCUs : kCUs;
  return n <= rows ? 1 : std::min<int64_t>((n + rows - 1) / rows, most);
}

int64_t joint_pitch(int64_t d) { return (d + 7) & ~int64_t(7); }

JointArgs joint_args(const abcd_joint& j, int64_t n) {
  JointArgs a{};
  a.post_w = j.post_weight;
  a.post_b = j.post_bias;
  a.pre_w = j.pre_weight;
  a.pre_b = j.pre_bias;
  a.scale = j.scale;
  a.n = n;
  a.pitch = joint_pitch(j.d);
  a.d = (int)j.d;
  a.post = j.post;
  a.pre = j.pre;
  a.gate_mode = j.gate;
  a.wf32 = j.wdtype == ABCD_F32 && j.dtype != ABCD_F32;
  a.eps = j.eps;
  a.inv_d = 1.0f / (float)j.d;
  return a;
}

}  // namespace

size_t residual_norm_bwd_workspace_bytes(const abcd_joint& j, int64_t n) {
  return align256((size_t)joint_blocks(j, n) * 4 * joint_pitch(j.d) * sizeof(float));
}

int32_t launch_residual_norm(const abcd_joint& j, int64_t n, const void* f, int64_t ldf, const void* x, int64_t ldx,
                             const void* gate, int64_t ldg, void* y, int64_t ldy, void* z, int64_t ldz, float* post_mean,
                             float* post_rstd, float* pre_mean, float* pre_rstd, hipStream_t stream) {
  if (n == 0) return ABCD_OK;
  JointArgs a = joint_args(j, n);
  a.f = f;
  a.ldf = ldf;
  a.x = x;
  a.ldx = ldx;
  a.gate = gate;
  a.ldg = ldg;
  a.y = y;
  a.ldy = ldy;
  a.z = z;
  a.ldz = ldz;
  a.post_mean = post_mean;
  a.post_rstd = post_rstd;
  a.pre_mean = pre_mean;
  a.pre_rstd = pre_rstd;
  return j.dtype == ABCD_F32   ? residual_norm_f32(a, stream)
         : j.dtype == ABCD_F16 ? residual_norm_f16(a, stream)
                               : residual_norm_bf16(a, stream);
}

int32_t launch_residual_norm_bwd(const abcd_joint& j, int64_t n, const void* dz, int64_t lddz, const void* dy, int64_t lddy,
                                 const void* f, int64_t ldf, const void* y, int64_t ldy, const void* gate, int64_t ldg,
                                 const float* post_mean, const float* post_rstd, const float* pre_mean,
                                 const float* pre_rstd, void* dx, int64_t lddx, void* df, int64_t lddf, void* dgate,
                                 int64_t lddg, void* dpost_weight, void* dpost_bias, void* dpre_weight, void* dpre_bias,
                                 void* dscale, void* workspace, hipStream_t stream) {
  JointArgs a = joint_args(j, n);
  a.dz = dz;
  a.lddz = lddz;
  a.dy = dy;
  a.lddy = lddy;
  a.f = f;
  a.ldf = ldf;
  a.y = const_cast<void*>(y);
  a.ldy = ldy;
  a.gate = gate;
  a.ldg = ldg;
  a.post_mean = const_cast<float*>(post_mean);
  a.post_rstd = const_cast<float*>(post_rstd);
  a.pre_mean = const_cast<float*>(pre_mean);
  a.pre_rstd = const_cast<float*>(pre_rstd);
  a.dx = dx;
  a.lddx = lddx;
  a.df = df;
  a.lddf = lddf;
  a.dgate = dgate;
  a.lddg = lddg;
  a.dpost_w = dpost_weight;
  a.dpost_b = dpost_bias;
  a.dpre_w = dpre_weight;
  a.dpre_b = dpre_bias;
  a.dscale = dscale;
  if (dpost_weight || dpost_bias || dpre_weight || dpre_bias || dscale) a.part = static_cast<float*>(workspace);
  const int64_t blocks = joint_blocks(j, n);
  return j.dtype == ABCD_F32   ? residual_norm_bwd_f32(a, blocks, stream)
         : j.dtype == ABCD_F16 ? residual_norm_bwd_f16(a, blocks, stream)
                               : residual_norm_bwd_bf16(a, blocks, stream);
}

}  // namespace abcd
