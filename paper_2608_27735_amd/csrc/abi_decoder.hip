// abi_decoder.hip -- the extern "C" entry points of the decoder's operators:
// argument validation on the host (before any HIP call) and dispatch.
#include <cmath>

#include "rows.h"

using namespace abcd;

namespace {

int32_t check_rows(int32_t dtype, int64_t n, int64_t d) {
  REQUIRE(dtype == ABCD_F32 || dtype == ABCD_F16 || dtype == ABCD_BF16, "unknown dtype %d", dtype);
  REQUIRE(n >= 0 && n <= ABCD_MAX_GAUSSIANS, "n = %lld out of range", (long long)n);
  REQUIRE(d >= 1 && d <= ABCD_MAX_WIDTH, "width %lld not in [1, %d]", (long long)d, ABCD_MAX_WIDTH);
  return ABCD_OK;
}

// An array of n rows of d elements, ld apart (n = 0: nothing is read of it).
int32_t check_matrix(const char* name, const void* p, int32_t dtype, int64_t n, int64_t d, int64_t ld,
                     bool optional) {
  if (n == 0 || (optional && p == nullptr)) return ABCD_OK;
  REQUIRE(p != nullptr, "%s is NULL", name);
  REQUIRE((reinterpret_cast<uintptr_t>(p) & (type_bytes(dtype) - 1)) == 0, "%s is not aligned to its elements",
          name);
  REQUIRE(ld >= d && ld <= (int64_t(1) << 40), "%s: %lld elements between rows of %lld", name, (long long)ld,
          (long long)d);
  return ABCD_OK;
}

int32_t check_vector(const char* name, const void* p, int32_t dtype) {
  REQUIRE((reinterpret_cast<uintptr_t>(p) & (type_bytes(dtype) - 1)) == 0, "%s is not aligned to its elements",
          name);
  return ABCD_OK;
}

int32_t check_wdtype(int32_t dtype, int32_t wdtype) {
  REQUIRE(wdtype == dtype || wdtype == ABCD_F32, "wdtype %d is neither dtype nor fp32", wdtype);
  return ABCD_OK;
}

int32_t check_workspace(const void* ws, size_t have, size_t need) {
  REQUIRE(ws != nullptr && (reinterpret_cast<uintptr_t>(ws) & 255) == 0,
          "workspace must be non-NULL and 256-byte aligned");
  REQUIRE(have >= need, "workspace of %zu bytes, %zu needed", have, need);
  return ABCD_OK;
}

int32_t check_ffn(const abcd_ffn* f, int64_t n) {
  REQUIRE(f != nullptr, "ffn is NULL");
  TRY_STATUS(check_rows(f->dtype, n, f->d));
  TRY_STATUS(check_rows(f->dtype, n, f->h));
  TRY_STATUS(check_rows(f->dtype, n, f->o));
  REQUIRE(f->act == ABCD_ACT_SILU || f->act == ABCD_ACT_GELU || f->act == ABCD_ACT_RELU, "unknown act %d", f->act);
  REQUIRE(f->p >= 0.0 && f->p <= 1.0, "p must be in [0, 1]");
  return ABCD_OK;
}

int32_t check_ffn_weights(const abcd_ffn& f) {
  REQUIRE(f.w_gate && f.w_up && f.w_down, "a weight is NULL");
  TRY_STATUS(check_vector("w_gate", f.w_gate, f.dtype));
  TRY_STATUS(check_vector("w_up", f.w_up, f.dtype));
  TRY_STATUS(check_vector("w_down", f.w_down, f.dtype));
  TRY_STATUS(check_vector("b_gate", f.b_gate, f.dtype));
  TRY_STATUS(check_vector("b_up", f.b_up, f.dtype));
  return check_vector("b_down", f.b_down, f.dtype);
}

int32_t check_saved(const void* by_gate, const void* by_up, const void* hidden) {
  REQUIRE((by_gate == nullptr) == (by_up == nullptr) && (by_up == nullptr) == (hidden == nullptr),
          "by_gate, by_up and hidden go together");
  for (const void* p : {by_gate, by_up, hidden})
    REQUIRE((reinterpret_cast<uintptr_t>(p) & 15) == 0, "by_gate, by_up and hidden must be 16-byte aligned");
  return ABCD_OK;
}

int32_t check_index(int32_t bits, const void* index, int64_t n) {
  REQUIRE(bits == 32 || bits == 64, "indexes of %d bits", bits);
  if (n == 0) return ABCD_OK;
  REQUIRE(index != nullptr, "index is NULL");
  REQUIRE((reinterpret_cast<uintptr_t>(index) & (bits / 8 - 1)) == 0, "index is not aligned to its elements");
  return ABCD_OK;
}

int32_t check_table_rows(int64_t n, int64_t m) {
  REQUIRE(n >= 0 && n <= ABCD_MAX_GAUSSIANS, "n = %lld out of range", (long long)n);
  REQUIRE(m >= 1 && m <= ABCD_MAX_GAUSSIANS, "a table of %lld rows", (long long)m);
  return ABCD_OK;
}

int32_t check_ints(const char* name, const void* p, size_t align, int64_t n) {
  if (n == 0) return ABCD_OK;
  REQUIRE(p != nullptr && (reinterpret_cast<uintptr_t>(p) & (align - 1)) == 0, "%s must be non-NULL and %zu-byte aligned",
          name, align);
  return ABCD_OK;
}

int32_t check_joint(const abcd_joint* joint, int64_t n) {
  REQUIRE(joint != nullptr, "joint is NULL");
  const abcd_joint& j = *joint;
  TRY_STATUS(check_rows(j.dtype, n, j.d));
  TRY_STATUS(check_wdtype(j.dtype, j.wdtype));
  for (int32_t k : {j.post, j.pre})
    REQUIRE(k == ABCD_NORM_NONE || k == ABCD_NORM_LAYER || k == ABCD_NORM_RMS, "unknown norm %d", k);
  REQUIRE(j.gate == ABCD_GATE_NONE || j.gate == ABCD_GATE_ROW || j.gate == ABCD_GATE_ELEMENT, "unknown gate %d", j.gate);
  REQUIRE((j.post != ABCD_NORM_NONE || !j.post_weight) && (j.post == ABCD_NORM_LAYER || !j.post_bias) &&
              (j.pre != ABCD_NORM_NONE || !j.pre_weight) && (j.pre == ABCD_NORM_LAYER || !j.pre_bias),
          "a parameter of no norm");
  for (const void* p : {j.post_weight, j.post_bias, j.pre_weight, j.pre_bias, j.scale})
    TRY_STATUS(check_vector("a parameter", p, j.wdtype));
  REQUIRE(j.eps >= 0.0f && std::isfinite(j.eps), "eps must be finite and >= 0");
  return ABCD_OK;
}

int32_t check_layer(const abcd_layer* layer, int64_t n) {
  REQUIRE(layer != nullptr, "layer is NULL");
  const abcd_layer& l = *layer;
  TRY_STATUS(check_rows(l.dtype, n, l.i));
  TRY_STATUS(check_rows(l.dtype, n, l.o));
  REQUIRE(l.act >= ABCD_ACT_SILU && l.act <= ABCD_ACT_NONE, "unknown act %d", l.act);
  return ABCD_OK;
}

int32_t check_layer_weights(const abcd_layer& l, const void* slope) {
  REQUIRE(l.w != nullptr, "w is NULL");
  TRY_STATUS(check_vector("w", l.w, l.dtype));
  TRY_STATUS(check_vector("b", l.b, l.dtype));
  REQUIRE((reinterpret_cast<uintptr_t>(slope) & 15) == 0, "slope must be 16-byte aligned");
  return ABCD_OK;
}

int32_t check_gate(const char* name, const abcd_joint& j, const void* gate, int64_t n, int64_t ldg, bool optional) {
  if (j.gate == ABCD_GATE_NONE) {
    REQUIRE(gate == nullptr, "%s without a gate", name);
    return ABCD_OK;
  }
  return check_matrix(name, gate, j.dtype, n, j.gate == ABCD_GATE_ROW ? 1 : j.d, ldg, optional);
}

}  // namespace

extern "C" {

int32_t abcd_gated_ffn_keeps(const abcd_ffn* ffn, int64_t n, int32_t* keeps) {
  TRY_STATUS(check_ffn(ffn, n));
  REQUIRE(keeps != nullptr, "keeps is NULL");
  *keeps = gated_ffn_keeps(*ffn, n) ? 1 : 0;
  return ABCD_OK;
}

int32_t abcd_gated_ffn_workspace_size(const abcd_ffn* ffn, int64_t n, int32_t saved, size_t* bytes) {
  TRY_STATUS(check_ffn(ffn, n));
  REQUIRE(bytes != nullptr, "bytes is NULL");
  *bytes = gated_ffn_workspace_bytes(*ffn, n, saved != 0, false);
  return ABCD_OK;
}

int32_t abcd_gated_ffn_bwd_workspace_size(const abcd_ffn* ffn, int64_t n, int32_t saved, size_t* bytes) {
  TRY_STATUS(check_ffn(ffn, n));
  REQUIRE(bytes != nullptr, "bytes is NULL");
  *bytes = gated_ffn_workspace_bytes(*ffn, n, saved != 0, true);
  return ABCD_OK;
}

int32_t abcd_gated_ffn(const abcd_ffn* ffn, int64_t n, const void* x, int64_t ldx, const void* residual, int64_t ldr,
                       void* y, int64_t ldy, void* by_gate, void* by_up, void* hidden, void* workspace, size_t ws_bytes,
                       hipStream_t stream) {
  TRY_STATUS(check_ffn(ffn, n));
  const abcd_ffn& f = *ffn;
  TRY_STATUS(check_ffn_weights(f));
  TRY_STATUS(check_matrix("x", x, f.dtype, n, f.d, ldx, false));
  TRY_STATUS(check_matrix("residual", residual, f.dtype, n, f.o, ldr, true));
  TRY_STATUS(check_matrix("y", y, f.dtype, n, f.o, ldy, false));
  TRY_STATUS(check_saved(by_gate, by_up, hidden));
  if (n > 0)
    TRY_STATUS(check_workspace(workspace, ws_bytes, gated_ffn_workspace_bytes(f, n, hidden != nullptr, false)));
  return launch_gated_ffn(f, n, x, ldx, residual, ldr, y, ldy, by_gate, by_up, hidden, workspace, stream);
}

int32_t abcd_gated_ffn_bwd(const abcd_ffn* ffn, int64_t n, const void* dy, int64_t lddy, const void* x, int64_t ldx,
                           const void* by_gate, const void* by_up, const void* hidden, void* dx, int64_t lddx,
                           void* dw_gate, void* dw_up, void* dw_down, void* db_gate, void* db_up, void* db_down,
                           void* workspace, size_t ws_bytes, hipStream_t stream) {
  TRY_STATUS(check_ffn(ffn, n));
  const abcd_ffn& f = *ffn;
  TRY_STATUS(check_ffn_weights(f));
  TRY_STATUS(check_matrix("dy", dy, f.dtype, n, f.o, lddy, false));
  TRY_STATUS(check_matrix("x", x, f.dtype, n, f.d, ldx, false));
  TRY_STATUS(check_matrix("dx", dx, f.dtype, n, f.d, lddx, true));
  TRY_STATUS(check_saved(by_gate, by_up, hidden));
  for (const void* g : {dw_gate, dw_up, dw_down, db_gate, db_up, db_down})
    TRY_STATUS(check_vector("a gradient", g, f.dtype));
  TRY_STATUS(check_workspace(workspace, ws_bytes, gated_ffn_workspace_bytes(f, n, hidden != nullptr, true)));
  return launch_gated_ffn_bwd(f, n, dy, lddy, x, ldx, by_gate, by_up, hidden, dx, lddx, dw_gate, dw_up, dw_down, db_gate,
                              db_up, db_down, workspace, stream);
}

int32_t abcd_layer_norm(int32_t dtype, int64_t n, int64_t d, const void* x, int64_t ldx, int32_t wdtype,
                        const void* weight, const void* bias, float eps, void* y, int64_t ldy, float* mean,
                        float* rstd, hipStream_t stream) {
  TRY_STATUS(check_rows(dtype, n, d));
  TRY_STATUS(check_wdtype(dtype, wdtype));
  TRY_STATUS(check_matrix("x", x, dtype, n, d, ldx, false));
  TRY_STATUS(check_matrix("y", y, dtype, n, d, ldy, false));
  TRY_STATUS(check_vector("weight", weight, wdtype));
  TRY_STATUS(check_vector("bias", bias, wdtype));
  TRY_STATUS(check_vector("mean", mean, ABCD_F32));
  TRY_STATUS(check_vector("rstd", rstd, ABCD_F32));
  REQUIRE(eps >= 0.0f && std::isfinite(eps), "eps must be finite and >= 0");
  return launch_layer_norm(dtype, n, d, x, ldx, wdtype, weight, bias, eps, y, ldy, mean, rstd, stream);
}

int32_t abcd_layer_norm_bwd_workspace_size(int32_t dtype, int64_t n, int64_t d, size_t* bytes) {
  TRY_STATUS(check_rows(dtype, n, d));
  REQUIRE(bytes != nullptr, "bytes is NULL");
  *bytes = layer_norm_bwd_workspace_bytes(dtype, n, d);
  return ABCD_OK;
}

int32_t abcd_layer_norm_bwd(int32_t dtype, int64_t n, int64_t d, const void* dy, int64_t lddy, const void* x,
                            int64_t ldx, const float* mean, const float* rstd, int32_t wdtype, const void* weight,
                            const void* add, int64_t ldadd, void* dx, int64_t lddx, void* dweight, void* dbias,
                            void* workspace, size_t ws_bytes, hipStream_t stream) {
  TRY_STATUS(check_rows(dtype, n, d));
  TRY_STATUS(check_wdtype(dtype, wdtype));
  TRY_STATUS(check_matrix("dy", dy, dtype, n, d, lddy, false));
  TRY_STATUS(check_matrix("x", x, dtype, n, d, ldx, false));
  TRY_STATUS(check_matrix("add", add, dtype, n, d, ldadd, true));
  TRY_STATUS(check_matrix("dx", dx, dtype, n, d, lddx, true));
  REQUIRE(n == 0 || (mean != nullptr && rstd != nullptr), "mean or rstd is NULL");
  TRY_STATUS(check_vector("mean", mean, ABCD_F32));
  TRY_STATUS(check_vector("rstd", rstd, ABCD_F32));
  TRY_STATUS(check_vector("weight", weight, wdtype));
  TRY_STATUS(check_vector("dweight", dweight, wdtype));
  TRY_STATUS(check_vector("dbias", dbias, wdtype));
  if (dweight || dbias)
    TRY_STATUS(check_workspace(workspace, ws_bytes, layer_norm_bwd_workspace_bytes(dtype, n, d)));
  return launch_layer_norm_bwd(dtype, n, d, dy, lddy, x, ldx, mean, rstd, wdtype, weight, add, ldadd, dx, lddx,
                               dweight, dbias, workspace, stream);
}

int32_t abcd_dropout(int32_t dtype, int64_t n, int64_t d, const void* x, int64_t ldx, const void* residual,
                     int64_t ldr, void* y, int64_t ldy, double p, uint64_t seed, uint64_t offset,
                     hipStream_t stream) {
  TRY_STATUS(check_rows(dtype, n, d));
  TRY_STATUS(check_matrix("x", x, dtype, n, d, ldx, false));
  TRY_STATUS(check_matrix("residual", residual, dtype, n, d, ldr, true));
  TRY_STATUS(check_matrix("y", y, dtype, n, d, ldy, false));
  REQUIRE(p >= 0.0 && p <= 1.0, "p must be in [0, 1]");
  return launch_dropout(dtype, n, d, x, ldx, residual, ldr, y, ldy, p, seed, offset, stream);
}

int32_t abcd_embed(int32_t dtype, int64_t n, int64_t m, int64_t d, int32_t tdtype, const void* table, int64_t ldt,
                   int32_t index_bits, const void* index, float scale, void* y, int64_t ldy, hipStream_t stream) {
  TRY_STATUS(check_rows(dtype, n, d));
  TRY_STATUS(check_table_rows(n, m));
  TRY_STATUS(check_wdtype(dtype, tdtype));
  TRY_STATUS(check_matrix("table", table, tdtype, m, d, ldt, false));
  TRY_STATUS(check_index(index_bits, index, n));
  REQUIRE(std::isfinite(scale), "scale must be finite");
  TRY_STATUS(check_matrix("y", y, dtype, n, d, ldy, false));
  return launch_embed(dtype, n, m, d, tdtype, table, ldt, index_bits, index, scale, y, ldy, stream);
}

int32_t abcd_embed_sort_workspace_size(int64_t n, int64_t m, size_t* bytes) {
  TRY_STATUS(check_table_rows(n, m));
  REQUIRE(bytes != nullptr, "bytes is NULL");
  *bytes = embed_sort_workspace_bytes(n, m);
  return ABCD_OK;
}

int32_t abcd_embed_sort(int64_t n, int64_t m, int32_t index_bits, const void* index, int32_t* order, int32_t* rows,
                        int32_t* ranges, void* workspace, size_t ws_bytes, hipStream_t stream) {
  TRY_STATUS(check_table_rows(n, m));
  TRY_STATUS(check_index(index_bits, index, n));
  TRY_STATUS(check_ints("order", order, 4, n));
  TRY_STATUS(check_ints("rows", rows, 4, n));
  TRY_STATUS(check_ints("ranges", ranges, 8, m));
  TRY_STATUS(check_workspace(workspace, ws_bytes, embed_sort_workspace_bytes(n, m)));
  return launch_embed_sort(n, m, index_bits, index, order, rows, ranges, workspace, stream);
}

int32_t abcd_embed_bwd_workspace_size(int64_t n, int64_t d, size_t* bytes) {
  TRY_STATUS(check_rows(ABCD_F32, n, d));
  REQUIRE(bytes != nullptr, "bytes is NULL");
  *bytes = embed_bwd_workspace_bytes(n, d);
  return ABCD_OK;
}

int32_t abcd_embed_bwd(int32_t dtype, int64_t n, int64_t m, int64_t d, const void* dy, int64_t lddy,
                       const int32_t* order, const int32_t* rows, const int32_t* ranges, float scale, int32_t wdtype,
                       void* dtable, int64_t ldt, void* workspace, size_t ws_bytes, hipStream_t stream) {
  TRY_STATUS(check_rows(dtype, n, d));
  TRY_STATUS(check_table_rows(n, m));
  TRY_STATUS(check_matrix("dy", dy, dtype, n, d, lddy, false));
  TRY_STATUS(check_ints("order", order, 4, n));
  TRY_STATUS(check_ints("rows", rows, 4, n));
  TRY_STATUS(check_ints("ranges", ranges, 8, m));
  REQUIRE(std::isfinite(scale), "scale must be finite");
  TRY_STATUS(check_wdtype(dtype, wdtype));
  TRY_STATUS(check_matrix("dtable", dtable, wdtype, m, d, ldt, false));
  TRY_STATUS(check_workspace(workspace, ws_bytes, embed_bwd_workspace_bytes(n, d)));
  return launch_embed_bwd(dtype, n, m, d, dy, lddy, order, rows, ranges, scale, wdtype, dtable, ldt, workspace, stream);
}

int32_t abcd_embed_bwd_few(int32_t dtype, int64_t n, int64_t m, int64_t d, const void* dy, int64_t lddy,
                           int32_t index_bits, const void* index, float scale, int32_t wdtype, void* dtable, int64_t ldt,
                           hipStream_t stream) {
  TRY_STATUS(check_rows(dtype, n, d));
  TRY_STATUS(check_table_rows(n, m));
  REQUIRE(n <= ABCD_EMBED_FEW, "%lld positions, more than %d", (long long)n, ABCD_EMBED_FEW);
  TRY_STATUS(check_matrix("dy", dy, dtype, n, d, lddy, false));
  TRY_STATUS(check_index(index_bits, index, n));
  REQUIRE(std::isfinite(scale), "scale must be finite");
  TRY_STATUS(check_wdtype(dtype, wdtype));
  TRY_STATUS(check_matrix("dtable", dtable, wdtype, m, d, ldt, false));
  return launch_embed_bwd_few(dtype, n, m, d, dy, lddy, index_bits, index, scale, wdtype, dtable, ldt, stream);
}

int32_t abcd_residual_norm(const abcd_joint* joint, int64_t n, const void* f, int64_t ldf, const void* x, int64_t ldx,
                           const void* gate, int64_t ldg, void* y, int64_t ldy, void* z, int64_t ldz, float* post_mean,
                           float* post_rstd, float* pre_mean, float* pre_rstd, hipStream_t stream) {
  TRY_STATUS(check_joint(joint, n));
  const abcd_joint& j = *joint;
  TRY_STATUS(check_matrix("f", f, j.dtype, n, j.d, ldf, false));
  TRY_STATUS(check_matrix("x", x, j.dtype, n, j.d, ldx, false));
  TRY_STATUS(check_gate("gate", j, gate, n, ldg, false));
  TRY_STATUS(check_matrix("y", y, j.dtype, n, j.d, ldy, false));
  if (j.pre == ABCD_NORM_NONE)
    REQUIRE(z == nullptr, "z without a norm");
  else
    TRY_STATUS(check_matrix("z", z, j.dtype, n, j.d, ldz, false));
  for (const float* p : {post_mean, post_rstd, pre_mean, pre_rstd}) TRY_STATUS(check_vector("a statistic", p, ABCD_F32));
  return launch_residual_norm(j, n, f, ldf, x, ldx, gate, ldg, y, ldy, z, ldz,
                              j.post == ABCD_NORM_LAYER ? post_mean : nullptr, post_rstd,
                              j.pre == ABCD_NORM_LAYER ? pre_mean : nullptr, pre_rstd, stream);
}

int32_t abcd_residual_norm_bwd_workspace_size(const abcd_joint* joint, int64_t n, size_t* bytes) {
  TRY_STATUS(check_joint(joint, n));
  REQUIRE(bytes != nullptr, "bytes is NULL");
  *bytes = residual_norm_bwd_workspace_bytes(*joint, n);
  return ABCD_OK;
}

int32_t abcd_residual_norm_bwd(const abcd_joint* joint, int64_t n, const void* dz, int64_t lddz, const void* dy,
                               int64_t lddy, const void* f, int64_t ldf, const void* y, int64_t ldy, const void* gate,
                               int64_t ldg, const float* post_mean, const float* post_rstd, const float* pre_mean,
                               const float* pre_rstd, void* dx, int64_t lddx, void* df, int64_t lddf, void* dgate,
                               int64_t lddg, void* dpost_weight, void* dpost_bias, void* dpre_weight, void* dpre_bias,
                               void* dscale, void* workspace, size_t ws_bytes, hipStream_t stream) {
  TRY_STATUS(check_joint(joint, n));
  const abcd_joint& j = *joint;
  const bool post = j.post != ABCD_NORM_NONE, pre = j.pre != ABCD_NORM_NONE;
  if (pre) {
    TRY_STATUS(check_matrix("dz", dz, j.dtype, n, j.d, lddz, false));
    TRY_STATUS(check_matrix("y", y, j.dtype, n, j.d, ldy, false));
  } else {
    REQUIRE(dz == nullptr, "dz without a norm");
  }
  TRY_STATUS(check_matrix("dy", dy, j.dtype, n, j.d, lddy, pre));
  TRY_STATUS(check_matrix("f", f, j.dtype, n, j.d, ldf, false));
  TRY_STATUS(check_gate("gate", j, gate, n, ldg, false));
  REQUIRE(n == 0 || ((!post || post_rstd) && (!pre || pre_rstd) && (j.post != ABCD_NORM_LAYER || post_mean) &&
                     (j.pre != ABCD_NORM_LAYER || pre_mean)),
          "a statistic is NULL");
  for (const float* p : {post_mean, post_rstd, pre_mean, pre_rstd}) TRY_STATUS(check_vector("a statistic", p, ABCD_F32));
  TRY_STATUS(check_matrix("dx", dx, j.dtype, n, j.d, lddx, true));
  TRY_STATUS(check_matrix("df", df, j.dtype, n, j.d, lddf, true));
  TRY_STATUS(check_gate("dgate", j, dgate, n, lddg, true));
  REQUIRE((post || !dpost_weight) && (j.post == ABCD_NORM_LAYER || !dpost_bias) && (pre || !dpre_weight) &&
              (j.pre == ABCD_NORM_LAYER || !dpre_bias),
          "a gradient of no norm's parameter");
  bool sums = false;
  for (const void* p : {dpost_weight, dpost_bias, dpre_weight, dpre_bias, dscale}) {
    TRY_STATUS(check_vector("a gradient", p, j.wdtype));
    sums = sums || p;
  }
  if (sums) TRY_STATUS(check_workspace(workspace, ws_bytes, residual_norm_bwd_workspace_bytes(j, n)));
  return launch_residual_norm_bwd(j, n, dz, lddz, dy, lddy, f, ldf, y, ldy, gate, ldg, post_mean, post_rstd, pre_mean,
                                  pre_rstd, dx, lddx, df, lddf, dgate, lddg, dpost_weight, dpost_bias, dpre_weight,
                                  dpre_bias, dscale, workspace, stream);
}

int32_t abcd_linear_workspace_size(const abcd_layer* layer, int64_t n, size_t* bytes) {
  TRY_STATUS(check_layer(layer, n));
  REQUIRE(bytes != nullptr, "bytes is NULL");
  *bytes = linear_workspace_bytes(*layer, n, false);
  return ABCD_OK;
}

int32_t abcd_linear_bwd_workspace_size(const abcd_layer* layer, int64_t n, size_t* bytes) {
  TRY_STATUS(check_layer(layer, n));
  REQUIRE(bytes != nullptr, "bytes is NULL");
  *bytes = linear_workspace_bytes(*layer, n, true);
  return ABCD_OK;
}

int32_t abcd_linear(const abcd_layer* layer, int64_t n, const void* x, int64_t ldx, const void* residual, int64_t ldr,
                    void* y, int64_t ldy, void* slope, void* workspace, size_t ws_bytes, hipStream_t stream) {
  TRY_STATUS(check_layer(layer, n));
  const abcd_layer& l = *layer;
  TRY_STATUS(check_layer_weights(l, slope));
  TRY_STATUS(check_matrix("x", x, l.dtype, n, l.i, ldx, false));
  TRY_STATUS(check_matrix("residual", residual, l.dtype, n, l.o, ldr, true));
  TRY_STATUS(check_matrix("y", y, l.dtype, n, l.o, ldy, false));
  const size_t need = linear_workspace_bytes(l, n, false);
  if (n > 0 && need > 0) TRY_STATUS(check_workspace(workspace, ws_bytes, need));
  return launch_linear(l, n, x, ldx, residual, ldr, y, ldy, slope, workspace, stream);
}

int32_t abcd_linear_bwd(const abcd_layer* layer, int64_t n, const void* dy, int64_t lddy, const void* x, int64_t ldx,
                        const int8_t* q, const uint8_t* e, const void* slope, void* dx, int64_t lddx, void* dw, void* db,
                        void* workspace, size_t ws_bytes, hipStream_t stream) {
  TRY_STATUS(check_layer(layer, n));
  const abcd_layer& l = *layer;
  TRY_STATUS(check_layer_weights(l, slope));
  TRY_STATUS(check_matrix("dy", dy, l.dtype, n, l.o, lddy, false));
  REQUIRE((q == nullptr) == (e == nullptr) && (n == 0 || (x == nullptr) != (q == nullptr)), "either x, or q and e");
  if (q)
    TRY_STATUS(check_ints("q", q, 16, n));
  else
    TRY_STATUS(check_matrix("x", x, l.dtype, n, l.i, ldx, false));
  TRY_STATUS(check_matrix("dx", dx, l.dtype, n, l.i, lddx, true));
  TRY_STATUS(check_vector("dw", dw, l.dtype));
  TRY_STATUS(check_vector("db", db, l.dtype));
  const size_t need = linear_workspace_bytes(l, n, true);
  if (need > 0) TRY_STATUS(check_workspace(workspace, ws_bytes, need));
  return launch_linear_bwd(l, n, dy, lddy, x, ldx, q, e, slope, dx, lddx, dw, db, workspace, stream);
}

int32_t abcd_pack8(int32_t dtype, int64_t n, int64_t d, const void* x, int64_t ldx, int8_t* q, uint8_t* e,
                   hipStream_t stream) {
  TRY_STATUS(check_rows(dtype, n, d));
  TRY_STATUS(check_matrix("x", x, dtype, n, d, ldx, false));
  TRY_STATUS(check_ints("q", q, 16, n));
  TRY_STATUS(check_ints("e", e, 1, n));
  return launch_pack8(dtype, n, d, x, ldx, q, e, stream);
}

int32_t abcd_unpack8(int32_t dtype, int64_t n, int64_t d, const int8_t* q, const uint8_t* e, void* y, int64_t ldy,
                     hipStream_t stream) {
  TRY_STATUS(check_rows(dtype, n, d));
  TRY_STATUS(check_ints("q", q, 16, n));
  TRY_STATUS(check_ints("e", e, 1, n));
  TRY_STATUS(check_matrix("y", y, dtype, n, d, ldy, false));
  return launch_unpack8(dtype, n, d, q, e, y, ldy, stream);
}

}  // extern "C"
