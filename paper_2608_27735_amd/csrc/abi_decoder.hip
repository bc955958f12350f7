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

}  // extern "C"
