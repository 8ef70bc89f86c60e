// C ABI of the layer operators: argument validation on the host, then kernel launches on the caller's stream.  See
// include/bsr_layer_ops.h for the contract of every entry point.
#include <cmath>

#include "layer_ops.h"

namespace bsr {

namespace {

constexpr int64_t kMaxRows = (int64_t(1) << 31) - 1;          // rows and columns are counted in 32 bits by the kernels

bool misaligned(const void *p, size_t a) { return p != nullptr && (uintptr_t)p % a != 0; }

bool known_type(int dtype) { return dtype == BSR_F32 || dtype == BSR_BF16; }

// a matrix of `rows` rows with leading dimension ld
int check_matrix(int64_t rows, int64_t cols, int64_t ld) {
  if (rows < 0 || cols < 0 || ld < cols || rows > kMaxRows || cols > kMaxRows || ld > (int64_t(1) << 40)) return BSR_ERR_SHAPE;
  if ((double)rows * (double)ld * 8.0 > 9.0e18) return BSR_ERR_SHAPE;
  return BSR_OK;
}

int check_workspace(size_t need, const void *ws, size_t ws_bytes) {
  if (need == 0) return BSR_OK;
  if (ws == nullptr || ws_bytes < need) return BSR_ERR_WORKSPACE;
  return misaligned(ws, 16) ? BSR_ERR_ALIGN : BSR_OK;
}

bool magnitude_in_range(float v) { return v >= 0x1p-126f && v <= 0x1p126f; }

#define BSR_REQUIRE(call)              \
  do {                                 \
    const int rc_ = (call);            \
    if (rc_ != BSR_OK) return rc_;     \
  } while (0)

int check_gated(const GatedArgs &a) {
  if (!known_type(a.dtype)) return BSR_ERR_DTYPE;
  if (a.F < 0 || a.F > kMaxRows / 2) return BSR_ERR_SHAPE;
  BSR_REQUIRE(check_matrix(a.D, 2 * a.F, a.ldw));
  if (a.D > BSR_MAX_GATED_WIDTH || 2 * a.F > BSR_MAX_GATED_WIDTH) return BSR_ERR_LIMIT;
  return a.act < BSR_ACT_SILU || a.act > BSR_ACT_RELU ? BSR_ERR_VALUE : BSR_OK;
}

}  // namespace

}  // namespace bsr

using namespace bsr;

extern "C" {

int bsr_layer_norm(const void *X, int dtype, int64_t M, int64_t D, int64_t ldx, const void *gamma, const void *beta, int param_dtype,
                   float eps, void *Y, int64_t ldy, float *stats, void *stream) {
  if (!known_type(dtype) || !known_type(param_dtype)) return BSR_ERR_DTYPE;
  BSR_REQUIRE(check_matrix(M, D, ldx));
  BSR_REQUIRE(check_matrix(M, D, ldy));
  if (Y == X && Y != nullptr && ldy != ldx) return BSR_ERR_SHAPE;
  if (!magnitude_in_range(eps)) return BSR_ERR_VALUE;
  if (M == 0 || D == 0) return BSR_OK;
  if (X == nullptr || Y == nullptr) return BSR_ERR_NULL;
  const int e = elem_bytes(dtype), pe = elem_bytes(param_dtype);
  if (misaligned(X, e) || misaligned(Y, e) || misaligned(gamma, pe) || misaligned(beta, pe) || misaligned(stats, 4)) return BSR_ERR_ALIGN;
  return launch_layer_norm(X, dtype, M, D, ldx, gamma, beta, param_dtype, eps, Y, ldy, stats, static_cast<hipStream_t>(stream));
}

size_t bsr_layer_norm_grad_workspace_bytes(int64_t M, int64_t D) {
  if (check_matrix(M, D, D) != BSR_OK) return 0;
  return M == 0 || D == 0 ? 0 : layer_norm_grad_ws_bytes(M, D);
}

int bsr_layer_norm_grad(const void *X, int dtype, int64_t M, int64_t D, int64_t ldx, const void *gamma, int param_dtype,
                        const float *stats, const void *dY, int64_t lddy, void *dX, int64_t lddx, float *dgamma, float *dbeta,
                        int accumulate, void *ws, size_t ws_bytes, void *stream) {
  if (!known_type(dtype) || !known_type(param_dtype)) return BSR_ERR_DTYPE;
  BSR_REQUIRE(check_matrix(M, D, ldx));
  BSR_REQUIRE(check_matrix(M, D, lddy));
  BSR_REQUIRE(check_matrix(M, D, lddx));
  if (dX != nullptr && ((dX == dY && lddx != lddy) || (dX == X && lddx != ldx))) return BSR_ERR_SHAPE;
  if (D == 0) return BSR_OK;
  if (M > 0 && (X == nullptr || stats == nullptr || dY == nullptr || dX == nullptr)) return BSR_ERR_NULL;
  const int e = elem_bytes(dtype);
  if (misaligned(X, e) || misaligned(dY, e) || misaligned(dX, e) || misaligned(gamma, elem_bytes(param_dtype)) || misaligned(stats, 4) ||
      misaligned(dgamma, 4) || misaligned(dbeta, 4))
    return BSR_ERR_ALIGN;
  if (dgamma != nullptr || dbeta != nullptr) BSR_REQUIRE(check_workspace(bsr_layer_norm_grad_workspace_bytes(M, D), ws, ws_bytes));
  return launch_layer_norm_grad(X, dtype, M, D, ldx, gamma, param_dtype, stats, dY, lddy, dX, lddx, dgamma, dbeta, accumulate, ws,
                                static_cast<hipStream_t>(stream));
}

size_t bsr_gated_ff_workspace_bytes(const void *X, int dtype, int64_t M, int64_t D, int64_t ldx, const void *W, int64_t F, int64_t ldw) {
  const GatedArgs a = {X, dtype, M, D, ldx, W, F, ldw, 0};
  if (check_gated(a) != BSR_OK || check_matrix(M, D, ldx) != BSR_OK || check_matrix(M, 2 * F, 2 * F) != BSR_OK) return 0;
  return M == 0 || F == 0 ? 0 : gated_ff_ws_bytes(a);
}

int bsr_gated_ff(const void *X, int dtype, int64_t M, int64_t D, int64_t ldx, const void *W, int64_t F, int64_t ldw, int act, void *H,
                 int64_t ldh, void *GU, int64_t ldgu, void *ws, size_t ws_bytes, void *stream) {
  const GatedArgs a = {X, dtype, M, D, ldx, W, F, ldw, act};
  BSR_REQUIRE(check_gated(a));
  BSR_REQUIRE(check_matrix(M, D, ldx));
  BSR_REQUIRE(check_matrix(M, F, ldh));
  BSR_REQUIRE(check_matrix(M, 2 * F, GU != nullptr ? ldgu : 2 * F));
  if (M == 0 || F == 0) return BSR_OK;
  if (H == nullptr || (D > 0 && (X == nullptr || W == nullptr))) return BSR_ERR_NULL;
  const int e = elem_bytes(dtype);
  if (misaligned(X, e) || misaligned(W, e) || misaligned(H, e) || misaligned(GU, e)) return BSR_ERR_ALIGN;
  BSR_REQUIRE(check_workspace(gated_ff_ws_bytes(a), ws, ws_bytes));
  return launch_gated_ff(a, H, ldh, GU, ldgu, ws, static_cast<hipStream_t>(stream));
}

size_t bsr_gated_ff_grad_workspace_bytes(const void *dGU, int dtype, int64_t M, int64_t F, int64_t lddgu, const void *W, int64_t D,
                                         int64_t ldw) {
  const GatedArgs a = {nullptr, dtype, M, D, D, W, F, ldw, 0};
  if (check_gated(a) != BSR_OK || check_matrix(M, D, D) != BSR_OK || check_matrix(M, 2 * F, lddgu) != BSR_OK) return 0;
  return M == 0 || D == 0 ? 0 : gated_ff_grad_ws_bytes(a, dGU, lddgu);
}

int bsr_gated_ff_grad(const void *GU, int dtype, int64_t M, int64_t F, int64_t ldgu, const void *dH, int64_t lddh, int act,
                      const void *W, int64_t D, int64_t ldw, void *dGU, int64_t lddgu, void *dX, int64_t lddx, void *ws, size_t ws_bytes,
                      void *stream) {
  const GatedArgs a = {nullptr, dtype, M, D, D, W, F, ldw, act};
  if (dX == nullptr) {                               // W has no part in it
    if (!known_type(dtype)) return BSR_ERR_DTYPE;
    if (F < 0 || F > kMaxRows / 2) return BSR_ERR_SHAPE;
    if (act < BSR_ACT_SILU || act > BSR_ACT_RELU) return BSR_ERR_VALUE;
  } else {
    BSR_REQUIRE(check_gated(a));
    BSR_REQUIRE(check_matrix(M, D, lddx));
  }
  BSR_REQUIRE(check_matrix(M, 2 * F, ldgu));
  BSR_REQUIRE(check_matrix(M, F, lddh));
  BSR_REQUIRE(check_matrix(M, 2 * F, lddgu));
  if (dGU == GU && dGU != nullptr && lddgu != ldgu) return BSR_ERR_SHAPE;
  if (M == 0) return BSR_OK;
  if (F > 0 && (GU == nullptr || dH == nullptr || dGU == nullptr || (dX != nullptr && D > 0 && W == nullptr))) return BSR_ERR_NULL;
  const int e = elem_bytes(dtype);
  if (misaligned(GU, e) || misaligned(dH, e) || misaligned(dGU, e) || misaligned(dX, e) || (dX != nullptr && misaligned(W, e)))
    return BSR_ERR_ALIGN;
  if (dX != nullptr && D > 0) BSR_REQUIRE(check_workspace(gated_ff_grad_ws_bytes(a, dGU, lddgu), ws, ws_bytes));
  return launch_gated_ff_grad(a, GU, ldgu, dH, lddh, dGU, lddgu, dX, lddx, ws, static_cast<hipStream_t>(stream));
}

int64_t bsr_adamw_blocks(int64_t n) { return n < 0 ? -1 : ceil_div(n, (int64_t)kMomentBlock); }

int bsr_adamw_batched(const bsr_adamw_item *items, int n_items, int param_dtype, int grad_dtype, int moments,
                      const bsr_adamw_options *options, void *stream) {
  if (!known_type(param_dtype) || !known_type(grad_dtype) || (moments != BSR_MOMENTS_F32 && moments != BSR_MOMENTS_8BIT))
    return BSR_ERR_DTYPE;
  if (n_items < 0) return BSR_ERR_SHAPE;
  if (options == nullptr || (n_items > 0 && items == nullptr)) return BSR_ERR_NULL;
  const bsr_adamw_options &o = *options;
  const bool betas = o.beta1 >= 0.0 && o.beta1 < 1.0 && o.beta2 >= 0.0 && o.beta2 < 1.0;
  if (!std::isfinite((float)o.lr) || !std::isfinite((float)o.grad_scale) || !betas || !magnitude_in_range((float)o.eps) || o.step < 1)
    return BSR_ERR_VALUE;
  if (misaligned(o.lr_device, 4) || misaligned(o.grad_scale_device, 4) || misaligned(o.step_device, 8)) return BSR_ERR_ALIGN;
  const bool small = moments == BSR_MOMENTS_8BIT;
  for (int i = 0; i < n_items; ++i) {
    const bsr_adamw_item &x = items[i];
    if (x.n < 0 || x.n > (int64_t(1) << 40)) return BSR_ERR_SHAPE;
    if (!std::isfinite(x.weight_decay)) return BSR_ERR_VALUE;
    if (x.n == 0) continue;
    if (small && x.scales_stride < bsr_adamw_blocks(x.n)) return BSR_ERR_SHAPE;
    if (x.param == nullptr || x.grad == nullptr || x.m == nullptr || x.v == nullptr || (small && x.scales == nullptr)) return BSR_ERR_NULL;
    if (misaligned(x.param, elem_bytes(param_dtype)) || misaligned(x.grad, elem_bytes(grad_dtype)) || misaligned(x.copy, 2) ||
        (!small && (misaligned(x.m, 4) || misaligned(x.v, 4))))
      return BSR_ERR_ALIGN;
  }
  return launch_adamw(items, n_items, param_dtype, grad_dtype, moments, o, static_cast<hipStream_t>(stream));
}

int bsr_adamw_state_values(const uint8_t *codes, const uint8_t *scales, int64_t n, int which, void *out, int dtype, void *stream) {
  if (!known_type(dtype)) return BSR_ERR_DTYPE;
  if (n < 0 || n > (int64_t(1) << 40)) return BSR_ERR_SHAPE;
  if (which != 0 && which != 1) return BSR_ERR_VALUE;
  if (n == 0) return BSR_OK;
  if (codes == nullptr || scales == nullptr || out == nullptr) return BSR_ERR_NULL;
  if (misaligned(out, elem_bytes(dtype))) return BSR_ERR_ALIGN;
  return launch_adamw_state_values(codes, scales, n, which, out, dtype, static_cast<hipStream_t>(stream));
}

}  // extern "C"
