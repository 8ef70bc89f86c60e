// C ABI of the token operators: argument validation on the host, then kernel launches on the caller's stream.  See
// include/bsr_token_step.h for the contract of every entry point.
#include <cmath>

#include "token_step.h"

namespace bsr {

namespace {

constexpr int64_t kMaxRows = (int64_t(1) << 31) - 1;          // rows, entries and columns are counted in 32 bits by the kernels
constexpr int64_t kMaxWidth = int64_t(1) << 40;

bool misaligned(const void *p, size_t a) { return p != nullptr && (uintptr_t)p % a != 0; }
int index_bytes(int index_type) { return index_type == BSR_I64 ? 8 : 4; }

int check_types(int dtype, int index_type) {
  if (dtype != BSR_F32 && dtype != BSR_BF16) return BSR_ERR_DTYPE;
  if (index_type != BSR_I32 && index_type != BSR_I64) return BSR_ERR_DTYPE;
  return BSR_OK;
}

// a matrix of `rows` rows with leading dimension ld
int check_matrix(int64_t rows, int64_t cols, int64_t ld) {
  if (rows < 0 || cols < 0 || ld < cols || rows > kMaxRows || cols > kMaxWidth || ld > kMaxWidth) return BSR_ERR_SHAPE;
  if ((double)rows * (double)ld * 8.0 > 9.0e18) return BSR_ERR_SHAPE;
  return BSR_OK;
}

// tokens [T] or routing [T x k]
int check_routing(int64_t T, int64_t k, int64_t rows) {
  if (T < 0 || k < 0 || rows < 0 || T > kMaxRows || rows > kMaxRows || (k > 0 && T > kMaxRows / k)) return BSR_ERR_SHAPE;
  return BSR_OK;
}

#define BSR_REQUIRE(call)              \
  do {                                 \
    const int rc_ = (call);            \
    if (rc_ != BSR_OK) return rc_;     \
  } while (0)

int check_distill(const DistillArgs &a) {
  BSR_REQUIRE(check_types(a.dtype, a.index_type));
  if (a.teacher_dtype != BSR_F32 && a.teacher_dtype != BSR_BF16) return BSR_ERR_DTYPE;
  BSR_REQUIRE(check_matrix(a.N, a.V, a.ldz));
  if (a.V > kMaxRows || a.K < 0) return BSR_ERR_SHAPE;
  if (a.K > kMaxTeacher) return BSR_ERR_LIMIT;
  if (!(a.temperature >= 0x1p-60f && a.temperature <= 0x1p60f)) return BSR_ERR_VALUE;
  if (a.N == 0) return BSR_OK;
  if ((a.V > 0 && a.logits == nullptr) || (a.K > 0 && (a.ids == nullptr || a.teacher == nullptr))) return BSR_ERR_NULL;
  if (misaligned(a.logits, elem_bytes(a.dtype)) || misaligned(a.ids, index_bytes(a.index_type)) ||
      misaligned(a.teacher, elem_bytes(a.teacher_dtype)))
    return BSR_ERR_ALIGN;
  return BSR_OK;
}

int check_workspace(size_t need, const void *ws, size_t ws_bytes) {
  if (need == 0) return BSR_OK;
  if (ws == nullptr || ws_bytes < need) return BSR_ERR_WORKSPACE;
  return misaligned(ws, 16) ? BSR_ERR_ALIGN : BSR_OK;
}

// the gradient's matrix, which may be the logits
int check_dlogits(const DistillArgs &a, const void *dlogits, int64_t ldd) {
  BSR_REQUIRE(check_matrix(a.N, a.V, ldd));
  if (dlogits == a.logits && dlogits != nullptr && ldd != a.ldz) return BSR_ERR_SHAPE;
  if (a.N > 0 && a.V > 0 && dlogits == nullptr) return BSR_ERR_NULL;
  return misaligned(dlogits, elem_bytes(a.dtype)) ? BSR_ERR_ALIGN : BSR_OK;
}

}  // namespace

}  // namespace bsr

using namespace bsr;

extern "C" {

int bsr_embedding_lookup(const void *table, int dtype, int64_t V, int64_t D, int64_t ldt, const void *tokens, int index_type,
                         int64_t T, float scale, void *out, int64_t ldo, void *stream) {
  BSR_REQUIRE(check_types(dtype, index_type));
  BSR_REQUIRE(check_matrix(V, D, ldt));
  BSR_REQUIRE(check_matrix(T, D, ldo));
  if (!std::isfinite(scale)) return BSR_ERR_VALUE;
  if (T == 0 || D == 0) return BSR_OK;
  if (tokens == nullptr || out == nullptr || (V > 0 && table == nullptr)) return BSR_ERR_NULL;
  if (misaligned(table, elem_bytes(dtype)) || misaligned(out, elem_bytes(dtype)) || misaligned(tokens, index_bytes(index_type)))
    return BSR_ERR_ALIGN;
  return launch_embedding_lookup(table, dtype, V, D, ldt, tokens, index_type, T, scale, out, ldo, static_cast<hipStream_t>(stream));
}

size_t bsr_embedding_grad_workspace_bytes(int64_t T, int64_t V, int64_t D) {
  if (check_matrix(T, D, D) != BSR_OK || check_matrix(V, D, D) != BSR_OK || V > BSR_MAX_VOCAB) return 0;
  return T == 0 || V == 0 || D == 0 ? 0 : embedding_grad_ws_bytes(T, V, D);
}

int bsr_embedding_grad(const void *tokens, int index_type, int64_t T, const void *dY, int dtype, int64_t D, int64_t lddy,
                       float scale, int64_t V, float *dE, int64_t ldde, int accumulate, void *ws, size_t ws_bytes, void *stream) {
  BSR_REQUIRE(check_types(dtype, index_type));
  BSR_REQUIRE(check_matrix(T, D, lddy));
  BSR_REQUIRE(check_matrix(V, D, ldde));
  if (V > BSR_MAX_VOCAB) return BSR_ERR_SHAPE;
  if (!std::isfinite(scale)) return BSR_ERR_VALUE;
  if (V == 0 || D == 0 || (T == 0 && accumulate)) return BSR_OK;
  if (dE == nullptr || (T > 0 && (tokens == nullptr || dY == nullptr))) return BSR_ERR_NULL;
  if (misaligned(dE, 4) || misaligned(dY, elem_bytes(dtype)) || misaligned(tokens, index_bytes(index_type))) return BSR_ERR_ALIGN;
  BSR_REQUIRE(check_workspace(bsr_embedding_grad_workspace_bytes(T, V, D), ws, ws_bytes));
  return launch_embedding_grad(tokens, index_type, T, dY, dtype, D, lddy, scale, V, dE, ldde, accumulate, ws,
                               static_cast<hipStream_t>(stream));
}

int64_t bsr_expert_capacity(int64_t n, int64_t E, int64_t align) {
  if (n < 0 || E < 1 || align < 1 || n > kMaxRows || align > kMaxRows) return -1;
  const int64_t used = E < n ? E : n;
  if (used > 0 && align - 1 > kMaxRows / used) return -1;
  const int64_t rows = (n + used * (align - 1)) / align * align;
  return rows > kMaxRows ? -1 : rows;
}

size_t bsr_expert_sort_workspace_bytes(int64_t n, int64_t E) {
  if (n < 0 || n > kMaxRows || E < 1 || E > kMaxExperts) return 0;
  return expert_sort_ws_bytes(n, E);
}

int bsr_expert_sort(const void *expert_ids, int index_type, int64_t n, int64_t E, int64_t align, int32_t *offsets, int32_t *counts,
                    int32_t *order, int32_t *slots, void *ws, size_t ws_bytes, void *stream) {
  BSR_REQUIRE(check_types(BSR_F32, index_type));
  const int64_t rows = bsr_expert_capacity(n, E, align);
  if (rows < 0) return BSR_ERR_SHAPE;
  if (E > kMaxExperts) return BSR_ERR_LIMIT;
  if (offsets == nullptr || counts == nullptr || (n > 0 && (expert_ids == nullptr || slots == nullptr)) ||
      (rows > 0 && order == nullptr))
    return BSR_ERR_NULL;
  if (misaligned(expert_ids, index_bytes(index_type)) || misaligned(offsets, 4) || misaligned(counts, 4) || misaligned(order, 4) ||
      misaligned(slots, 4))
    return BSR_ERR_ALIGN;
  BSR_REQUIRE(check_workspace(expert_sort_ws_bytes(n, E), ws, ws_bytes));
  return launch_expert_sort(expert_ids, index_type, n, E, align, offsets, counts, order, rows, slots, ws,
                            static_cast<hipStream_t>(stream));
}

int bsr_expert_gather(const void *X, int dtype, int64_t T, int64_t D, int64_t ldx, const int32_t *slots, int64_t k,
                      const int32_t *order, int64_t rows, void *Xs, int64_t ldxs, void *stream) {
  BSR_REQUIRE(check_types(dtype, BSR_I32));
  BSR_REQUIRE(check_routing(T, k, rows));
  BSR_REQUIRE(check_matrix(T, D, ldx));
  BSR_REQUIRE(check_matrix(rows, D, ldxs));
  if (rows == 0 || D == 0) return BSR_OK;
  if (order == nullptr || Xs == nullptr || (T > 0 && k > 0 && (X == nullptr || slots == nullptr))) return BSR_ERR_NULL;
  if (misaligned(X, elem_bytes(dtype)) || misaligned(Xs, elem_bytes(dtype)) || misaligned(slots, 4) || misaligned(order, 4))
    return BSR_ERR_ALIGN;
  return launch_expert_gather(X, dtype, k > 0 ? T : 0, D, ldx, slots, k, order, rows, Xs, ldxs, static_cast<hipStream_t>(stream));
}

int bsr_expert_combine(const void *Ys, int dtype, int64_t rows, int64_t D, int64_t ldys, const int32_t *slots, int64_t T, int64_t k,
                       const float *weights, void *out, int64_t ldo, void *stream) {
  BSR_REQUIRE(check_types(dtype, BSR_I32));
  BSR_REQUIRE(check_routing(T, k, rows));
  BSR_REQUIRE(check_matrix(rows, D, ldys));
  BSR_REQUIRE(check_matrix(T, D, ldo));
  if (T == 0 || D == 0) return BSR_OK;
  if (out == nullptr || (k > 0 && slots == nullptr) || (rows > 0 && k > 0 && Ys == nullptr)) return BSR_ERR_NULL;
  if (misaligned(Ys, elem_bytes(dtype)) || misaligned(out, elem_bytes(dtype)) || misaligned(slots, 4) || misaligned(weights, 4))
    return BSR_ERR_ALIGN;
  return launch_expert_combine(Ys, dtype, rows, D, ldys, slots, T, k, weights, out, ldo, static_cast<hipStream_t>(stream));
}

int bsr_expert_combine_grad(const void *Ys, int dtype, int64_t rows, int64_t D, int64_t ldys, const int32_t *slots,
                            const int32_t *order, int64_t T, int64_t k, const float *weights, const void *dOut, int64_t lddo,
                            void *dYs, int64_t lddys, float *dweights, void *stream) {
  BSR_REQUIRE(check_types(dtype, BSR_I32));
  BSR_REQUIRE(check_routing(T, k, rows));
  BSR_REQUIRE(check_matrix(rows, D, ldys));
  BSR_REQUIRE(check_matrix(rows, D, lddys));
  BSR_REQUIRE(check_matrix(T, D, lddo));
  const bool entries = T > 0 && k > 0;
  if (!entries && (rows == 0 || D == 0)) return BSR_OK;
  if (entries && (slots == nullptr || weights == nullptr || dweights == nullptr || (D > 0 && dOut == nullptr))) return BSR_ERR_NULL;
  if (rows > 0 && D > 0 && (Ys == nullptr || dYs == nullptr)) return BSR_ERR_NULL;
  if (rows > 0 && order == nullptr) return BSR_ERR_NULL;
  if (misaligned(Ys, elem_bytes(dtype)) || misaligned(dYs, elem_bytes(dtype)) || misaligned(dOut, elem_bytes(dtype)) ||
      misaligned(slots, 4) || misaligned(order, 4) || misaligned(weights, 4) || misaligned(dweights, 4))
    return BSR_ERR_ALIGN;
  return launch_expert_combine_grad(Ys, dtype, rows, D, ldys, slots, order, entries ? T : 0, k, weights, dOut, lddo, dYs, lddys,
                                    dweights, static_cast<hipStream_t>(stream));
}

size_t bsr_distill_workspace_bytes(int64_t N, int64_t V, int64_t K) {
  if (check_matrix(N, V, V) != BSR_OK || V > kMaxRows || K < 0 || K > kMaxTeacher) return 0;
  return N == 0 ? 0 : distill_ws_bytes(N, V, K);
}

int bsr_distill_loss(const void *logits, int dtype, int64_t N, int64_t V, int64_t ldz, const void *ids, int index_type,
                     const void *teacher, int teacher_dtype, int64_t K, float temperature, float *loss, float *stats, void *ws,
                     size_t ws_bytes, void *stream) {
  const DistillArgs a = {logits, dtype, N, V, ldz, ids, index_type, teacher, teacher_dtype, K, temperature};
  BSR_REQUIRE(check_distill(a));
  if (N == 0) return BSR_OK;
  if (loss == nullptr || stats == nullptr) return BSR_ERR_NULL;
  if (misaligned(loss, 4) || misaligned(stats, 8)) return BSR_ERR_ALIGN;
  BSR_REQUIRE(check_workspace(distill_ws_bytes(N, V, K), ws, ws_bytes));
  return launch_distill_loss(a, loss, stats, ws, static_cast<hipStream_t>(stream));
}

int bsr_distill_grad(const void *logits, int dtype, int64_t N, int64_t V, int64_t ldz, const void *ids, int index_type,
                     const void *teacher, int teacher_dtype, int64_t K, float temperature, const float *stats, const float *dloss,
                     void *dlogits, int64_t ldd, void *stream) {
  const DistillArgs a = {logits, dtype, N, V, ldz, ids, index_type, teacher, teacher_dtype, K, temperature};
  BSR_REQUIRE(check_distill(a));
  BSR_REQUIRE(check_dlogits(a, dlogits, ldd));
  if (N == 0 || V == 0) return BSR_OK;
  if (stats == nullptr || dloss == nullptr) return BSR_ERR_NULL;
  if (misaligned(stats, 8) || misaligned(dloss, 4)) return BSR_ERR_ALIGN;
  return launch_distill_grad(a, stats, dloss, dlogits, ldd, static_cast<hipStream_t>(stream));
}

int bsr_distill_loss_grad(const void *logits, int dtype, int64_t N, int64_t V, int64_t ldz, const void *ids, int index_type,
                          const void *teacher, int teacher_dtype, int64_t K, float temperature, const float *dloss, float *loss,
                          void *dlogits, int64_t ldd, void *ws, size_t ws_bytes, void *stream) {
  const DistillArgs a = {logits, dtype, N, V, ldz, ids, index_type, teacher, teacher_dtype, K, temperature};
  BSR_REQUIRE(check_distill(a));
  BSR_REQUIRE(check_dlogits(a, dlogits, ldd));
  if (N == 0) return BSR_OK;
  if (loss == nullptr || dloss == nullptr) return BSR_ERR_NULL;
  if (misaligned(loss, 4) || misaligned(dloss, 4)) return BSR_ERR_ALIGN;
  BSR_REQUIRE(check_workspace(distill_ws_bytes(N, V, K), ws, ws_bytes));
  return launch_distill_loss_grad(a, dloss, loss, dlogits, ldd, ws, static_cast<hipStream_t>(stream));
}

}  // extern "C"
