/*
 * bsr_token_step.h -- C ABI of the token operators of libbsr_actprune: the parts of
 * a token model's training step around its pruned linear layers that are no
 * matrix products.
 *
 *   token table : rows looked up and scaled; the table's gradient from tokens
 *                 sorted by value (every row's positions added in one order);
 *   experts     : tokens sorted by the expert that a router chose, in segments that
 *                 end on whole block-rows, so that bsr_score_select / bsr_compress
 *                 take the sorted matrix as it is and every expert's weight
 *                 gradient is one item of bsr_t_dense_matmul_batched; the experts'
 *                 outputs weighted and returned to their tokens; the gradients;
 *   loss        : distillation from the largest logits that a teacher left for every
 *                 position, forward, backward, and both in one call.
 *
 * Conventions are those of bsr_actprune.h: device pointers unless it says "host", all
 * buffers (workspaces included) the caller's, work enqueued on `stream`, checks on
 * the host before anything is launched, BSR_ERR_* codes, dtype BSR_F32 or BSR_BF16,
 * matrices row-major with a leading dimension in elements.  Sums are binary32, in an
 * order that depends on the sizes and the data's positions alone (for distillation also
 * on the address of a row of logits modulo 16 bytes), so results are reproducible bit
 * for bit; a bfloat16 result is rounded once, to nearest even, from the binary32 sum.
 * Rows of padding and of dropped tokens have no part in any result, NaN in them
 * included (some are read all the same).
 * Index arrays of the caller (tokens, expert_ids, ids) are int32 or int64 (index_type);
 * an index outside its range, -1 for instance, means "none" and is never followed.
 */
#ifndef BSR_TOKEN_STEP_H
#define BSR_TOKEN_STEP_H

#include "bsr_actprune.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { BSR_I32 = 0, BSR_I64 = 1 };

/* experts of a sort; rows of a token table whose gradient is wanted */
enum { BSR_MAX_EXPERTS = 1024, BSR_MAX_VOCAB = (1 << 30) - 1 };

enum { BSR_ERR_VALUE = -9 /* a number is outside its range: temperature outside [2^-60, 2^60], scale not finite */ };

/*
 * Token table, forward: out[t, :] = scale * table[tokens[t], :], rounded to dtype;
 * +0.0 where tokens[t] is outside [0, V).  table: [V x D], leading dimension ldt;
 * tokens: [T]; out: [T x D], leading dimension ldo, must not overlap table.
 */
int bsr_embedding_lookup(const void *table, int dtype, int64_t V, int64_t D,
                         int64_t ldt, const void *tokens, int index_type,
                         int64_t T, float scale, void *out, int64_t ldo,
                         void *stream);

/*
 * Token table, backward:
 *   dE[v, :] (+)= scale * (sum over t with tokens[t] == v, t ascending, of dY[t, :]).
 * dY: [T x D] of dtype, leading dimension lddy; dE: [V x D] binary32, leading
 * dimension ldde >= D: with accumulate == 0 every row is written (+0.0 for tokens that
 * do not occur), otherwise only rows of tokens that occur are touched, and added to.
 * Positions whose token is outside [0, V) have no gradient.  (A long sum is cut into
 * pieces of consecutive positions, which are added in order.)
 * T < 2^31, V <= BSR_MAX_VOCAB (BSR_ERR_SHAPE).  Workspace: the function below (0 for invalid sizes).
 */
size_t bsr_embedding_grad_workspace_bytes(int64_t T, int64_t V, int64_t D);
int bsr_embedding_grad(const void *tokens, int index_type, int64_t T,
                       const void *dY, int dtype, int64_t D, int64_t lddy,
                       float scale, int64_t V, float *dE, int64_t ldde,
                       int accumulate, void *ws, size_t ws_bytes, void *stream);

/*
 * Host, pure.  Rows that the sorted matrix of n entries needs, however they fall on E
 * experts whose segments start at multiples of `align`:
 * n + min(E, n) * (align - 1), rounded down to a multiple of align.  -1 for n < 0,
 * E < 1, align < 1 or a result of 2^31 or more.
 */
int64_t bsr_expert_capacity(int64_t n, int64_t E, int64_t align);

/*
 * Entries sorted by expert.  expert_ids: [n], for instance the [T x k] choices of a
 * router, entry t*k + j being the j-th choice of token t; ids outside [0, E) are
 * dropped.  Stable: the entries of an expert keep their order.
 *   counts  [E]     entries of every expert;
 *   offsets [E + 1] first row of every expert's segment; offsets[e + 1] = offsets[e] +
 *                   counts[e] rounded up to a multiple of align;
 *   order   [rows]  entry that a row holds, -1 for rows of padding (also behind the last
 *                   segment); rows = bsr_expert_capacity(n, E, align);
 *   slots   [n]     row that holds an entry, -1 for a dropped one.
 * E <= BSR_MAX_EXPERTS (BSR_ERR_LIMIT beyond).  Workspace: the function below.
 */
size_t bsr_expert_sort_workspace_bytes(int64_t n, int64_t E);
int bsr_expert_sort(const void *expert_ids, int index_type, int64_t n, int64_t E,
                    int64_t align, int32_t *offsets, int32_t *counts,
                    int32_t *order, int32_t *slots, void *ws, size_t ws_bytes,
                    void *stream);

/*
 * Tokens to the experts: Xs[s, :] = X[order[s] / k, :] bit for bit, +0.0 in rows of
 * padding.  X: [T x D]; slots: [T x k] and order: [rows] from bsr_expert_sort; Xs:
 * [rows x D], must not overlap X.  Its gradient is bsr_expert_combine of the gradient of
 * Xs without weights.
 */
int bsr_expert_gather(const void *X, int dtype, int64_t T, int64_t D, int64_t ldx,
                      const int32_t *slots, int64_t k, const int32_t *order,
                      int64_t rows, void *Xs, int64_t ldxs, void *stream);

/*
 * ... and back: out[t, :] = sum over j (ascending) with a slot of weights[t, j] *
 * Ys[slots[t, j], :], rounded to dtype; +0.0 for a token without any.  weights: [T x k]
 * binary32, or NULL for a plain sum.  out: [T x D], must not overlap Ys.
 */
int bsr_expert_combine(const void *Ys, int dtype, int64_t rows, int64_t D,
                       int64_t ldys, const int32_t *slots, int64_t T, int64_t k,
                       const float *weights, void *out, int64_t ldo, void *stream);

/*
 * Gradient of bsr_expert_combine with weights:
 *   dYs[slots[t, j], :] = weights[t, j] * dOut[t, :], rounded to dtype; +0.0 in rows of
 *                         padding (every row of dYs [rows x D] is written);
 *   dweights[t, j]      = sum over d of Ys[slots[t, j], d] * dOut[t, d], binary32; +0.0
 *                         for a dropped entry.
 * dYs must not overlap Ys or dOut.
 */
int bsr_expert_combine_grad(const void *Ys, int dtype, int64_t rows, int64_t D,
                            int64_t ldys, const int32_t *slots,
                            const int32_t *order, int64_t T, int64_t k,
                            const float *weights, const void *dOut, int64_t lddo,
                            void *dYs, int64_t lddys, float *dweights,
                            void *stream);

/*
 * Distillation.  logits z: [N x V] of dtype, leading dimension ldz; for every row K
 * entries of the teacher: ids [N x K] (columns; outside [0, V): no entry; a column may
 * occur more than once) and teacher [N x K], the teacher's logits, of teacher_dtype.
 * With the temperature tau,
 *   q = softmax over a row's entries of teacher / tau,   p = softmax over v of z / tau,
 *   loss[n]   = tau^2 * sum_j q_j * (log q_j - log p[ids_j])          (binary32)
 *   stats[n]  = (m, L): m = max_v z_v, L = log sum_v exp((z_v - m) / tau)   [N x 2], binary32
 *   dlogits[n, v] = dloss[n] * tau * (p_v - sum over j with ids_j == v of q_j), rounded to dtype.
 * An entry with q_j = 0 adds nothing: a teacher logit of -inf, or one so far below the
 * row's largest that exp of the difference over tau is less than 2^-126.  A row without
 * entries, or whose entries are all -inf, has the loss 0 and the gradient 0, whatever its
 * logits (its statistics are still those of its logits).  A row with a NaN or +inf logit
 * or with nothing but -inf has no distribution: its L, loss and gradient are NaN.  Logits
 * of -inf otherwise count as p = 0 (loss +inf where q is not 0).  So do logits of the
 * type's lowest value in the gradient of a row with larger ones; an entry there costs
 * tau * q * (m - z), which binary32 holds where tau * q < 1 and rounds to +inf from about
 * there on.
 * A teacher logit of NaN or +inf makes its row's loss and the gradient at its entries NaN.
 * K = 1 with any finite teacher logit is the cross entropy of a class.
 * K <= 1024 (BSR_ERR_LIMIT beyond).
 * bsr_distill_loss is the forward pass, bsr_distill_grad the backward pass from its stats;
 * bsr_distill_loss_grad does both in one call for callers that know dloss beforehand,
 * which saves a pass over the logits.  dlogits ([N x V], leading dimension ldd) may be
 * logits itself (with ldd == ldz), and must not overlap it otherwise.
 * Workspace of bsr_distill_loss and bsr_distill_loss_grad: the function below.
 */
size_t bsr_distill_workspace_bytes(int64_t N, int64_t V, int64_t K);
int bsr_distill_loss(const void *logits, int dtype, int64_t N, int64_t V, int64_t ldz,
                     const void *ids, int index_type, const void *teacher,
                     int teacher_dtype, int64_t K, float temperature, float *loss,
                     float *stats, void *ws, size_t ws_bytes, void *stream);
int bsr_distill_grad(const void *logits, int dtype, int64_t N, int64_t V, int64_t ldz,
                     const void *ids, int index_type, const void *teacher,
                     int teacher_dtype, int64_t K, float temperature,
                     const float *stats, const float *dloss, void *dlogits,
                     int64_t ldd, void *stream);
int bsr_distill_loss_grad(const void *logits, int dtype, int64_t N, int64_t V,
                          int64_t ldz, const void *ids, int index_type,
                          const void *teacher, int teacher_dtype, int64_t K,
                          float temperature, const float *dloss, float *loss,
                          void *dlogits, int64_t ldd, void *ws, size_t ws_bytes,
                          void *stream);

#ifdef __cplusplus
}
#endif
#endif /* BSR_TOKEN_STEP_H */
