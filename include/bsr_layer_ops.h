/*
 * bsr_layer_ops.h -- C ABI of the layer operators of libbsr_actprune: what a training
 * step needs around and behind the pruned linear layers besides the token operators
 * (bsr_token_step.h).
 *
 *   layer norm  : forward and backward pass, with the gradients of weight and bias;
 *   gated block : H = act(X Wg) * (X Wu), both products, the activation and the product
 *                 in one kernel; its backward pass, whose dGU is the dY of the weights'
 *                 gradient (bsr_t_dense_matmul of the pruned X);
 *   optimizer   : one AdamW step over many tensors, moments in binary32 or in 8 bits.
 *
 * Conventions are those of bsr_actprune.h: device pointers unless it says "host", all
 * buffers (workspaces included) the caller's, work enqueued on `stream`, checks on
 * the host before anything is launched, BSR_ERR_* codes, dtype BSR_F32 or BSR_BF16,
 * matrices row-major with a leading dimension in elements, pointers aligned to their
 * element type.  Sums are binary32, in an order that depends on types, sizes, leading dimensions
 * and addresses modulo 128 bytes alone, so results are reproducible bit for bit; a bfloat16 result is
 * rounded once, to nearest even, from a binary32 value.
 * Outputs must not overlap inputs or each other except where it says so.
 */
#ifndef BSR_LAYER_OPS_H
#define BSR_LAYER_OPS_H

#include "bsr_token_step.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Layer norm of the rows of X [M x D]:
 *   Y[m, d] = (X[m, d] - mean[m]) * rstd[m] * gamma[d] + beta[d],
 *   mean = sum_d X / D, rstd = 1 / sqrt(sum_d (X - mean)^2 / D + eps).
 * gamma, beta: [D] of param_dtype; NULL: 1 and 0.  stats: [M x 2] binary32, (mean, rstd) of
 * every row, or NULL.  Y (of dtype) may be X itself, with ldy == ldx.
 * eps in [2^-126, 2^126] (BSR_ERR_VALUE).  A row that holds a NaN or an infinity, or whose
 * squares overflow binary32, gives NaN or the values that this arithmetic has; other rows are
 * not touched by it.  D == 0: nothing is written, stats neither.
 */
int bsr_layer_norm(const void *X, int dtype, int64_t M, int64_t D, int64_t ldx,
                   const void *gamma, const void *beta, int param_dtype, float eps,
                   void *Y, int64_t ldy, float *stats, void *stream);

/*
 * Its gradient, from X and its stats, with xh = (X - mean) * rstd and g = dY * gamma:
 *   dX[m, d]  = rstd[m] * (g - sum_d g / D - xh * sum_d (g * xh) / D), rounded to dtype;
 *   dgamma[d] (+)= sum_m dY * xh;   dbeta[d] (+)= sum_m dY          (binary32; added to what is
 *   there when accumulate != 0).
 * gamma NULL: 1.  dX may be dY itself (with lddx == lddy), or X (with lddx == ldx).  dgamma and dbeta
 * may be NULL, each on its own.  M == 0 writes zeros into them (nothing when accumulating).
 * Workspace: the function below (0 for invalid sizes).
 */
size_t bsr_layer_norm_grad_workspace_bytes(int64_t M, int64_t D);
int bsr_layer_norm_grad(const void *X, int dtype, int64_t M, int64_t D, int64_t ldx,
                        const void *gamma, int param_dtype, const float *stats,
                        const void *dY, int64_t lddy, void *dX, int64_t lddx,
                        float *dgamma, float *dbeta, int accumulate, void *ws,
                        size_t ws_bytes, void *stream);

/* widest rows of the gated block: D and 2F (BSR_ERR_LIMIT beyond) */
enum { BSR_MAX_GATED_WIDTH = (1 << 20) };

/* Activations of the gated block. */
enum {
  BSR_ACT_SILU = 0,      /* g / (1 + exp(-g)) */
  BSR_ACT_GELU = 1,      /* g * (1 + erf(g / sqrt 2)) / 2 */
  BSR_ACT_GELU_TANH = 2, /* g * (1 + tanh(sqrt(2/pi) * (g + 0.044715 g^3))) / 2 */
  BSR_ACT_RELU = 3       /* max(g, 0); derivative 0 at 0 */
};

/*
 * Gated feed-forward block, forward.  W: [D x 2F] of dtype, leading dimension ldw: the
 * gate's weights in columns [0, F), the other projection's in [F, 2F).
 *   [G | U] = X W,   H[m, f] = act(G[m, f]) * U[m, f], rounded to dtype.
 * X: [M x D]; H: [M x F]; GU: [M x 2F], G and U rounded to dtype, or NULL where no backward
 * pass follows (H is computed from the unrounded sums either way).
 * act: BSR_ACT_* (BSR_ERR_VALUE otherwise).  D == 0: zeros.
 * Workspace: the function below (host, pure; of X and W it only uses the addresses modulo 128
 * bytes; 0 for invalid arguments).
 */
size_t bsr_gated_ff_workspace_bytes(const void *X, int dtype, int64_t M, int64_t D,
                                    int64_t ldx, const void *W, int64_t F, int64_t ldw);
int bsr_gated_ff(const void *X, int dtype, int64_t M, int64_t D, int64_t ldx,
                 const void *W, int64_t F, int64_t ldw, int act, void *H, int64_t ldh,
                 void *GU, int64_t ldgu, void *ws, size_t ws_bytes, void *stream);

/*
 * ... backward, from the GU that the forward pass kept and dH [M x F]:
 *   dGU[m, f]     = dH * U * act'(G),  dGU[m, F + f] = dH * act(G), rounded to dtype;
 *   dX[m, d]      = sum over the 2F columns of dGU[m, :] * W[d, :], rounded to dtype, of the
 *                   rounded dGU where dtype is BSR_BF16 (the matrix cores' operands).
 * dGU [M x 2F] may be GU itself (with lddgu == ldgu).  dX [M x D] may be NULL: dGU alone (W is not
 * read then).  The gradient of W is X^T dGU: bsr_t_dense_matmul of the pruned X.
 * Workspace: the function below (as above, of dGU and W).
 */
size_t bsr_gated_ff_grad_workspace_bytes(const void *dGU, int dtype, int64_t M, int64_t F,
                                         int64_t lddgu, const void *W, int64_t D,
                                         int64_t ldw);
int bsr_gated_ff_grad(const void *GU, int dtype, int64_t M, int64_t F, int64_t ldgu,
                      const void *dH, int64_t lddh, int act, const void *W, int64_t D,
                      int64_t ldw, void *dGU, int64_t lddgu, void *dX, int64_t lddx,
                      void *ws, size_t ws_bytes, void *stream);

/*
 * One AdamW step over n tensors, in a handful of launches:
 *   g = grad_scale * grad;   m = beta1 m + (1 - beta1) g;   v = beta2 v + (1 - beta2) g^2;
 *   param = param * (1 - lr * weight_decay)
 *           - lr / (1 - beta1^step) * m / (sqrt(v / (1 - beta2^step)) + eps).
 * All of it is computed in binary32 (the powers of beta, and moments that are held in 8 bits, in binary64: v may leave
 * binary32's range there, its root may not) from the values before the step and rounded where it is stored; the update takes
 * m and v before they are rounded to 8 bits.  A v below 2^-150 held in binary32 is 0, and the update then m over eps.  Where
 * sqrt(v / (1 - beta2^step)) + eps is above 2^126 the update may be 0.
 * Moments in binary32: m [n], v [n].  In 8 bits (BSR_MOMENTS_8BIT): m [n] and v [n] are bytes,
 * and scales holds two rows of bsr_adamw_blocks(n) bytes, those of m and those of v, `scales_stride` bytes apart.  128
 * consecutive elements share a scale byte b:
 *   m = (-1)^(c >> 7) * k(c & 127, 3) * 2^(b - 144),    sqrt(v) = k(c, 4) * 2^(b - 145),
 *   k(c, f) with e = c >> f, r = c mod 2^f:  r where e == 0, else (r + 2^f) * 2^(e - 1).
 * Zeroed bytes are zero moments.  b follows the block's largest magnitude; below 2^-95 the block
 * is 0; b == 255: the block held a NaN, an infinity or more than 1.875 * 2^127, and all of it is NaN from then on.
 * A number x between two neighbours goes to the upper one with the probability of its distance
 * from the lower one: k = floor(x / step + u), u a multiple of 2^-16 made from (seed, step, the
 * element's number: tensors in order, each from a multiple of 128 on).  (To the nearest, sqrt(v) would
 * stand still: a step changes it by less than half the distance of its codes.)  A sqrt(v) of 2^-148 or more does not become 0 in a
 * block that does not.
 */
enum { BSR_MOMENTS_F32 = 0, BSR_MOMENTS_8BIT = 1 };

typedef struct {
  void *param;          /* [n] of param_dtype */
  const void *grad;     /* [n] of grad_dtype */
  void *m, *v;          /* [n] each: binary32, or bytes */
  uint8_t *scales;      /* 8 bits: see above; NULL otherwise */
  void *copy;           /* [n] bfloat16: receives the new param too; NULL: none */
  int64_t n;
  int64_t scales_stride;
  float weight_decay;
} bsr_adamw_item;

typedef struct {
  double lr, beta1, beta2, eps, grad_scale;
  int64_t step;                /* 1 for the first */
  uint64_t seed;               /* 8-bit moments: names the random numbers of all steps */
  /* Device pointers to single numbers, or NULL.  Where one is set it is read by the kernels in the place of
     the number above, unchecked, so that a captured graph can be replayed with another. */
  const float *lr_device, *grad_scale_device;
  const int64_t *step_device;
} bsr_adamw_options;

/*
 * items: host, not needed after the call.  Tensors must not overlap.  lr, grad_scale and weight decays finite, beta1 and
 * beta2 in [0, 1), eps in [2^-126, 2^126], step >= 1: BSR_ERR_VALUE otherwise.  n_items < 0, n < 0 or n > 2^40, or scales_stride < bsr_adamw_blocks(n)
 * where there are scales: BSR_ERR_SHAPE.
 */
int bsr_adamw_batched(const bsr_adamw_item *items, int n_items, int param_dtype,
                      int grad_dtype, int moments, const bsr_adamw_options *options,
                      void *stream);

/* Host, pure.  Scale bytes of n elements: ceil(n / 128); -1 for n < 0. */
int64_t bsr_adamw_blocks(int64_t n);

/*
 * The values that 8-bit moments stand for, for a checkpoint or to look at: out[i] = m (which == 0)
 * or sqrt(v) (which == 1) of dtype (either holds them exactly).  codes: [n]; scales: [bsr_adamw_blocks(n)]
 * of that moment.
 */
int bsr_adamw_state_values(const uint8_t *codes, const uint8_t *scales, int64_t n,
                           int which, void *out, int dtype, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* BSR_LAYER_OPS_H */
