/* xmem_ops.h -- C ABI of libxmem_ops.so: the operators of a dense training step
 * whose device memory is known before it runs, on one AMD Instinct MI355X (gfx950).
 *
 * The estimator of xmem.h says what a recorded step needs; these operators are
 * the parts of a step that allocate nothing by themselves: every output and
 * every workspace is the caller's, and its size a function of the shapes.
 *
 *   xmem_linear_forward/_backward  y = act(x w^T + b) + r and its gradients
 *   xmem_policy_loss               clipped policy loss with a KL term over a
 *                                  vocabulary, forward and backward in one pass
 *   xmem_muon_update               momentum and an update orthogonalised by
 *                                  Newton-Schulz products
 *
 * All calls run on the caller's stream, which has to be one of the current device,
 * allocate nothing, keep nothing and do not synchronise.  Pointers named d_* are device memory owned by the caller.
 * Matrices are row-major; ld* is the distance between rows in elements and at
 * least the row's length.  Rows need no more than their elements' alignment;
 * the fast loads want 16-byte aligned pointers and ld a multiple of 8 (and k a
 * multiple of 8 where rows are summed along).  Rows that are not are copied where
 * the product is large; an operand whose pointer alone is not aligned is read
 * through registers, at less than half the speed of a large product.  Errors are the XMEM_E* codes of xmem.h. */
#ifndef XMEM_OPS_H
#define XMEM_OPS_H

#include <stddef.h>
#include <stdint.h>

#include "../xmem.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
#define XMEM_BF16 0
#define XMEM_F16 1
#define XMEM_F32 2

/* Activations. */
#define XMEM_ACT_NONE 0
#define XMEM_ACT_RELU 1 /* max(z, 0) */
#define XMEM_ACT_GELU 2 /* z/2 (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3))) */
#define XMEM_ACT_SILU 3 /* z / (1 + exp(-z)) */

/* Workspace of xmem_linear_forward (may be 0: then d_workspace may be NULL):
 * sums of products with few outputs, and copies of operands whose rows are no
 * multiple of 8 elements apart or long.  0 for invalid sizes too. */
size_t xmem_linear_forward_workspace_bytes(int64_t m, int64_t n, int64_t k, int64_t ldx, int64_t ldw);

/* z = x w^T + b;  y = act(z) + r.  Sums and the epilogue are in 32 bits, y and
 * z are rounded once.
 *   d_x        : [m, k] of dtype (XMEM_BF16 or XMEM_F16)
 *   d_w        : [n, k] of dtype
 *   d_bias     : float32 [n] or NULL
 *   d_residual : [m, n] of dtype or NULL; may be d_y itself (with ldr == ldy)
 *   d_y        : [m, n] of dtype, written
 *   d_z        : [m, n] of dtype or NULL, written: what the backward pass needs
 *                of an activation
 *   d_workspace: >= its size, 256-byte aligned
 * k == 0 gives z = b.  No output may overlap another operand (d_residual apart).
 * Returns XMEM_OK, XMEM_EINVAL (null pointer, negative or too large size (2^30 and more), ld too
 * small, unknown dtype or activation), XMEM_EWORKSPACE or XMEM_EHIP. */
int xmem_linear_forward(const void* d_x, int64_t ldx, const void* d_w, int64_t ldw, const float* d_bias,
                        const void* d_residual, int64_t ldr, int64_t m, int64_t n, int64_t k, int dtype,
                        int activation, void* d_y, int64_t ldy, void* d_z, int64_t ldz, void* d_workspace,
                        size_t workspace_bytes, void* hip_stream);

/* Workspace of xmem_linear_backward: it holds dz where an activation has one
 * (activation != XMEM_ACT_NONE), partial sums, and copies as above. */
size_t xmem_linear_backward_workspace_bytes(int64_t m, int64_t n, int64_t k, int64_t lddy, int64_t ldx, int64_t ldw,
                                            int activation);

/* The gradients of xmem_linear_forward for an output gradient dy:
 *   dz = dy act'(z);  dx = dz w;  dw = dz^T x;  db = sum over rows of dz.
 * The residual's gradient is dy itself.  dz is rounded to dtype for the two
 * products (db sums it before that): a float16 dz past 65,504 becomes infinite.
 *   d_dy : [m, n] of dtype
 *   d_z  : [m, n] of dtype as xmem_linear_forward wrote it; not looked at (and
 *          NULL allowed) where activation is XMEM_ACT_NONE
 *   d_x, d_w : as in the forward pass; d_x may be NULL without d_dw, d_w without d_dx (their ld is
 *          looked at all the same: the workspace goes by it)
 *   d_dx : [m, k] of dtype or NULL, written
 *   d_dw : [n, k] of dtype or NULL, written
 *   d_db : float32 [n] or NULL, written
 * m == 0 gives dw = 0 and db = 0.  Returns as xmem_linear_forward. */
int xmem_linear_backward(const void* d_dy, int64_t lddy, const void* d_z, int64_t ldz, const void* d_x, int64_t ldx,
                         const void* d_w, int64_t ldw, int64_t m, int64_t n, int64_t k, int dtype, int activation,
                         void* d_dx, int64_t lddx, void* d_dw, int64_t lddw, float* d_db, void* d_workspace,
                         size_t workspace_bytes, void* hip_stream);

/* Workspace of xmem_policy_loss.  0 for invalid sizes and for 0 tokens. */
size_t xmem_policy_loss_workspace_bytes(int64_t tokens, int64_t vocab);

/* The clipped policy loss with a KL term, over logits x [tokens, vocab] and the
 * sampled tokens y:
 *   lp_t  = x_t[y_t] - log sum_j exp(x_tj)
 *   rho   = exp(lp_t - old_t)
 *   pg_t  = -min(rho A_t, min(max(rho, 1 - clip_low), 1 + clip_high) A_t)
 *   kl_t  = exp(ref_t - lp_t) - (ref_t - lp_t) - 1            (0 without d_ref_logp)
 *   loss  = sum_t w_t (pg_t + kl_coef kl_t)
 *   dlogits_tj = grad_scale dloss/dx_tj
 * The weights carry the mask and the normalisation (1/tokens kept, or a mean
 * over each sequence first).  A token with weight 0 is not looked at, whatever
 * its logits hold: its lp is 0 and its gradient 0.  Logits of -inf are entries the
 * vocabulary does not offer.  A row without one finite or +inf logit, a row with NaN or
 * +inf, and a token outside [0, vocab) give NaN for that row (and the sums).  A ratio
 * that overflows times an advantage of 0 is 0; with kl_coef 0 the KL term is reported and nothing else.
 *   d_logits  : [tokens, vocab] of dtype (XMEM_BF16, XMEM_F16 or XMEM_F32), rows ldl apart
 *   d_tokens  : int64 [tokens]
 *   d_weights : float32 [tokens], or NULL for 1/tokens each
 *   d_old_logp, d_advantages : float32 [tokens]
 *   d_ref_logp: float32 [tokens] or NULL
 *   d_stats   : float32 [4], written: the loss, sum w pg, sum w kl, sum of w
 *               over the tokens where the clipped branch was taken
 *   d_logp    : float32 [tokens], written
 *   d_dlogits : [tokens, vocab] of dtype, rows ldd apart, written; may be d_logits
 *               itself (ldd == ldl); NULL for the loss alone
 *   d_workspace: >= xmem_policy_loss_workspace_bytes(tokens, vocab), 256-byte aligned
 * With d_old_logp, d_advantages and d_stats all NULL (and d_ref_logp and
 * d_dlogits NULL) only d_logp is written and no workspace is needed.
 * Sums run in a fixed order: the same inputs give the same bits.
 * Returns XMEM_OK, XMEM_EINVAL, XMEM_EWORKSPACE or XMEM_EHIP. */
int xmem_policy_loss(const void* d_logits, int64_t ldl, const int64_t* d_tokens, const float* d_weights,
                     const float* d_old_logp, const float* d_advantages, const float* d_ref_logp, int64_t tokens,
                     int64_t vocab, int dtype, float clip_low, float clip_high, float kl_coef, float grad_scale,
                     float* d_stats, float* d_logp, void* d_dlogits, int64_t ldd, void* d_workspace,
                     size_t workspace_bytes, void* hip_stream);

/* Coefficients of a Newton-Schulz step and the most steps a call takes. */
#define XMEM_NS_A 3.4445f
#define XMEM_NS_B -4.7750f
#define XMEM_NS_C 2.0315f
#define XMEM_NS_MAX_STEPS 16

/* Workspace of xmem_muon_update.  0 for invalid sizes and for 0 matrices. */
size_t xmem_muon_update_workspace_bytes(int64_t count, int64_t rows, int64_t cols);

/* Momentum and the orthogonalised update of `count` matrices [rows, cols]:
 *   m <- mu m + g;   u = g + mu m (nesterov) or m
 *   X = u / (|u|_F + 1e-7), transposed where rows > cols
 *   steps times:  P = X X^T;  X <- a X + (b P + c P P) X      (XMEM_NS_A, _B, _C)
 *   update = scale X, transposed back
 * The products take 16-bit floating operands and sum in 32 bits.
 *   d_grad    : [count, rows, cols] contiguous, of grad_dtype (XMEM_BF16, XMEM_F16, XMEM_F32)
 *   d_momentum: float32 [count, rows, cols], read and written
 *   d_update  : bfloat16 [count, rows, cols], written
 *   d_workspace: >= xmem_muon_update_workspace_bytes(count, rows, cols), 256-byte aligned
 * Returns XMEM_OK, XMEM_EINVAL (null pointer, negative or too large size (rows or
 * cols of 2^21 - 64 or more, count past 65,535, rows cols of 2^40 or more, 2^28 tiles of 64 x 64 or more in all), steps
 * outside 0..XMEM_NS_MAX_STEPS, unknown type), XMEM_EWORKSPACE or XMEM_EHIP. */
int xmem_muon_update(const void* d_grad, int grad_dtype, float* d_momentum, int64_t count, int64_t rows, int64_t cols,
                     float mu, int nesterov, int steps, float scale, void* d_update, void* d_workspace,
                     size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* XMEM_OPS_H */
