/* xmem_step.h -- more operators of libxmem_ops.so: what a training step does around its products, on one AMD
 * Instinct MI355X (gfx950).
 *
 *   xmem_residual_norm_forward/_backward  norm of a block's output, gate, scale, residual sum and the next block's
 *                                         norm, and the gradients of all of them
 *   xmem_embedding_forward/_backward      scaled rows of a table, and the table's gradient
 *   xmem_clip_grad_norm                   the norm of many gradients as one vector, and their scaling
 *
 * The conventions are those of xmem_ops.h: calls run on the caller's stream of the current device, allocate nothing,
 * keep nothing and do not synchronise; pointers named d_* are the caller's device memory; matrices are row-major with
 * ld* elements between rows, which need no more than their elements' alignment (16-byte aligned rows are faster).
 * Element types are XMEM_BF16, XMEM_F16 and XMEM_F32, sums are in 32 bits or more and run in a fixed order: the same
 * inputs give the same bits.  Errors are the XMEM_E* codes of xmem.h. */
#ifndef XMEM_STEP_H
#define XMEM_STEP_H

#include "xmem_ops.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Norms of a row x of n elements: (x - mu) rho, with rho = 1 / sqrt(mean of (x - mu)^2 + eps). */
#define XMEM_NORM_NONE 0
#define XMEM_NORM_RMS 1   /* mu = 0 */
#define XMEM_NORM_LAYER 2 /* mu = mean of x */

/* What a gate g multiplies with. */
#define XMEM_GATE_NONE 0 /* g itself */
#define XMEM_GATE_SIGMOID 1
#define XMEM_GATE_SILU 2

/* Between two blocks:
 *   u = norm_post(h) w1 + b1;   v = a(gate) u;   out = r + alpha s v;   y = norm_pre(out) w2 + b2
 * Everything between is in 32 bits; out and y are rounded once (y is computed from the sum before its rounding).
 *   d_r    : [tokens, width] of dtype, the residual stream
 *   d_h    : [tokens, width] of dtype, the block's output; NULL: there is none, y is the norm of d_r (then d_gate,
 *            d_scale, d_w1, d_b1 and d_out are NULL and post is XMEM_NORM_NONE)
 *   d_gate : [tokens, width] of dtype, or NULL for 1
 *   d_scale, d_w1, d_w2 : float32 [width], or NULL for 1;  d_b1, d_b2 : float32 [width], or NULL for 0
 *            (d_w1 and d_b1 are NULL where post is XMEM_NORM_NONE, d_w2 and d_b2 where pre is)
 *   d_out  : [tokens, width] of dtype, written; may be d_r itself (with ldo == ldr)
 *   d_y    : [tokens, width] of dtype, written; NULL where (and only where) pre is XMEM_NORM_NONE
 *   d_stats: float32 [4, tokens] or NULL, written: mu and rho of the first norm, then of the second; 0 where there is no
 *            such norm, and for mu of XMEM_NORM_RMS
 * No output may overlap another operand (d_out on d_r apart).  A row is its own: NaN or infinity stays in its row.
 * Sums of squares are in 32 bits: a row whose squares add up to more than they hold has rho = 0.
 * Returns XMEM_OK, XMEM_EINVAL (null pointer, what the lines above rule out, tokens outside 0..2^31-1, width outside
 * 1..2^31-1, ld below width or 2^40 and more, unknown type, norm or gate, eps negative or NaN) or XMEM_EHIP. */
int xmem_residual_norm_forward(const void* d_r, int64_t ldr, const void* d_h, int64_t ldh, const void* d_gate, int64_t ldg,
                               const float* d_scale, float alpha, int post, const float* d_w1, const float* d_b1, int pre,
                               const float* d_w2, const float* d_b2, int gate_activation, float eps, int64_t tokens, int64_t width,
                               int dtype, void* d_out, int64_t ldo, void* d_y, int64_t ldy, float* d_stats, void* hip_stream);

/* Workspace of xmem_residual_norm_backward: partial sums of the vectors' gradients (none of these wanted: it may be 0
 * bytes and NULL).  0 for invalid sizes and for 0 tokens.  It never shrinks with more tokens. */
size_t xmem_residual_norm_backward_workspace_bytes(int64_t tokens, int64_t width, int dtype);

/* The gradients of xmem_residual_norm_forward, for dy of y and dout of out (what comes to the sum past y).
 *   d_dy   : [tokens, width] of dtype; NULL where (and only where) pre is XMEM_NORM_NONE
 *   d_dout : [tokens, width] of dtype, or NULL for 0 (wanted where pre is XMEM_NORM_NONE)
 *   d_out  : as the forward pass wrote it (d_r where d_h is NULL); not looked at, and may be NULL, without d_dy
 *   d_stats: as the forward pass wrote it
 *   d_h, d_gate, d_scale, alpha, post, d_w1, d_b1, pre, d_w2, gate_activation: as in the forward pass
 *   d_dr   : [tokens, width] of dtype, written: the gradient of the residual stream; may be d_dout (lddr == lddout)
 *   d_dh   : [tokens, width] of dtype, written; NULL where (and only where) d_h is NULL
 *   d_dgate: [tokens, width] of dtype, or NULL, written
 *   d_dscale, d_dw1, d_db1, d_dw2, d_db2 : float32 [width], or NULL, written
 *   d_workspace: >= its size, 256-byte aligned, where one of those five is wanted
 * tokens == 0 gives 0 for the five.  No output may overlap another operand (d_dr on d_dout apart); a workspace that does is refused.
 * Returns as the forward pass, XMEM_EINVAL for a workspace that overlaps too, or XMEM_EWORKSPACE. */
int xmem_residual_norm_backward(const void* d_dy, int64_t lddy, const void* d_dout, int64_t lddout, const void* d_out, int64_t ldo,
                                const float* d_stats, const void* d_h, int64_t ldh, const void* d_gate, int64_t ldg,
                                const float* d_scale, float alpha, int post, const float* d_w1, const float* d_b1, int pre,
                                const float* d_w2, int gate_activation, int64_t tokens, int64_t width, int dtype, void* d_dr,
                                int64_t lddr, void* d_dh, int64_t lddh, void* d_dgate, int64_t lddg, float* d_dscale, float* d_dw1,
                                float* d_db1, float* d_dw2, float* d_db2, void* d_workspace, size_t workspace_bytes,
                                void* hip_stream);

/* A padding_id that no token has. */
#define XMEM_NO_PADDING INT64_MIN

/* y_t = scale table[id_t].  A token equal to padding_id gives a row of 0; any other outside [0, vocab) gives NaN.
 *   d_table: [vocab, width] of dtype, rows ldt apart
 *   d_ids  : int64 [tokens]
 *   d_y    : [tokens, width] of dtype, written
 * Returns XMEM_OK, XMEM_EINVAL (null pointer, tokens outside 0..2^31-1, vocab or width outside 1..2^31-1, ld below width
 * or 2^40 and more, unknown type) or XMEM_EHIP. */
int xmem_embedding_forward(const void* d_table, int64_t ldt, const int64_t* d_ids, int64_t tokens, int64_t vocab, int64_t width,
                           int dtype, float scale, int64_t padding_id, void* d_y, int64_t ldy, void* hip_stream);

/* Workspace of xmem_embedding_backward, whether it adds or not.  0 for invalid sizes; it may be 0 otherwise too.  It never shrinks with
 * more tokens: that of the largest batch holds every smaller one of the same table. */
size_t xmem_embedding_backward_workspace_bytes(int64_t tokens, int64_t vocab, int64_t width);

/* dtable_v = scale * (the sum of dy_t over the tokens t with id_t = v), added to what d_dtable holds where add is not 0.
 * Rows that no token names are not looked at then, and are 0 without it, whatever scale is.  Sums are in 32 bits, in a fixed
 * order, and rounded once.  Tokens equal to padding_id and tokens outside [0, vocab) add nothing and name no row.
 *   d_dy    : [tokens, width] of dtype, rows lddy apart
 *   d_dtable: [vocab, width] of dtype or of XMEM_F32 (out_dtype), rows ldd apart, written
 *   d_workspace: >= its size, 256-byte aligned
 * d_dtable may overlap neither d_dy nor d_ids; a workspace that overlaps one of the three is refused.
 * Returns as xmem_embedding_forward, XMEM_EINVAL for a workspace that overlaps too, or XMEM_EWORKSPACE. */
int xmem_embedding_backward(const void* d_dy, int64_t lddy, const int64_t* d_ids, int64_t tokens, int64_t vocab, int64_t width,
                            int dtype, float scale, int64_t padding_id, int add, int out_dtype, void* d_dtable, int64_t ldd,
                            void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* Workspace of xmem_clip_grad_norm. */
size_t xmem_clip_grad_norm_workspace_bytes(void);

/* The 2-norm of `count` gradients as one vector, and their scaling:
 *   norm = scale sqrt(sum of all g^2);   factor = scale min(1, max_norm / (norm + 1e-6));   g <- factor g
 * With max_norm = INFINITY and scale = 1 the factor is 1: nothing but the norm is computed and no gradient is written.
 * A factor of 1 leaves the gradients as they are.  scale is what the gradients are to be multiplied with anyway (1 over a loss
 * scale, or over the number of batches that were added up).  Squares are added up in 64 bits.  A norm of NaN makes every
 * gradient NaN; where it is infinite they become 0, or NaN where infinite themselves (under an infinite limit the factor stays scale).
 *   d_tensors: host array of `count` device pointers; sizes, dtypes: host arrays of their elements and element types.
 *              All three are read before the call returns.  Elements of a gradient are contiguous and need no more than their
 *              own alignment.  Gradients that overlap are refused where they would be written.
 *   d_stats  : float32 [2], written: norm and factor
 *   d_workspace: >= its size, 256-byte aligned
 * Returns XMEM_OK, XMEM_EINVAL (null pointer, negative or too large count (2^31) or size (2^48), unknown type, max_norm
 * negative or NaN, scale negative or not finite, overlap, a workspace on a gradient or on d_stats), XMEM_EWORKSPACE or XMEM_EHIP. */
int xmem_clip_grad_norm(void* const* d_tensors, const int64_t* sizes, const int* dtypes, int64_t count, float max_norm, float scale,
                        float* d_stats, void* d_workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* XMEM_STEP_H */
