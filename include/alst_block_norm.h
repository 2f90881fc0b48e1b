/*
 * alst_block_norm.h -- C ABI of the MI355X (gfx950) norms around a transformer block, fused with the block's
 * gate and its scaled residual addition.
 *
 * What stands between two blocks (alst_mlp.h) of a layer: the norm after a block, the gate on its output, the
 * addition to the residual stream and the norm before the next block.  Rows are independent, so it belongs to
 * the work that is done without looking across the sequence.
 *
 *   p  = b * q1 * (w_post + o)       q1 = 1 / sqrt(mean(b^2) + eps)       (p = b without w_post)
 *   r' = r + s * sigmoid(z) * p      z: a gate logit for each element or for each row (1 without a gate)
 *   n  = r' * q2 * (w_pre + o)       q2 = 1 / sqrt(mean(r'^2) + eps)
 *
 * b [N,H] the block's output, r [N,H] the residual stream, w_post, w_pre [H], z [N,H] or [N], s = branch_scale
 * and o = weight_offset (0, or 1 for weights kept as their difference from one) host scalars.  Every part is
 * optional: without w_pre there is no n (the end of a layer whose next block has no norm before it), without
 * b there is only the norm n of r (before the first block).
 *
 * Gradients, with dn and dr' upstream (x2 = r' q2, x1 = b q1):
 *   dr   = dr' + q2 (dn (w_pre + o) - x2 mean(dn (w_pre + o) x2))          dw_pre  = sum_rows dn x2
 *   dp   = s sigmoid(z) dr,  dz = s sigmoid'(z) p dr (summed over the row for a gate of one logit a row)
 *   db   = q1 (dp (w_post + o) - x1 mean(dp (w_post + o) x1))              dw_post = sum_rows dp x1
 *
 * All arithmetic is fp32 (a row whose sum of squares is beyond it, 4096 values of 3e17 or one of 2e19, is normalised to zeros) and every
 * output is rounded once; n is made from the r' before its rounding, the
 * gradients from the r' as it was stored.  Conventions are those of alst.h: device pointers, dense row-major
 * without strides, H a multiple of 8, 16-byte aligned base pointers, the caller owns every buffer, calls
 * validate on the host, enqueue on `stream` and return an alst_status without synchronising; they allocate
 * nothing and can be captured into a HIP graph.  1 <= N <= 2^30, 8 <= H <= 16384 (a row stays in the registers
 * of one workgroup), eps a normal positive number.
 * ALST_FLAG_RESIDUAL_FP32: r, r', dr' and dr are fp32 instead of bf16.  Everything else but the weight
 * gradients is bf16.
 */
#ifndef ALST_BLOCK_NORM_H
#define ALST_BLOCK_NORM_H

#include "alst.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of device scratch that alst_block_norm_backward needs (partial sums of the weight gradients, at most
 * 8 H bytes for each of 256 workgroups), 0 if the shape is invalid.  Pure host arithmetic. */
size_t alst_block_norm_workspace_bytes(int64_t N, int64_t H);

/*
 *   residual      [N,H]
 *   branch        [N,H] or NULL: then w_post, gate and residual_out are NULL and w_pre is not
 *   w_post        [H] or NULL: the block's output is not normalised
 *   gate          [N,H] (gate_cols = H), [N] (gate_cols = 1; it and d_gate need no alignment beyond their elements') or NULL
 *                 (gate_cols = 0)
 *   w_pre         [H] or NULL: then normed is NULL
 *   residual_out  [N,H] r', overwritten; may be `residual` itself, or `branch` if both are of the same type
 *   normed        [N,H] n, overwritten; may be `branch` itself
 * Apart from that no output may overlap another buffer.
 */
int alst_block_norm_forward(const void* residual, const void* branch, const void* w_post, const void* gate,
                            int64_t gate_cols, const void* w_pre, int64_t N, int64_t H, float branch_scale,
                            float eps, float weight_offset, void* residual_out, void* normed, uint32_t flags,
                            void* stream);

/*
 *   residual_out    [N,H] r' as forward wrote it (without a branch: forward's `residual`); without w_pre it is not
 *                   read and may be NULL
 *   d_normed        [N,H] dn; NULL exactly if w_pre is
 *   d_residual_out  [N,H] dr', or NULL for zeros (only with w_pre)
 *   d_residual      [N,H] dr, overwritten; may be `d_residual_out` itself; NULL only if there is no w_pre: dr is
 *                   then dr' and need not be written
 *   d_branch        [N,H] db, overwritten; NULL exactly if branch is.  May be `branch` or `d_normed` itself
 *   d_gate          like gate, overwritten; NULL exactly if gate is.  May be `gate` itself
 *   dw_post, dw_pre [H] bf16 (fp32 with ALST_FLAG_DW_FP32); overwritten, or += with ALST_FLAG_DW_ACCUMULATE;
 *                   NULL exactly if the weight is.  Sums over the rows are fp32, in an order that depends on N
 *                   and H alone.
 *   branch          may be NULL if there is neither w_post nor a gate, and is not read then; d_branch says that there
 *                   is a branch
 * Apart from that no output may overlap another buffer.
 */
int alst_block_norm_backward(const void* residual_out, const void* branch, const void* w_post,
                             const void* gate, int64_t gate_cols, const void* w_pre, const void* d_normed,
                             const void* d_residual_out, int64_t N, int64_t H, float branch_scale, float eps,
                             float weight_offset, void* d_residual, void* d_branch, void* d_gate,
                             void* dw_post, void* dw_pre, void* workspace, size_t workspace_bytes,
                             uint32_t flags, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* ALST_BLOCK_NORM_H */
