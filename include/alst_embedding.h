/*
 * alst_embedding.h -- C ABI of the MI355X (gfx950) token embedding.
 *
 * The operation (ALST paper, section "Sequence Tiling for Reducing Activation Memory Footprint": the token
 * embedding is among the operations without cross-sequence dependency): the first operation of a training
 * step, whose table is often the LM head's W (alst.h).
 *
 *   y[i]  = scale * E[t_i]                       tokens t [N], E [V,H], y [N,H]
 *   dE[v] = scale * sum_{i: t_i = v} dy[i]       dy [N,H], dE [V,H]
 *
 * A token equal to `ignore_index` (padding) has a row of zeros and takes no part in dE: its row of dy is not
 * read.  Conventions are those of alst.h: device pointers, dense row-major without strides, H a multiple of 8,
 * 16-byte aligned base pointers (tokens: 4 bytes), the caller owns every buffer, calls validate on the host, enqueue
 * on `stream` and return an alst_status without synchronising; they allocate nothing and can be captured into
 * a HIP graph.  1 <= N <= 2^30, 8 <= H <= 2^20, 1 <= V <= 2^24.  No output may overlap another buffer.
 * A token that is neither ignore_index nor in [0,V) is treated as ignored and reported in a status word.
 */
#ifndef ALST_EMBEDDING_H
#define ALST_EMBEDDING_H

#include "alst.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of device scratch that alst_embedding_backward needs, 0 if the shape is invalid.  Pure host
 * arithmetic.  Large terms: 16 N bytes for the tokens in sorted order, V bytes for the tokens that occur, and fp32 sums of tokens
 * whose sorted rows are cut into ranges: N H / 16 bytes, in short calls up to N H and 32 MB.  A workspace serves every N up
 * to its own. */
size_t alst_embedding_workspace_bytes(int64_t N, int64_t H, int64_t V);

/*
 *   tokens [N] int32, E [V,H] bf16     inputs, not modified
 *   scale                              host scalar; the product is rounded once
 *   y [N,H] bf16 (fp32 with ALST_FLAG_RESIDUAL_FP32)     overwritten, every row
 *   device_status_out [1] int32        may be NULL; set to ALST_ERR_LABEL_RANGE if a token is out of range, else
 *                                      left as it is: the caller clears it
 */
int alst_embedding_forward(const int32_t* tokens, const void* E, int64_t N, int64_t H, int64_t V,
                           int32_t ignore_index, float scale, void* y, int32_t* device_status_out,
                           uint32_t flags, void* stream);

/*
 *   dy [N,H] bf16 (fp32 with ALST_FLAG_RESIDUAL_FP32)
 *   dE [V,H] bf16 (fp32 with ALST_FLAG_DW_FP32); every row overwritten, or += with ALST_FLAG_DW_ACCUMULATE
 *            (rows of tokens that do not occur are then neither read nor written).  With a tied table and fp32
 *            gradients the call follows alst_tiled_ce_backward on the same dW.
 * The rows of a token are added up in fp32, in an order that depends on the tokens alone: calls with the same
 * inputs give the same bits.  alst_last_device_status(workspace) tells of a token out of range.
 */
int alst_embedding_backward(const int32_t* tokens, const void* dy, int64_t N, int64_t H, int64_t V,
                            int32_t ignore_index, float scale, void* dE, void* workspace,
                            size_t workspace_bytes, uint32_t flags, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* ALST_EMBEDDING_H */
