/*
 * alst_grads.h -- C ABI of the MI355X (gfx950) global gradient norm and clipping.
 *
 * The last operation on the weight gradients that the calls of alst.h, alst_mlp.h, alst_linear.h,
 * alst_embedding.h and alst_block_norm.h leave, before an optimizer takes them:
 *
 *   S = sum over the tensors, over their elements, of g^2        norm = sqrt(S)
 *   out = g * min(1, max_norm / norm)
 *
 * S is summed in fp64 in an order that depends on the tensors' sizes, types and 16-byte phases alone: the same gradients give the
 * same bits.  A norm that is not finite in fp32 (an infinity or NaN among the gradients) leaves the gradients as they
 * are: the caller sees it in norm_out and skips the step.
 *
 * Tensors may be of any size (0 too) and aligned to their elements only, as views into a flat buffer are, 2^45
 * bytes in all at most; two tensors of a call must not overlap.  Conventions are otherwise those of alst.h: the caller owns every
 * buffer, calls validate on the host, enqueue on `stream` and return an alst_status without synchronising; they
 * allocate nothing and can be captured into a HIP graph (the list of tensors is read during the call, into the
 * kernels' arguments).
 */
#ifndef ALST_GRADS_H
#define ALST_GRADS_H

#include "alst.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    const void* grad;      /* device; [n], dense */
    void* out;             /* device; [n] of the same type, may be `grad` itself, must not overlap it otherwise; not used by
                              alst_grad_norm */
    int64_t n;             /* elements, 0 <= n <= 2^40 */
    int32_t fp32;          /* 0: bf16, 1: fp32 */
    int32_t reserved;      /* 0 */
} alst_grad_tensor;

/* Bytes of device scratch for a list of `count` tensors (1 <= count <= 2^20), 0 if that is out of range.
 * Pure host arithmetic. */
size_t alst_grad_norm_workspace_bytes(int64_t count);

/*
 * The norm alone.  tensors: HOST array [count].
 *   sumsq_out [1] fp64      S: what ranks that hold different gradients add up before they clip
 *   norm_out  [1] fp32      sqrt(S); may be NULL
 */
int alst_grad_norm(const alst_grad_tensor* tensors, int64_t count, double* sumsq_out, float* norm_out,
                   void* workspace, size_t workspace_bytes, void* stream);

/*
 * Clipping alone, by sumsq [1] fp64 (device) as alst_grad_norm left it, or the sum of several.  max_norm > 0
 * (infinite: nothing is scaled); norm_out [1] fp32 receives sqrt(sumsq), may be NULL.  Where out is grad itself
 * and the norm is not above max_norm, nothing is read or written.
 */
int alst_grad_clip(const alst_grad_tensor* tensors, int64_t count, const double* sumsq, float max_norm,
                   float* norm_out, void* stream);

/* Both in one call, with the same results; sumsq_out and norm_out may be NULL. */
int alst_grad_norm_clip(const alst_grad_tensor* tensors, int64_t count, float max_norm, double* sumsq_out,
                        float* norm_out, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* ALST_GRADS_H */
