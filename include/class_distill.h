/*
 * class_distill.h -- C ABI of learning from a teacher's top logits on one MI355X (gfx950): loss and gradient of a batch of logits against
 * every class, where the teacher says for each sample which classes it holds likely and how much (a larger layer's answer: class_logits.h,
 * class_mxfp4.h).  It stands beside full_softmax_fwd_bwd (knnsoftmax.h), whose teacher names one class and which takes W and X: this call
 * takes the logits and gives their gradient, the products before and behind it are the caller's.  A row holds all classes of the layer:
 * where the layer is sharded, the shards' logits have to be gathered first (ids count from 0 to C - 1 in the row).
 *
 * Part of the same shared library; the conventions of knnsoftmax.h hold here too (device pointers, caller-owned memory and workspace,
 * nothing allocated, calls only enqueue work on `stream`, ks_status return values, KS_DEV_* bits in *dev_status, no floating-point
 * atomics).  The call may be captured into a graph.
 */
#ifndef CLASS_DISTILL_H
#define CLASS_DISTILL_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define KS_MAX_DISTILL_K 4096 /* most classes that a teacher names */

/* ------------------------------------------------------------------------------------------------------
 * class_distill_fwd_bwd -- with T = temperature, for every sample i:
 *     p = softmax(logits[i, :] / T) over all C classes
 *     q = softmax(t_logits[i, :] / T) over the entries that are not empty; of a class that is named more than once the sum of its entries
 *     loss_i = T^2 sum_c q_c (log q_c - log p_c)           (entries with q = 0 count nothing; each entry by itself where a class is
 *                                                           named more than once),      loss_mean = mean_i loss_i
 *     dlogits[i, c] = grad_scale * T / B * (p_c - q_c)     (the gradient of grad_scale * loss_mean)
 * Powers and a row's sum of them are fp32, the rest of the loss is fp64: a loss is off by at most T^2 / 50,000 (the roundings of
 * ln sum_c exp(z_c / T), up to some 200 of 2^-24) and a like share of itself, whatever number is added to all logits of the row, and may be
 * below 0 by as much.  p_c and q_c have as many roundings, powers below 2^-126 are 0; dlogits is rounded to its type once.
 *
 *   logits [B, C]     in, dtype KS_DTYPE_FP32 or KS_DTYPE_BF16, row i at element i * ldl (ldl >= C; aligned to its elements is enough; reads and
 *                     writes are fastest where rows of logits and dlogits begin equally many bytes beside a multiple of 16)
 *   t_ids [B, K]      class ids, negative: an empty entry; ids >= C set KS_DEV_BAD_LABEL and count as empty
 *   t_logits [B, K]   the teacher's logits, t_dtype KS_DTYPE_FP32 or KS_DTYPE_BF16, in any order; -infinity: q = 0
 *   loss_per_sample [B], loss_mean [1] fp32     out
 *   dlogits [B, C]    out, dtype of the logits, row i at element i * ldd; elements between C and ldd are not touched.  dlogits == logits (then
 *                     ldd == ldl): in place; any other overlap is not allowed
 * A sample without entries (or whose entries are all -infinity) has loss and gradient 0: padding.  A class with logit -infinity has p = 0; where
 * its q > 0 the loss is +infinity and the gradient as above.  A row of logits that are all -infinity has p = 0.  A NaN or +infinity among
 * the logits makes the row's loss and gradient NaN, one among the teacher's logits the loss and the gradient at the named classes.
 * Requires B >= 1, 1 <= C < 2^31, 1 <= K <= KS_MAX_DISTILL_K (KS_UNSUPPORTED beyond), 1e-30 <= temperature <= 1e30.
 * Workspace: class_distill_workspace, 0 for sizes that are refused.
 * ---------------------------------------------------------------------------------------------------- */
size_t class_distill_workspace(int64_t C, int B, int K);
int class_distill_fwd_bwd(const void *logits, int64_t ldl, int dtype, int64_t C, int B, const int32_t *t_ids, const void *t_logits,
                          int t_dtype, int K, float temperature, float grad_scale, float *loss_per_sample, float *loss_mean,
                          void *dlogits, int64_t ldd, void *ws, size_t ws_bytes, int32_t *dev_status, void *stream);

#ifdef __cplusplus
}
#endif
#endif
