/*
 * class_sample.h -- C ABI of drawing one class per request from a matrix of logits on one MI355X (gfx950), what a serving loop does after
 * class_logits_adjust (class_logits.h): temperature, top-k, top-p and min-p, by random numbers that the caller brings.  A row holds all
 * classes that a request can get: where the layer is sharded, the shards' logits have to be gathered first.
 *
 * Part of the same shared library as knnsoftmax.h; the conventions stated there hold here too (device pointers, caller-owned memory and
 * workspace, nothing allocated, calls only enqueue work on `stream`, ks_status return values).  The call may be captured into a graph.
 */
#ifndef CLASS_SAMPLE_H
#define CLASS_SAMPLE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------------------------------------------
 * class_sample -- for each row z of the logits, with the row's own temperature T, k, p, m and u:
 *     1  the classes in order: by z, largest first, of equal ones the lowest first.  -infinity (a masked class) and NaN are left out
 *     2  top-k: the first k of them are kept                                                  (k <= 0 or k >= C: all)
 *     3  weights w = exp((z - z_max) / T); where z_max is +infinity: 1 for +infinity, else 0
 *     4  top-p: of what is kept the shortest beginning whose weight is at least p times all of it, at least one class   (p >= 1 or NaN: all)
 *     5  min-p: of these the ones with w >= m                                                 (m <= 0 or NaN: all; m > 1 counts as 1)
 *     6  in order of their ids: the first class at which the running weight exceeds u times the weight of what is kept; u is brought
 *        into [0, 1), of a u beyond the last kept class is drawn
 * T <= 0 or NaN: the first class of the order, whatever u is (k = 1).
 *
 * Weights are whole numbers of 2^-s, s = min(48, 62 - ceil(log2 C)): exp() in fp64 rounded to the nearest, their sums exact; a class whose
 * weight is less than half of 2^-s is not drawn.  The weight of all classes, which rows without top-k need, is summed in fp64 over parts
 * of the row whose sizes C alone decides, in a fixed order, before it is rounded (a part of which no class has a weight counts nothing), and
 * without top-k, top-p and min-p the running weight at the beginning of the part that is drawn from is made of these sums.  The result
 * depends on the row and its settings alone.
 *
 *   logits [B, C]   in, dtype KS_DTYPE_FP32 or KS_DTYPE_BF16; row i begins at element i * ldl (ldl >= C; aligned to its elements is
 *                   enough, rows that begin on 16 bytes are read faster)
 *   u [B]           fp32, in [0, 1)
 *   temperature, top_p, min_p [B] fp32, top_k [B] int32      each may be NULL: 1, 1, 0, 0 for all rows
 *   ids [B]         out: the drawn class, -1 where a row has no class to draw (all of it -infinity or NaN)
 *   logprob [B]     out, fp32, may be NULL: the logarithm of its weight's share of what is kept; -infinity where ids is -1
 * Requires B >= 1, 1 <= C < 2^31.  Workspace: class_sample_workspace, 12 bytes for each of up to 4,096 parts of a row, and 25 to 57 KB a row of
 * 32,768 classes or more; 0 for sizes that are refused.
 * ---------------------------------------------------------------------------------------------------- */
size_t class_sample_workspace(int64_t C, int B);
int class_sample(const void *logits, int64_t ldl, int dtype, int64_t C, int B, const float *u, const float *temperature,
                 const int32_t *top_k, const float *top_p, const float *min_p, int32_t *ids, float *logprob, void *ws, size_t ws_bytes,
                 void *stream);

#ifdef __cplusplus
}
#endif
#endif
