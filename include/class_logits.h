/*
 * class_logits.h -- C ABI of answering with a trained output layer on one MI355X (gfx950): logits of a batch against every class of
 * this GPU's shard from 8-bit codes of the class weights, then the penalties, biases and masks that the requests bring.
 *
 * The layer is the one of Section 3.1 of "Large-Scale Training System for 100-Million Classification at Alibaba" (KDD'20): W [C, D]
 * holds one row per class, the logits of a feature row x are scale * <x, W[c]> (Section 3.2).  Part of the same shared library as
 * knnsoftmax.h; the conventions stated there hold here too (device pointers, caller-owned memory, nothing allocated, calls only
 * enqueue work on `stream`, ks_status return values, KS_DEV_* bits in *dev_status, no floating-point atomics).  All three calls
 * may be captured into a graph.  Nothing here has a gradient: training goes through knnsoftmax.h.
 */
#ifndef CLASS_LOGITS_H
#define CLASS_LOGITS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define KS_DTYPE_INT8 2 /* input of class_quantize_rows: codes as they are */

#define KS_QUANT_CLASSES 1u   /* the rows are class weights: codes in the order of the product's class side */
#define KS_QUANT_NORMALIZE 2u /* scales of the L2-normalised rows: row_scale is divided by the row's norm */

#define KS_MAX_INT8_D 65536   /* largest depth: the integer sums are at most 2^30 */
#define KS_MAX_INT8_B 4194240 /* largest batch of one class_logits_int8 call */

/* ------------------------------------------------------------------------------------------------------
 * class_quantize_rows -- rows as 8-bit integer codes with one scale each, in the order in which class_logits_int8 reads them.
 *
 *   V  [n, D]  rows, dtype KS_DTYPE_BF16, KS_DTYPE_FP32 or KS_DTYPE_INT8; row i begins at element i * ldv (ldv >= D; aligned to its
 *              elements is enough, 16-byte rows are read faster)
 *   row_scale [n] out:  a / 127 with a = max_d |V[i, d]|, rounded to fp32 once; with KS_QUANT_NORMALIZE a / (127 |V[i, :]|), so
 *              that code * row_scale stands for the normalised row (the codes are the same).  Must be NULL for KS_DTYPE_INT8
 *   codes      out: q[i, d] = 127 V[i, d] / a rounded to the nearest integer, halves to even, exactly (no rounding before that
 *              one); a KS_DTYPE_INT8 row is taken as it is.  class_codes_bytes(n, D, flags) bytes, 16-byte aligned, all of them
 *              written: blocks of 32 rows; a block holds ceil(D / 32) pieces of 1,024 bytes; in piece p, byte
 *              (h * 32 + r) * 16 + j  is the code of element 32 p + 16 h + j of the block's row r (h = 0, 1; j = 0 .. 15).
 *              Block b holds rows 32 b + r, with KS_QUANT_CLASSES rows 64 (b / 2) + 2 r + b % 2.  What lies beyond row n or
 *              element D is 0.
 * The codes must not overlap V.  A zero row has codes 0 and scale 0.  A row that holds an infinity or a NaN has codes 0 and scale NaN:
 * all its logits are NaN.
 * Requires 1 <= n < 2^31, 1 <= D <= KS_MAX_INT8_D (KS_UNSUPPORTED beyond); KS_QUANT_NORMALIZE not with KS_DTYPE_INT8.
 * class_codes_bytes is 0 for sizes that are refused.
 * ---------------------------------------------------------------------------------------------------- */
size_t class_codes_bytes(int64_t n, int D, uint32_t flags);
int class_quantize_rows(const void *V, int dtype, int64_t n, int D, int64_t ldv, uint32_t flags, int8_t *codes, float *row_scale,
                        void *stream);

/* ------------------------------------------------------------------------------------------------------
 * class_logits_int8 -- the fc forward of Section 3.2 over all classes of the shard, in 8-bit integers:
 *     logits[i, c] = scale * x_scale[i] * w_scale[c] * sum_d qx[i, d] qw[c, d]  (+ bias[c])
 * The sum is exact; it is converted to fp32, multiplied by fp32(scale * x_scale[i]) and by w_scale[c], the bias added, in fp32
 * (at most five roundings of 2^-24 while these stay within fp32's normal range), and rounded to the type of the logits.
 *
 *   x_codes  codes of the features [B, D] (class_quantize_rows without KS_QUANT_CLASSES), x_scale [B]
 *   w_codes  codes of the class weights [C, D] (with KS_QUANT_CLASSES), w_scale [C]
 *   bias     [C] fp32, may be NULL
 *   logits   [B, C] out, dtype KS_DTYPE_FP32 or KS_DTYPE_BF16; row i begins at element i * ldl (ldl >= C; elements between C and ldl
 *            are not touched, so that a node of a sharded layer may write its columns of a larger matrix).  Aligned to its
 *            elements is enough; rows that begin on whole 128-byte lines are written fastest.  With batches of more than 64 others
 *            take up to two and a half times as long (1,024 x 390,625 x 512 bf16: 260 us, ldl = 390,626 680, ldl = 390,625 490)
 * Requires 1 <= B <= KS_MAX_INT8_B, 1 <= C < 2^31, 1 <= D <= KS_MAX_INT8_D (KS_UNSUPPORTED beyond the maxima).
 * ---------------------------------------------------------------------------------------------------- */
int class_logits_int8(const int8_t *x_codes, const float *x_scale, const int8_t *w_codes, const float *w_scale, const float *bias,
                      int64_t C, int D, int B, float scale, void *logits, int dtype, int64_t ldl, void *stream);

/* ------------------------------------------------------------------------------------------------------
 * class_logits_adjust -- what a request changes in its row of the logits z, in this order:
 *     1  penalties for classes it has seen, where class c occurs in the request's list:
 *            z = z > 0 ? z / repetition : z * repetition
 *            z = z - (frequency * n + presence)          if c occurs n > 0 times behind the list's first n_prompt entries
 *     2  z = z + (bias of the class)
 *     3  z = -infinity where the request's mask does not allow the class, whatever z was (an infinity, a NaN)
 * Steps 1 and 2 are done in fp32 and rounded to the type of the logits once; a class that neither occurs in a list nor is masked
 * keeps its logit's bits.  A mask that allows nothing leaves a row of -infinity.
 *
 *   logits [B, C]    in, dtype KS_DTYPE_FP32 or KS_DTYPE_BF16, row i at element i * ldl
 *   out    [B, C]    out, same dtype, row i at element i * ldo; out == logits (then ldo == ldl): in place, where only listed and masked
 *                    classes' logits change; any other overlap is not allowed
 *   C, c0, Cg        the columns are the classes [c0, c0 + C) of a problem with Cg (c0 + C <= Cg).  Lists carry ids of the whole
 *                    problem: another node's classes are passed over, negative ids are empty entries, ids >= Cg set KS_DEV_BAD_LABEL
 *   seen_offsets [B + 1], seen_ids [seen_len]   the list of request i is seen_ids[seen_offsets[i] .. seen_offsets[i + 1]); NULL
 *                    offsets: no lists.  A list that is longer than seen_max or not inside the array sets KS_DEV_BAD_COUNT and is
 *                    not read
 *   n_prompt [B]     entries of the list that count for `repetition` alone (clamped to the list); NULL: none
 *   repetition, presence, frequency [B]         fp32; NULL: no such penalty.  repetition > 0 (1: no effect)
 *   bias_offsets [B + 1], bias_ids, bias_values [bias_len], bias_max   lists of single classes' biases, likewise, but that ids >= Cg
 *                    set KS_DEV_BAD_INDEX; of a class that is named twice the later entry counts
 *   allowed [n_masks, ld_allowed] uint32        masks: bit c % 32 of word c / 32 set: column c (class c0 + c) is allowed;
 *                    ld_allowed >= ceil(C / 32); bits beyond C are ignored.  NULL: no masks
 *   mask_row [B]     mask of request i, negative: everything is allowed; an index >= n_masks sets KS_DEV_BAD_INDEX and counts as
 *                    negative.  NULL: mask i (then n_masks >= B)
 * Requires B >= 1, 1 <= C, c0 >= 0, c0 + C <= Cg < 2^31, seen_max + bias_max < 2^30.
 * ---------------------------------------------------------------------------------------------------- */
int class_logits_adjust(const void *logits, int64_t ldl, void *out, int64_t ldo, int dtype, int64_t C, int64_t c0, int64_t Cg, int B,
                        const int64_t *seen_offsets, const int32_t *seen_ids, int64_t seen_len, int seen_max,
                        const int32_t *n_prompt, const float *repetition, const float *presence, const float *frequency,
                        const int64_t *bias_offsets, const int32_t *bias_ids, const float *bias_values, int64_t bias_len,
                        int bias_max, const uint32_t *allowed, int64_t ld_allowed, int n_masks, const int32_t *mask_row,
                        int32_t *dev_status, void *stream);

#ifdef __cplusplus
}
#endif
#endif
