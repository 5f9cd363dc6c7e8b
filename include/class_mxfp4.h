/*
 * class_mxfp4.h -- C ABI of answering with a trained output layer in 4 bits on one MI355X (gfx950): rows as microscaled 4-bit
 * floating point and back, logits of a batch against every class of this GPU's shard from such codes.
 *
 * The layer is the one of class_logits.h (logits = scale * <x, W[c]>, Section 3.2 of the paper named there); its 8-bit codes keep one scale
 * per row, these 4-bit codes one power of two per 32 elements: 17 bytes for 32 elements, at twice the rate of the matrix instructions.
 * Part of the same shared library; the conventions of knnsoftmax.h hold here too (device pointers, caller-owned memory, nothing
 * allocated, calls only enqueue work on `stream`, ks_status return values).  All calls may be captured into a graph.
 */
#ifndef CLASS_MXFP4_H
#define CLASS_MXFP4_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define KS_MXFP4_CLASSES 1u   /* the rows are class weights: codes in the order of the product's class side */

#define KS_MAX_MXFP4_D 65536   /* largest depth */
#define KS_MAX_MXFP4_B 4194240 /* largest batch of one class_logits_mxfp4 call */

/* ------------------------------------------------------------------------------------------------------
 * class_quantize_mxfp4 -- rows as 4-bit codes with a power of two per 32 elements of depth, in the order in which class_logits_mxfp4 reads them.
 *
 *   V  [n, D]  rows, dtype KS_DTYPE_BF16 or KS_DTYPE_FP32; row i begins at element i * ldv (ldv >= D; aligned to its elements is
 *              enough, 16-byte rows are read faster)
 *   The elements 32 b .. 32 b + 31 of a row are a block (a last one may be shorter).  With a its largest absolute value the block's
 *   exponent is e = max(floor(log2 a) - 2, -127), and an element v becomes the code of the value nearest to v / 2^e among
 *   0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives (codes 0 .. 7, and with bit 3 set; of two equally near ones the even code;
 *   beyond 6: 6).  A block of zeros has codes 0.  A block that holds an infinity or a NaN has codes 0 and the exponent byte 255: it
 *   stands for NaN, and so do all logits of its row.
 *   codes      out: class_mxfp4_bytes(n, D, flags) bytes, 16-byte aligned, all of them written: groups of 32 rows; a group holds
 *              P = ceil(D / 64) pieces of 1,024 bytes, then ceil(P / 4) pieces of 256 bytes of exponents.  Piece p: the low (even d) or
 *              high nibble of byte (h * 32 + r) * 16 + j is the code of element d = 64 p + 32 h + 2 j (+ 1) of the group's row r (h = 0, 1;
 *              j = 0 .. 15).  Exponents, piece p: byte (h * 32 + r) * 4 + t is e + 127 of the block at element 64 (4 p + t) + 32 h of row r.
 *              Group g holds rows 32 g + r, with KS_MXFP4_CLASSES rows 64 (g / 2) + 2 r + g % 2.  What lies beyond row n or
 *              element D is 0.
 * The codes must not overlap V.
 * class_dequantize_mxfp4 -- the values code * 2^e back as rows V [n, D] (exact in either type; NaN where the exponent byte is 255); elements
 * between D and ldv are not touched.
 * Both require 1 <= n < 2^31, 1 <= D <= KS_MAX_MXFP4_D (KS_UNSUPPORTED beyond).  class_mxfp4_bytes is 0 for sizes that are refused.
 * ---------------------------------------------------------------------------------------------------- */
size_t class_mxfp4_bytes(int64_t n, int D, uint32_t flags);
int class_quantize_mxfp4(const void *V, int dtype, int64_t n, int D, int64_t ldv, uint32_t flags, uint8_t *codes, void *stream);
int class_dequantize_mxfp4(const uint8_t *codes, int64_t n, int D, uint32_t flags, void *V, int dtype, int64_t ldv, void *stream);

/* ------------------------------------------------------------------------------------------------------
 * class_logits_mxfp4 -- the fc forward of Section 3.2 over all classes of the shard, from 4-bit codes of both sides:
 *     logits[i, c] = scale * sum over blocks of 2^(ex + ew) * sum_d qx[i, d] qw[c, d]  (+ bias[c])
 * The products are exact and summed in fp32; the sum is multiplied by scale and the bias added in fp32 with one rounding, and the
 * result rounded to the type of the logits.
 *
 *   x_codes  codes of the features [B, D] (class_quantize_mxfp4 without KS_MXFP4_CLASSES)
 *   w_codes  codes of the class weights [C, D] (with KS_MXFP4_CLASSES)
 *   bias     [C] fp32, may be NULL
 *   logits   [B, C] out, dtype KS_DTYPE_FP32 or KS_DTYPE_BF16; row i begins at element i * ldl (ldl >= C; elements between C and ldl
 *            are not touched).  Aligned to its elements is enough; rows that begin on whole 128-byte lines are written fastest
 * Requires 1 <= B <= KS_MAX_MXFP4_B, 1 <= C < 2^31, 1 <= D <= KS_MAX_MXFP4_D (KS_UNSUPPORTED beyond the maxima).
 * ---------------------------------------------------------------------------------------------------- */
int class_logits_mxfp4(const uint8_t *x_codes, const uint8_t *w_codes, const float *bias, int64_t C, int D, int B, float scale,
                       void *logits, int dtype, int64_t ldl, void *stream);

#ifdef __cplusplus
}
#endif
#endif
