/*
 * psc_norm.h - the model's end in front of the vocabulary projection: the last residual
 * addition and root-mean-square norm, with an output that psc_head_logits (8-bit integers) or
 * psc_head_logits_mx4 (4-bit floating point) reads.
 *
 * Conventions, status codes and psc_last_error are those of psc.h, with those that psc_ops.h
 * adds: calls only enqueue work on the stream, may be captured in a CUDA graph, and give the
 * same bits for the same inputs.  Arrays start at multiples of their elements' size (other calls are
 * refused); rows of whole multiples of 8 elements at multiples of 32 bytes are read fastest.
 */
#ifndef PSC_NORM_H
#define PSC_NORM_H

#include "psc_mx4.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The model's last residual addition and root-mean-square norm, quantised as psc_quantize_rows does:
 *     h = x + residual, rounded to their type      r = 1 / sqrt(mean_k h^2 + eps)
 *     v = h * gain      s = max_k |v| * (1 / 127)      q = rint(v / s)      scale = s * r
 * in f32, ties to even: q * scale stands for the normalised row r * h * gain.  r is a factor
 * of the whole row, so it is in the scale alone, and the codes depend on h and gain only.  A
 * row of zeros (or one whose s underflows to zero) gets scale 0 and q 0; a row in which some
 * h or v is an infinity or a NaN gets scale NaN and q 0.  mean_k h^2 neither overflows nor
 * underflows for finite h.  A row's results do not depend on the batch that it is in, nor on how the
 * other tensors lie (where rows of x do not all start at multiples of 32 bytes, a scale's last bits
 * depend on where its row starts).
 *   d_x, d_residual : [T] rows of dtype, K used (d_residual NULL: h = x)
 *   d_sum    : [T] rows of dtype that receive h, or NULL; may be d_x or d_residual (then with the
 *              same stride), otherwise overlaps no input
 *   d_gain   : float [K], or NULL (ones)
 *   eps      : finite, not negative
 *   d_q      : int8 [T] rows of q_stride bytes; bytes past K are left as they are
 *   d_scale  : float [T]
 * PSC_ERR_LIMIT: K over 2^30. */
psc_status psc_norm_quantize_rows(const void* d_x, psc_dtype dtype, int64_t row_stride, const void* d_residual,
                                  int64_t residual_stride, void* d_sum, int64_t sum_stride, const float* d_gain,
                                  float eps, int32_t T, int32_t K, int8_t* d_q, int64_t q_stride, float* d_scale,
                                  void* stream);

/* psc_norm_quantize_rows with an output in the format of psc_mx4.h: h, v and r as there,
 *     the codes and blocks of v as psc_quantize_mx4 makes them      scale = r
 * (scale NaN for a row in which some h or v is not finite; 0 for a row of zeros with eps 0;
 * infinity where r is beyond f32, for which eps has to be 0 and the root mean square 2^-128 or less).
 * As r is in the scale alone, the codes and blocks hold v as it is, and its size goes through the
 * sums of psc_head_logits_mx4: see there.
 * PSC_ERR_LIMIT: K over 2^30. */
psc_status psc_norm_quantize_mx4(const void* d_x, psc_dtype dtype, int64_t row_stride, const void* d_residual,
                                 int64_t residual_stride, void* d_sum, int64_t sum_stride, const float* d_gain,
                                 float eps, int32_t T, int32_t K, uint8_t* d_q, int64_t q_stride, uint8_t* d_blocks,
                                 float* d_scale, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* PSC_NORM_H */
