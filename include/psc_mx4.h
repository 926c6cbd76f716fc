/*
 * psc_mx4.h - the vocabulary projection in microscaled 4-bit floating point: half of
 * the weights' bytes of psc_head_logits, on the tensor cores' own 4-bit products.
 *
 * The format (OCP Microscaling Formats, MXFP4): a row's columns are cut into blocks of
 * 32; a block's values are codes of 4 bits times 2^e of the block.
 *     code   : sign (bit 3) and magnitude 0, 1/2, 1, 3/2, 2, 3, 4, 6 (bits 0-2);
 *              two a byte, the even column in the low half; a row is whole blocks, 16
 *              bytes each, zeros past K
 *     block  : a byte e + 127 (0 to 254; 255: the block is NaN), in tiles of 128 rows by 4
 *              blocks, 512 bytes, in the order in which the tensor core takes them: of row r
 *              and block b, with n = ceil(K / 128) tiles of a row,
 *                  512 * ((r / 128) * n + b / 4) + 16 * (r % 32) + 4 * (r % 128 / 32) + b % 4
 *              psc_mx4_block_bytes(rows, K) bytes in all.  Blocks past K in a row's last tile
 *              are zeros (psc_quantize_mx4 writes them); rows past the last are never used.
 * A matrix may have a factor per row besides (float).
 *
 * Conventions, status codes and psc_last_error are those of psc.h, with those that
 * psc_ops.h adds: calls only enqueue work on the stream, may be captured in a CUDA graph,
 * and give the same bits for the same inputs.  Codes start at multiples of 16 bytes with
 * strides that are multiples of 16, blocks at multiples of 16 bytes, other arrays at multiples of
 * their elements; other calls are refused.  (Codes at multiples of 128 bytes are read fastest.)
 */
#ifndef PSC_MX4_H
#define PSC_MX4_H

#include "psc_ops.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of the blocks' exponents of a matrix (0 for sizes that are refused). */
int64_t psc_mx4_block_bytes(int32_t rows, int32_t K);

/* The rows of a matrix in 4 bits: with m the largest magnitude of a block,
 *     e = max(floor(log2 m) - 2, -127)      code = the magnitude nearest to x / 2^e
 * ties to the code with bit 0 clear, 6 where x / 2^e is larger; a block of zeros has e = -127.
 * A block that holds an infinity or a NaN is NaN (its codes 0).
 *   d_x      : [T] rows of row_stride elements of dtype, K of them used
 *   d_q      : uint8 [T] rows of q_stride bytes, the first 16 ceil(K / 32) written
 *   d_blocks : uint8 [psc_mx4_block_bytes(T, K)]; of rows past T nothing is written
 * PSC_ERR_LIMIT: K over 2^30. */
psc_status psc_quantize_mx4(const void* d_x, psc_dtype dtype, int64_t row_stride, int32_t T, int32_t K, uint8_t* d_q,
                            int64_t q_stride, uint8_t* d_blocks, void* stream);

/* The values again: y[t][k] = code * 2^e * scale[t], in f32, rounded once to dtype.
 *   d_scale  : float [T], or NULL (ones)
 *   d_y      : [T] rows of row_stride elements of dtype; columns >= K are left as they are
 * PSC_ERR_LIMIT: K over 2^30. */
psc_status psc_dequantize_mx4(const uint8_t* d_q, int64_t q_stride, const uint8_t* d_blocks, const float* d_scale,
                              int32_t T, int32_t K, void* d_y, psc_dtype dtype, int64_t row_stride, void* stream);

/* The vocabulary projection in 4 bits, under the mask:
 *     logits[t][v] = (sum_k x_t[k] w_v[k]) * scale[t] * w_scale[v]
 * over the values of both matrices, where the mask allows v for row t, -inf elsewhere; rows of
 * w that no token allows need not be read.  Products are exact; sums over K are in f32, in an
 * order that depends on the sizes, and come before the factors: sums of |x_t[k] w_v[k]| from 2^-100 to
 * 2^127 keep f32's accuracy; from 2^128 on a logit may be infinite or NaN where its formula is not, and
 * smaller ones lose bits.
 *   d_q, d_q_blocks : the tokens, [T] rows    d_w, d_w_blocks : the weights, [V] rows
 *   d_scale         : float [T], d_w_scale : float [V], each NULL for ones
 *   d_bitmask       : uint32 [T][ceil(V/32)], or NULL (every token allowed)
 *   d_logits        : [T] rows of row_stride elements of dtype; columns >= V are left as they are
 * A block in which a bounded wait gives up (a pipeline fault) leaves some logits unwritten and
 * is counted (psc_mx4_faults).
 * PSC_ERR_LIMIT: K over 131,072, T over 2^24 or V over 2^30. */
psc_status psc_head_logits_mx4(const uint8_t* d_q, int64_t q_stride, const uint8_t* d_q_blocks, const float* d_scale,
                               int32_t T, const uint8_t* d_w, int64_t w_stride, const uint8_t* d_w_blocks,
                               const float* d_w_scale, int32_t V, int32_t K, const uint32_t* d_bitmask, void* d_logits,
                               psc_dtype dtype, int64_t row_stride, void* stream);

/* Blocks of psc_head_logits_mx4 on the current device in which a bounded wait gave up, since the
 * library was loaded or the last reset; synchronises the stream (not while it is captured).  reset != 0 takes
 * off the count what it reports: each fault is in one of several callers' reports, whatever runs beside them. */
psc_status psc_mx4_faults(int32_t* h_faults, int32_t reset, void* stream);

/* Self-test of that fault path: psc_head_logits_mx4 into f32 logits, with waits that give up after `limit`
 * looks (0 to 2^22; some tens of nanoseconds each, where the projection itself waits for seconds).  Blocks
 * in which one does leave logits unwritten, wait for what they have under way, end, and are counted;
 * nothing faults, and the device stays usable. */
psc_status psc_mx4_check_wait(const uint8_t* d_q, int64_t q_stride, const uint8_t* d_q_blocks, const float* d_scale,
                              int32_t T, const uint8_t* d_w, int64_t w_stride, const uint8_t* d_w_blocks,
                              const float* d_w_scale, int32_t V, int32_t K, const uint32_t* d_bitmask, void* d_logits,
                              psc_dtype dtype, int64_t row_stride, int32_t limit, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* PSC_MX4_H */
