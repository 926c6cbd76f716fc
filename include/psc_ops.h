/*
 * psc_ops.h - the operators around the grammar mask: the vocabulary projection
 * that makes the logits, the penalties and biases that change them, and the
 * draw of a token among the allowed ones.
 *
 * They take packed masks as psc_fill_mask writes them (bit v of a row is bit
 * (v & 31) of word (v >> 5), ceil(V / 32) words a row), so that one decoding
 * step is
 *     psc_fill_mask, psc_quantize_rows, psc_head_logits, psc_process_logits,
 *     psc_sample, psc_advance
 * on one stream.  Conventions, status codes and psc_last_error are those of
 * psc.h: d_* pointers are device memory owned by the caller, calls only enqueue
 * work on the stream and never synchronise or allocate, a refused call
 * (PSC_ERR_ARG, PSC_ERR_LIMIT) has launched nothing, and every call may be
 * captured in a CUDA graph.  Results do not depend on the order in which
 * threads run: the same inputs give the same bits.
 */
#ifndef PSC_OPS_H
#define PSC_OPS_H

#include "psc.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Symmetric 8-bit quantisation of the rows of a matrix: activations (a row is a
 * token) or, once, weights (a row is an output channel).
 *     scale[t] = max_k |x[t][k]| * (1 / 127)     q[t][k] = rint(x[t][k] / scale[t])
 * in f32, ties to even.  A row of zeros (or one whose scale underflows to zero)
 * gets scale 0 and q 0; a row that holds an infinity or a NaN gets scale NaN
 * and q 0, so that whatever is computed from it shows it.
 *   d_x      : [T] rows of row_stride elements of dtype, K of them used
 *   d_q      : int8 [T] rows of q_stride bytes; bytes past K are left as they are
 *   d_scale  : float [T]
 * PSC_ERR_LIMIT: K over 2^30. */
psc_status psc_quantize_rows(const void* d_x, psc_dtype dtype, int64_t row_stride, int32_t T, int32_t K,
                             int8_t* d_q, int64_t q_stride, float* d_scale, void* stream);

/* Bytes of workspace that psc_head_logits needs for these sizes; aligned: whether d_w
 * and w_stride are multiples of 16.  (256 for sizes that it refuses.) */
int64_t psc_head_work_bytes(int32_t T, int32_t V, int32_t K, int32_t aligned);

/* The vocabulary projection in 8-bit integers, under the mask:
 *     logits[t][v] = (sum_k q[t][k] * w[v][k]) * scale[t] * w_scale[v]
 * where the mask allows v for row t, -inf elsewhere; rows of w that no token
 * allows need not be read.  Sums are exact while every partial sum stays within
 * 2^24 in magnitude (always for K <= 1024; for K <= 1040 where neither side holds -128).
 * Beyond, they carry roundings that depend on T: up to 16 tokens may be summed in whole
 * numbers of 32 bits and rounded once, larger batches are summed in f32, so that a token's
 * logits may differ in their last bits between a small batch and a large one.
 *   d_q, d_w      : int8 [T] and [V] rows of q_stride and w_stride bytes, K of them used
 *   d_scale       : float [T], d_w_scale : float [V]
 *   d_bitmask     : uint32 [T][ceil(V/32)], or NULL (every token allowed)
 *   d_logits      : [T] rows of row_stride elements of dtype; columns >= V are left as they are
 *   d_work        : at least psc_head_work_bytes bytes, 256-byte aligned; calls that overlap
 *                   on the GPU need workspaces of their own.  Its first int32 is afterwards
 *                   the number of blocks in which a bounded wait gave up (a pipeline fault;
 *                   some logits are then not written), 0 otherwise
 * Weights whose rows are at 16-byte-aligned addresses (d_w and w_stride; any K) are
 * read where they are; others are packed into the workspace first, a slab at a time.
 * PSC_ERR_LIMIT: K over 131,072 (a sum could pass 32 bits), T over 2^24, V over 2^30, or
 * ceil(T/256) * ceil(V/128) over 2^31 - 1. */
psc_status psc_head_logits(const int8_t* d_q, int64_t q_stride, const float* d_scale, int32_t T, const int8_t* d_w,
                           int64_t w_stride, const float* d_w_scale, int32_t V, int32_t K, const uint32_t* d_bitmask,
                           void* d_logits, psc_dtype dtype, int64_t row_stride, void* d_work, int64_t work_bytes,
                           void* stream);

/* Penalties for repeated tokens, biases and the mask, on logits:
 *     y = logits[b][v]
 *     v in the history (prompt or output)  : y = y > 0 ? y / repetition[b] : y * repetition[b]
 *     v n > 0 times in the output          : y = y - frequency[b] * n - presence[b]
 *     v among the row's biases             : y = y + bias
 *     v forbidden by the mask              : y = -inf
 * in f32, rounded once to the logits' type; tokens that none of these names keep
 * their exact bits.
 *   d_logits, d_out : [B] rows of dtype; d_out may be d_logits (then row_stride = out_stride;
 *                     otherwise the two must not overlap).  Columns >= V are left as they are.
 *   d_history       : int32 [B] rows of history_stride token ids, H at most (NULL with H = 0: none);
 *                     ids outside [0, V) are skipped (padding)
 *   d_history_len   : int32 [B] ids used of each row (NULL: H; clamped to [0, H])
 *   d_prompt_len    : int32 [B] of those, how many at the front are the prompt (NULL: 0)
 *   d_repetition, d_frequency, d_presence : float [B], each NULL for 1, 0, 0
 *   d_bias_ids, d_bias : int32 and float [B][n_bias] (NULL with n_bias = 0); ids outside [0, V)
 *                     are skipped, of equal ids in a row the last counts
 *   d_bitmask       : uint32 [B][ceil(V/32)], or NULL
 * PSC_ERR_LIMIT: V over 2^30, H over 16,777,215 or n_bias over 4,096. */
psc_status psc_process_logits(const void* d_logits, psc_dtype dtype, int64_t row_stride, void* d_out,
                              int64_t out_stride, int32_t B, int32_t V, const int32_t* d_history,
                              int64_t history_stride, int32_t H, const int32_t* d_history_len,
                              const int32_t* d_prompt_len, const float* d_repetition, const float* d_frequency,
                              const float* d_presence, const int32_t* d_bias_ids, const float* d_bias, int32_t n_bias,
                              const uint32_t* d_bitmask, void* stream);

/* Bytes of workspace that psc_sample needs for a batch of this size (0: none). */
int64_t psc_sample_work_bytes(int32_t B);

/* Draws one token per row among the allowed ones, from one uniform number.
 * Candidates are the tokens that the mask allows whose logit is neither NaN nor
 * -inf (+inf counts as the largest finite value).  With m the largest candidate,
 *     z = (x - m) * (1 / T)      e = exp(z)      weight = rint(2^40 e)
 * A candidate stays when all of these hold:
 *     top_k : fewer than k candidates are strictly larger            (k <= 0: off)
 *     top_p : the weight of the strictly larger ones, among those top_k leaves,
 *             is below p times the weight of all that top_k leaves   (p >= 1: off)
 *     min_p : e >= min_p                                             (min_p <= 0: off)
 * (ties at a boundary stay together; the largest always stays).  The draw is the
 * first token by index at which the running weight of what stays passes
 * uniform[b] times its sum.  Weights are whole numbers, so every sum is exact
 * and the draw depends on the inputs alone.  T below 1e-6 (or NaN) is greedy: the
 * lowest index of the largest candidate, with log-probability 0; +inf counts as the
 * largest finite value (an even draw among what stays).
 *   d_logits   : [B] rows of row_stride elements of dtype, unchanged
 *   d_bitmask  : uint32 [B][ceil(V/32)], or NULL
 *   d_uniform  : float [B] in [0, 1), of which the first 24 bits are used
 *   d_temperature, d_top_p, d_min_p : float [B], d_top_k : int32 [B]; each NULL: 1, off, off, off
 *   d_tokens   : int32 [B]; -1 where a row has no candidate (as psc_argmax_masked)
 *   d_logprobs : float [B] or NULL: ln of the probability with which the token was drawn
 *                (weight over the sum of what stays; -inf where there is no candidate)
 *   d_work     : at least psc_sample_work_bytes(B) bytes (NULL if that is 0); calls that
 *                overlap on the GPU need workspaces of their own
 * PSC_ERR_LIMIT: V over 4,194,304 (the sum of the weights stays below 2^63). */
psc_status psc_sample(const void* d_logits, psc_dtype dtype, int64_t row_stride, int32_t B, int32_t V,
                      const uint32_t* d_bitmask, const float* d_uniform, const float* d_temperature,
                      const int32_t* d_top_k, const float* d_top_p, const float* d_min_p, int32_t* d_tokens,
                      float* d_logprobs, void* d_work, int64_t work_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* PSC_OPS_H */
