/*
 * sbw_step.h -- the operators beside the watermark in a decode or training step, exported
 * by the same libsbw as sbw.h and following its conventions (status codes, dtypes, streams,
 * caller-owned buffers, checks on the host before any HIP call, nothing allocated, no host
 * synchronisation, no memset: every call can be captured in a HIP graph).
 *
 *   head_logits          next-token logits of a few hidden states by a head with 4-bit weights:
 *                        what the watermark takes
 *   top_candidates       the k largest logits of every row, in order: what
 *                        sbw_watermark_candidates takes
 *   token_logprobs       log probabilities of given tokens, log sum, entropy and the most
 *                        likely alternatives: what a step answers beside its token
 *   token_logprobs_grad  the gradient of those with respect to the logits
 *   sample_tokens        a token of every row by temperature, top-k, top-p and min-p
 *   quantize_fp8         a matrix in 8-bit floating point with a scale for each block of 128
 *   matmul_fp8           the product of two such matrices
 *
 * Logits are [B, row_stride] of dtype, element (b, v) at logits[b * row_stride + v], v < V;
 * columns from V on are neither read nor written.  Rows may start at any element.  Limits on
 * B, V and row_stride as in sbw.h (V < 2^32 - 2^16 here, else SBW_ERR_UNSUPPORTED).
 *
 * Order of logits (alternatives, candidates): larger first, equal ones by the lower column; a
 * NaN stands above every number; -0 and +0 are equal.
 *
 * Rows out of the ordinary.  A row whose every logit is -inf (a mask that leaves nothing) has
 * log sum -inf, log probabilities -inf, entropy 0 and gradient 0.  A row with a NaN or +inf has no
 * distribution: its log sum, log probabilities and entropy are NaN, and with them its gradient.
 * A logit of -inf in any other row is a token of probability 0; so is one further below the row's largest than
 * fp32's largest number, and the type's lowest value beside ordinary logits at ordinary temperatures.
 */
#ifndef SBW_STEP_H
#define SBW_STEP_H

#include "sbw.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Most tokens of a row (n), alternatives (top) and candidates (k) of one call. */
#define SBW_STEP_MAX_TOKENS 1024

/*
 * sbw_token_logprobs -- for every row, with y_v = logits_v * inv_temperature:
 *     lse      = log sum_v exp(y_v)
 *     logprob  = y_t - lse of each given token t
 *     entropy  = -sum_v p_v log p_v,  p_v = exp(y_v - lse)
 *     the `top` largest logits' columns and log probabilities, in order.
 * The logits are read once, and those of a few parts of each row again where alternatives are asked
 * for.  Sums are held in fp32 relative to the row's largest logit.
 *
 *   tokens       device, [B, n] int32.  An id outside [0, V) is padding: its log probability
 *                is 0.  May be NULL when n == 0.
 *   n            tokens per row, 0 <= n <= 1024 (n < 0 or top < 0: SBW_ERR_INVALID_ARG; beyond
 *                1024: SBW_ERR_UNSUPPORTED).
 *   inv_temperature  1/T, finite and > 0 (else SBW_ERR_INVALID_ARG).
 *   top          alternatives per row, 0 <= top <= 1024.
 *   logprobs     device, [B, n] float, written (may be NULL when n == 0).
 *   lse, entropy device, [B] float, written (either may be NULL).
 *   stats        device, [B, 2] float, written (may be NULL): the row's largest logit and log S,
 *                S = sum exp(y_v - largest y).  lse is their sum rounded once; the gradient takes the two
 *                apart, which stay exact for logits of any size.
 *   top_ids, top_logprobs  device, [B, top] int32 and float, written (may be NULL when top == 0;
 *                top_logprobs may be NULL).  Places beyond V hold -1 and -inf.
 *   workspace    device, sbw_token_logprobs_workspace(B, V, top) uint64 elements, caller-owned;
 *                contents on entry do not matter.  Calls that share one must be ordered.
 *   V == 0 with B > 0 is SBW_ERR_INVALID_ARG.
 */
sbw_status_t sbw_token_logprobs(const void *logits, sbw_dtype_t dtype, int64_t B, int64_t V,
                                int64_t row_stride, const int32_t *tokens, int64_t n,
                                float inv_temperature, int64_t top, float *logprobs, float *lse,
                                float *entropy, float *stats, int32_t *top_ids,
                                float *top_logprobs, uint64_t *workspace, void *stream);

/* Workspace sizes in uint64 elements (0 when a size is not positive or beyond the limits). */
int64_t sbw_token_logprobs_workspace(int64_t B, int64_t V, int64_t top);
int64_t sbw_top_candidates_workspace(int64_t B, int64_t V, int64_t k);

/*
 * sbw_token_logprobs_grad -- the gradient of sbw_token_logprobs's outputs with respect to the
 * logits: for the upstream gradients g_j of logprob j, g_l of lse and g_H of entropy,
 *     d_v = inv_temperature * ( sum_j g_j [v = t_j] + p_v * (g_l - sum_j g_j - g_H (log p_v + H)) ).
 * Padding tokens take no part.  A token given twice adds both gradients, in order.  Only a gradient beyond the
 * range of dtype is infinite, as long as the upstream gradients and their sums stay below 2^117.
 *
 *   tokens, n, inv_temperature   as for sbw_token_logprobs.
 *   stats, entropy  device, [B, 2] and [B] float, as sbw_token_logprobs wrote them (entropy may
 *                 be NULL when grad_entropy is).
 *   grad_logprobs device, [B, n] float, or NULL (all 0).
 *   grad_lse, grad_entropy   device, [B] float, each or NULL (0).
 *   grad          device, [B, grad_stride] of dtype, written for v < V; grad_stride >= V.  May be
 *                 the logits themselves (same pointer and stride: in place), and must not
 *                 overlap them otherwise.
 */
sbw_status_t sbw_token_logprobs_grad(const void *logits, sbw_dtype_t dtype, int64_t B, int64_t V,
                                     int64_t row_stride, const int32_t *tokens, int64_t n,
                                     const float *stats, const float *entropy,
                                     const float *grad_logprobs, const float *grad_lse,
                                     const float *grad_entropy, float inv_temperature, void *grad,
                                     int64_t grad_stride, void *stream);

/*
 * sbw_top_candidates -- the k largest logits of every row, in order.
 *
 *   v_offset     token id of column 0 (a vocabulary shard): ids are v_offset + column, as for
 *                the _shard calls of sbw.h.
 *   k            1 <= k <= 1024 (less: SBW_ERR_INVALID_ARG, more: SBW_ERR_UNSUPPORTED).
 *   ids          device, [B, k] int32, written.  Places beyond V hold -1, which
 *                sbw_watermark_candidates ignores.
 *   values       device, [B, k] float, written (may be NULL): the logits, bf16 widened exactly;
 *                a zero comes back as +0, places beyond V hold -inf.
 *   workspace    device, sbw_top_candidates_workspace(B, V, k) uint64 elements.
 */
sbw_status_t sbw_top_candidates(const void *logits, sbw_dtype_t dtype, int64_t B, int64_t V,
                                int64_t row_stride, int64_t v_offset, int64_t k, int32_t *ids,
                                float *values, uint64_t *workspace, void *stream);

/*
 * sbw_head_logits -- logits[b, v] = sum_c hidden[b, c] * scales[v, c / group] * (q[v, c] - 8),
 * with 4-bit q[v, c]: the low half of byte codes[v * K/2 + c/2] for even c, the high half for odd.
 *
 *   hidden       device, [B, hidden_stride] bfloat16, hidden_stride >= K.  A row that holds an
 *                infinity or NaN gives NaN logits; so may one with a magnitude of 2^115 or more, whose
 *                sums on the way pass fp32's range.
 *   B            rows; the weights are read once for every 16 of them.
 *   K            length of a hidden state: a multiple of group, 0 < K <= 8192 (0 or not a
 *                multiple: SBW_ERR_INVALID_ARG; beyond 8192: SBW_ERR_UNSUPPORTED).
 *   codes        device, [V, K/2] bytes.   V: the head's rows, a vocabulary or a shard of one.
 *   scales       device, [V, K/group] of scale_dtype (fp32 or bf16).
 *   group        32, 64 or 128 (else SBW_ERR_UNSUPPORTED).
 *   logits       device, [B, row_stride] of dtype (fp32 or bf16, rounded once), written for
 *                v < V.
 * Products are exact in fp32 and summed in fp32; a group's sum is scaled in fp32.
 */
sbw_status_t sbw_head_logits(const void *hidden, int64_t B, int64_t K, int64_t hidden_stride,
                             const uint8_t *codes, const void *scales, sbw_dtype_t scale_dtype,
                             int64_t group, int64_t V, void *logits, sbw_dtype_t dtype,
                             int64_t row_stride, void *stream);

/*
 * sbw_sample_tokens -- one token of every row, drawn from what the filters keep of softmax(logits * inv_temperature).
 * In the order of logits, with the weights e_v = exp((logits_v - largest) * inv_temperature):
 *     top-k   the first top_k logits;
 *     top-p   of those the ones before which the weights sum to less than top_p times the sum over all of them,
 *             the first at least;
 *     min-p   of those the ones with e_v >= min_p.
 * The token is the one of the largest logits_v * inv_temperature + G_v (rounded in fp32 twice, the lower column of equal
 * ones), G_v the noise of sbw_watermark_sample for column v under the row's seed: without filters it is that
 * call's token with gamma = 0.  Sums of weights are made in one order, or of whole numbers: the same call gives the same
 * answer.  Weights and their sums hold as many bits as fp32 at least, tails of small weights among them, which decides for a
 * logit that ends just where top-p does.
 * A row with a NaN or +inf gives the first column of the order and NaN; one of -inf alone column 0 and -inf.
 *
 *   seeds            device, [B] uint64.
 *   inv_temperatures device, [B] float, or NULL: inv_temperature for all rows (finite and > 0, else
 *                    SBW_ERR_INVALID_ARG; a row whose own is not gives token -1 and NaN).
 *   top_ks           device, [B] int32, or NULL: top_k for all rows.  0 and less, V and more keep all.
 *   top_ps, min_ps   device, [B] float each, or NULL: top_p and min_p for all rows (not NaN, else
 *                    SBW_ERR_INVALID_ARG).  top_p keeps all from 1 on (or NaN) and the first alone up to 0, min_p all up
 *                    to 0 (or NaN); a min_p beyond 1 is 1.
 *   tokens           device, [B] int32, written.
 *   logprobs         device, [B] float, written (may be NULL): the token's log probability among the kept.
 *   workspace        device, sbw_sample_tokens_workspace(B, V) uint64 elements, caller-owned; contents on entry do
 *                    not matter.  Calls that share one must be ordered.
 */
int64_t sbw_sample_tokens_workspace(int64_t B, int64_t V);
sbw_status_t sbw_sample_tokens(const void *logits, sbw_dtype_t dtype, int64_t B, int64_t V, int64_t row_stride,
                               const uint64_t *seeds, const float *inv_temperatures, float inv_temperature,
                               const int32_t *top_ks, int64_t top_k, const float *top_ps, float top_p,
                               const float *min_ps, float min_p, int32_t *tokens, float *logprobs,
                               uint64_t *workspace, void *stream);

/* Kinds of scales of an 8-bit matrix. */
typedef enum SBW_ENUM_TYPE {
    SBW_SCALE_E8M0 = 0,     /* a power of two: one byte e for 2^(e - 127)  */
    SBW_SCALE_F32 = 1       /* any positive binary32 number               */
} sbw_scale_t;

/*
 * sbw_quantize_fp8 -- a matrix as e4m3 codes (OCP: 448 the largest, no infinity) with a scale for each block of
 * block_rows x 128 elements (those at the ends may be smaller), and the same of its transpose, whose blocks lie
 * along its own rows.  With a the largest finite magnitude of a block (0 if there is none)
 *     E8M0   scale = the smallest 2^e, -127 <= e, with a <= 448 * 2^e
 *     F32    scale = max(a / 448, 2^-126), rounded to binary32
 *     code   = the element times 1 / scale (both rounded to binary32; exact for E8M0), rounded to the nearest
 *              e4m3 value, ties to even.  An infinity or NaN becomes NaN.
 *
 *   x            device, [M, row_stride] of dtype, element (m, k) for k < K; read once.
 *   block_rows   1 or 128 (else SBW_ERR_UNSUPPORTED).
 *   codes        device, [M, codes_stride] bytes, written for k < K, or NULL.  scales: device,
 *                [ceil(M / block_rows), ceil(K / 128)] bytes or float, written (NULL exactly when codes is).
 *   codes_t      device, [K, codes_t_stride] bytes, written for m < M, or NULL.  scales_t: device,
 *                [ceil(K / block_rows), ceil(M / 128)].  Both codes and codes_t NULL is SBW_ERR_INVALID_ARG.
 */
sbw_status_t sbw_quantize_fp8(const void *x, sbw_dtype_t dtype, int64_t M, int64_t K, int64_t row_stride,
                              int64_t block_rows, sbw_scale_t scale_type, uint8_t *codes, int64_t codes_stride,
                              void *scales, uint8_t *codes_t, int64_t codes_t_stride, void *scales_t,
                              void *stream);

/*
 * sbw_matmul_fp8 -- out[m, n] = sum_k a(m, k) * b(n, k) of two matrices of e4m3 codes with scales, as
 * sbw_quantize_fp8 writes them: a(m, k) = a[m * a_stride + k] * a_scales[m / a_block_rows, k / 128].
 * An fp32 result is made of exact products and fp32 sums.  For a bf16 one each product may be cut off 13 bits below
 * the power of two of the largest of its eight neighbours (columns 8 i .. 8 i + 7) on its way into the fp32 sum.
 * The product of two blocks' scales is to lie in fp32's range.  out is rounded once.
 *
 *   a, b         device, [M, a_stride] and [N, b_stride] bytes, K columns of each row; strides < 2^23.  Where both start
 *                at multiples of 16 with strides that are, bytes that share an aligned 16 with a row's last
 *                columns are read too, and have no effect.
 *   a_scales, b_scales   device, [ceil(M / a_block_rows), ceil(K / 128)] and [ceil(N / b_block_rows),
 *                ceil(K / 128)], both of scale_type; block_rows 1 or 128.
 *   K            > 0 (else SBW_ERR_INVALID_ARG).  M < 2^23 - 128, N < 2^30, and fewer than 2^24 tiles of 128 x 128 (else
 *                SBW_ERR_UNSUPPORTED).
 *   out          device, [M, out_stride] of dtype (fp32 or bf16), written for n < N.
 *   workspace    device, sbw_matmul_fp8_workspace(M, N, K) uint64 elements (may be NULL where that is 0).
 */
int64_t sbw_matmul_fp8_workspace(int64_t M, int64_t N, int64_t K);
sbw_status_t sbw_matmul_fp8(const uint8_t *a, int64_t M, int64_t a_stride, const void *a_scales,
                            int64_t a_block_rows, const uint8_t *b, int64_t N, int64_t b_stride,
                            const void *b_scales, int64_t b_block_rows, int64_t K, sbw_scale_t scale_type,
                            void *out, sbw_dtype_t dtype, int64_t out_stride, uint64_t *workspace, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* SBW_STEP_H */
