/*
 * misample — the pick of a token from rows of logits on AMD Instinct MI355X
 * (gfx950), part of libmiconv: what a decoder answers with.
 *
 * Conventions as in miquant.h: device pointers owned by the caller, `stream` a
 * hipStream_t as void*, calls that validate their scalar arguments, enqueue
 * kernels and return, a caller-owned workspace, 0 or a negative miconv_status,
 * the same bits for the same inputs.
 */
#ifndef MISAMPLE_H
#define MISAMPLE_H

#include <stddef.h>
#include <stdint.h>

#pragma GCC visibility push(default)

#ifdef __cplusplus
extern "C" {
#endif

/* Draws a token of each row of logits x [rows][vocab] (dtype: 0 = fp32, 1 =
 * bf16; rows `stride` elements apart).  With the row's temperature t and m its
 * largest logit a token's weight is exp((x - m) / t).  Of the tokens in the order
 * of their logits, the largest first and of equal ones (-0 and 0 are equal) the
 * lowest index, those are kept that are
 *   top_k: among the first k                    (k < 1 or >= vocab: all)
 *   top_p: behind tokens of less than p times the weight of those first k, or
 *          the first one                        (p >= 1 or NaN: all)
 *   min_p: of at least the weight min_p, or the first one   (NaN: all)
 * The token drawn is the first in the vocabulary's order at which the weights of
 * the tokens kept, added up in that order, pass u times their sum; logprob is the
 * logarithm of its share of that sum.
 * u fp32 [rows] in 0 <= u < 1: smaller ones and NaN count as 0, larger ones as the
 * largest below 1.  temperature fp32 [rows], top_k int32 [rows], top_p fp32 [rows],
 * min_p fp32 [rows]: NULL for temperature 1 and no filter.  A temperature that is
 * not above 0 (NaN too) draws the first token, with logprob 0.  Minus infinity is
 * the logit of a token that is never drawn.  A row that holds a NaN or an
 * infinity, or nothing but minus infinities, gives token -1 and logprob NaN.
 * Weights are held in 64 bits as whole multiples of a power of two of the largest
 * one, 2^-37 at 2^25 tokens and finer for fewer (2^-45 at 2^17, 2^-51 at most), and
 * added exactly.
 * token int32 [rows]; logprob fp32 [rows] or NULL.
 * Errors: MICONV_ERR_NULL (x, u or token), MICONV_ERR_SHAPE (rows < 0, vocab < 1,
 * stride < vocab), MICONV_ERR_UNSUPPORTED (dtype), MICONV_ERR_ALIGN,
 * MICONV_ERR_TOO_LARGE (vocab > 2^25, rows >= 2^22), MICONV_ERR_WORKSPACE. */
long sample_tokens_workspace_bytes(long rows, long vocab, int dtype);
int sample_tokens(long rows, long vocab, int dtype, const void *x, long stride, const float *u,
                  const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p,
                  int32_t *token, float *logprob, void *ws, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#pragma GCC visibility pop

#endif /* MISAMPLE_H */
