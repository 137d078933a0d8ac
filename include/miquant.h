/*
 * miquant — the operators of a transformer block served in few bits on AMD
 * Instinct MI355X (gfx950), part of libmiconv: activations as 8-bit integers
 * with a scale for each token, weights as 8-bit integers with a scale for each
 * output channel, the keys and values of past tokens in 4 bits; or all of them
 * as 8-bit floats in blocks that share a power of two.
 *
 * Conventions (as in miconv.h)
 *  - Tensor pointers are DEVICE pointers owned by the caller; the library
 *    never frees them.  `stream` is a hipStream_t passed as void* (NULL = the
 *    default stream).  Calls validate their scalar arguments, enqueue kernels
 *    and return; they never allocate, free or synchronise, so every call can
 *    be captured into a HIP graph.  Scratch memory comes from a caller-owned
 *    workspace (`ws`, at least the bytes the matching *_workspace_bytes call
 *    reports, 256-byte aligned; it may be NULL when that is 0).
 *  - Return 0 (MICONV_OK) or a negative miconv_status (miconv.h); on a
 *    validation error nothing is enqueued.  Device-side data (slots, page
 *    tables, lengths, offsets) is not validated: the kernels clamp every index
 *    they derive from it, so bad data gives wrong results, never an access
 *    outside the buffers.
 *  - Rows are dense; the distance between rows is a stride in elements, at
 *    least the row's length.  dtype: 0 = fp32, 1 = bf16.  Pointers are aligned
 *    to their element; wider alignment (16 bytes, strides to match) is faster.
 *  - Zero rows, tokens or sequences: the call does nothing and returns
 *    MICONV_OK.
 *  - Results do not depend on the order in which work-groups run: a call on
 *    the same inputs gives the same bits.
 */
#ifndef MIQUANT_H
#define MIQUANT_H

#include <stddef.h>
#include <stdint.h>

#pragma GCC visibility push(default)

#ifdef __cplusplus
extern "C" {
#endif

/* Root-mean-square norm of each row, with the residual's addition before it
 * and an 8-bit output:
 *   h = x + residual, rounded to dtype (h = x without a residual)
 *   t = h * weight                     (fp32; weight NULL: t = h)
 *   A = max |t|,  q = rint(t * (127 / A)),  scale = A / sqrt(mean(h^2) + eps) / 127
 * so that q * scale is the normed row.  The norm's factor cancels out of q:
 * q is the same whatever the order of a sum.  A row with A < 2^-100 gets
 * q = 0 and scale 0; a row that holds a NaN or an infinity (or whose t
 * overflows) gets q = 0 and scale NaN.
 * x, residual, h: [rows][cols] of dtype; weight: fp32 [cols]; q: int8
 * [rows][cols]; scale: fp32 [rows].  h is given exactly when residual is, and
 * may be residual or x itself; nothing else may overlap.
 * Errors: MICONV_ERR_NULL, MICONV_ERR_SHAPE (rows < 0, cols < 1, a stride
 * below cols, eps negative or NaN), MICONV_ERR_UNSUPPORTED (dtype),
 * MICONV_ERR_ALIGN, MICONV_ERR_TOO_LARGE (rows or cols >= 2^31). */
int quant_rmsnorm_i8(long rows, long cols, int dtype, const void *x, long x_stride, const void *residual,
                     long residual_stride, const float *weight, float eps, void *h, long h_stride, int8_t *q,
                     long q_stride, float *scale, void *stream);

/* The 8-bit output alone: A = max |x|, q = rint(x * (127 / A)), scale =
 * A / 127, with the rules above. */
int quant_rows_i8(long rows, long cols, int dtype, const void *x, long x_stride, int8_t *q, long q_stride,
                  float *scale, void *stream);

/* y[m][n] = act(a_scale[m] * w_scale[n] * sum_k a[m][k] * w[n][k] + bias[n] + residual[m][n])
 * with a int8 [M][K], w int8 [N][K] (an output channel's weights in a row),
 * fp32 scales, fp32 bias [N] or NULL, residual [M][N] of y's type or NULL (it
 * may be y itself), y [M][N] of out_dtype, act = ReLU when relu != 0.  The sum
 * is an exact 32-bit integer; the rest is fp32, rounded once to out_dtype.
 * An operand whose rows are not 16-byte aligned (pointer, stride and K all
 * multiples of 16), or are 2^23 or more bytes apart, is first copied to the
 * workspace in rows that are aligned and dense; without one that needs it, no
 * workspace is used.  Weights kept in aligned rows save their copy.
 * Errors: MICONV_ERR_NULL, MICONV_ERR_SHAPE (M < 0, N or K < 1, a stride below
 * its row), MICONV_ERR_UNSUPPORTED (out_dtype), MICONV_ERR_ALIGN,
 * MICONV_ERR_TOO_LARGE (K > 131071, where the sum could pass 32 bits; M or
 * N > 2^31 - 256; so many outputs that a grid does not hold them, or 2^35 bytes
 * of rows to copy), MICONV_ERR_WORKSPACE. */
long quant_matmul_workspace_bytes(long M, long N, long K, const int8_t *a, long a_stride, const int8_t *w,
                                  long w_stride);
int quant_matmul_i8(long M, long N, long K, const int8_t *a, long a_stride, const float *a_scale, const int8_t *w,
                    long w_stride, const float *w_scale, const float *bias, const void *residual,
                    long residual_stride, int out_dtype, void *y, long y_stride, int relu, void *ws,
                    size_t ws_bytes, void *stream);

/* The kernels (as a profiler prints them, "a + b" for two launches) and the
 * number of launches of a call; buf is cut at buflen.  Nothing is launched, and
 * of the operands only the addresses matter.
 * Errors: those of the call, and MICONV_ERR_NULL for buf or launches. */
int quant_matmul_describe(long M, long N, long K, const int8_t *a, long a_stride, const int8_t *w, long w_stride,
                          int out_dtype, char *buf, int buflen, int *launches);

/* A paged cache of keys and values in 4 bits.  Along a head's channels every
 * 32 values share a power of two, 2^(byte - 127); a value is four bits, sign
 * then the index of 0, .5, 1, 1.5, 2, 3, 4, 6, two to a byte, the lower
 * channel in the lower bits.  Codes: uint8 [pages][heads][page_size]
 * [head_dim / 2]; exponents: uint8 [pages][heads][page_size][head_dim / 32].
 * A slot is page * page_size + place in the page.  An exponent byte above 252
 * stands for a group that is not finite, and reads as NaN.
 * head_dim: 32, 64, 96, 128, 192 or 256.  Codes are 16-byte aligned. */
typedef struct quant_kv4 {
    void *k_codes, *k_exps, *v_codes, *v_exps;
    long pages;
    int heads, page_size, head_dim;
} quant_kv4;

/* Writes tokens to the cache: token i's keys and values ([heads][head_dim] of
 * dtype at k + i * k_stride, v + i * v_stride) to slots[i]; a slot outside the
 * cache (a negative one, say) is skipped.  Slots of one call are distinct.
 * A group's exponent is the smallest e in -126 .. 125 with max|x| <= 7 * 2^e
 * (what lies above 6 * 2^e becomes 6 * 2^e, off by no more than the steps
 * between 4 and 6 allow), its values the nearest, ties to the even code.  A
 * group that holds a NaN or an infinity gets exponent byte 255 and codes 0.
 * Errors: MICONV_ERR_NULL, MICONV_ERR_SHAPE, MICONV_ERR_UNSUPPORTED (dtype,
 * head_dim), MICONV_ERR_ALIGN, MICONV_ERR_TOO_LARGE (2^31 slots, more than 2^25
 * tokens). */
int quant_kv4_write(const quant_kv4 *cache, long tokens, int dtype, const void *k, long k_stride, const void *v,
                    long v_stride, const int32_t *slots, void *stream);

/* Reads tokens back: the values at slots[i] into k + i * k_stride and
 * v + i * v_stride, of dtype (each is exact in bf16); zeros for a slot outside
 * the cache.  Errors as quant_kv4_write. */
int quant_kv4_read(const quant_kv4 *cache, long tokens, const int32_t *slots, int dtype, void *k, long k_stride,
                   void *v, long v_stride, void *stream);

/* Attention of new tokens over the cache, which holds them already.
 * Sequence s has lens[s] cached tokens, the token at place t in slot
 * table[s * table_stride + t / page_size] * page_size + t % page_size, and
 * queries at rows starts[s] .. starts[s + 1] of q (starts NULL: row s alone);
 * query i of n stands at place p = lens[s] - n + i.  It sees the places
 * 0 .. p (0 .. lens[s] - 1 unless causal), of these with window > 0 only those
 * above p - window.  max_new and max_len bound the queries and the places of any
 * sequence: rows past max_new are not computed, and places past max_len (or the
 * table's end) are not seen; where lens[s] passes these, the queries keep their
 * places.  For each of the `heads` query heads, head j reading key head
 * j / (heads / cache->heads):
 *   out = softmax(scale * q k^T over the places seen) v
 * zeros where none is seen, NaN where a key or value that is seen is not
 * finite; what is not seen never reaches the result.
 * q, out: bf16 [tokens][heads][head_dim], rows q_stride / out_stride elements
 * apart.  Scores, softmax statistics and sums are fp32: queries are finite and
 * scores within fp32's range, values below 2^90 (the sums hold up to 2^8 times a
 * value for each place).  For the matrix cores the probabilities are rounded to
 * bf16, and the sum they are divided by is that of the rounded ones; where a key
 * head has few query rows (64, 32 or 16 of head_dim 64, 128 or more) they keep a
 * second bf16 part, 16 bits in all.
 * Errors: MICONV_ERR_NULL, MICONV_ERR_SHAPE (heads no multiple of the cache's,
 * a stride below its row, max_new or max_len < 1, table_stride < 1, a scale that
 * is not finite, also times log2(e)), MICONV_ERR_UNSUPPORTED (head_dim),
 * MICONV_ERR_ALIGN, MICONV_ERR_TOO_LARGE (2^31 slots, 2^31 rows of heads in a
 * page, a max_len of 2^30, 2^16 sequences or heads, 2^24 query rows of a key
 * head, or so much work that a grid does not hold it), MICONV_ERR_WORKSPACE. */
long quant_attention_workspace_bytes(const quant_kv4 *cache, int seqs, int heads, int max_new, int max_len,
                                     int causal, int window);
int quant_attention_kv4(const quant_kv4 *cache, int seqs, int heads, long tokens, const void *q, long q_stride,
                        const int32_t *starts, const int32_t *lens, const int32_t *table, int table_stride,
                        int max_new, int max_len, float scale, int causal, int window, void *out, long out_stride,
                        void *ws, size_t ws_bytes, void *stream);
/* The kernels of a call, as quant_matmul_describe names them. */
int quant_attention_describe(const quant_kv4 *cache, int seqs, int heads, int max_new, int max_len, int causal,
                             int window, char *buf, int buflen, int *launches);

/* ---- 8-bit floating point in blocks ----
 *
 * A value is an e4m3 code (sign, four bits of exponent with bias 7, three of
 * mantissa; no infinities, 0x7F and 0xFF are NaN, the largest is 448) times a
 * power of two that its block shares, 2^(byte - 127).  The exponent e = byte -
 * 127 of a block that is written is the smallest in -117 .. 119 with max|x| <=
 * 448 * 2^e (values above 448 * 2^119 become that), its values the nearest, ties
 * to even; each is exact in bf16 and fp32. */

/* Root-mean-square norm of each row, with the residual's addition before it
 * and an output in blocks of 128 values of a row:
 *   h = x + residual, rounded to dtype (h = x without a residual)
 *   t = h * weight                     (fp32; weight NULL: t = h)
 *   q, exps = t in blocks,  scale = 1 / sqrt(mean(h^2) + eps)
 * so that the value of q times scale is the normed row.  The norm's factor
 * stays out of the blocks: q and exps do not depend on the order of a sum.
 * A block that holds a NaN or an infinity gets exponent byte 255 and values 0;
 * the scale of a row whose h does is NaN.  A factor beyond fp32's largest number
 * becomes that number (a row of zeros with eps = 0, say).
 * x, residual, h: [rows][cols] of dtype; weight: fp32 [cols]; q: e4m3
 * [rows][cols]; exps: uint8 [rows][blocks], blocks = cols / 128 rounded up;
 * scale: fp32 [rows].  h is given exactly when residual is, and may be residual
 * or x itself; nothing else may overlap.
 * Errors: as quant_rmsnorm_i8, with exps. */
int quant_rmsnorm_f8(long rows, long cols, int dtype, const void *x, long x_stride, const void *residual,
                     long residual_stride, const float *weight, float eps, void *h, long h_stride, void *q,
                     long q_stride, uint8_t *exps, long exps_stride, float *scale, void *stream);

/* The 8-bit output of x alone, with the rules above. */
int quant_rows_f8(long rows, long cols, int dtype, const void *x, long x_stride, void *q, long q_stride,
                  uint8_t *exps, long exps_stride, void *stream);

/* y[m][n] = act(a_scale[m] * sum_k a[m][k] * w[n][k] + bias[n] + residual[m][n])
 * of the values of a and w: e4m3 [M][K] and [N][K] (an output channel's weights
 * in a row) with exponents uint8 [M][blocks] and [N][blocks], blocks = K / 128
 * rounded up; a_scale fp32 [M] or NULL (1), fp32 bias [N] or NULL, residual
 * [M][N] of y's type or NULL (it may be y itself), y [M][N] of out_dtype, act =
 * ReLU when relu != 0.  Sums are fp32; a product whose powers of two pass fp32's
 * range is infinite or 0.  For bf16 outputs the matrix cores cut each of eight
 * products that they add at a time (k = 8i .. 8i + 7) to a multiple of 2^-13 of
 * the largest one's power of two; for fp32 outputs every product counts in full.
 * A NaN, or an exponent byte of 255, makes NaN of every output that it reaches;
 * exponent bytes other than that and those written, 10 to 246, may lose values.
 * Operands whose rows are not 16-byte aligned or far apart are copied to the
 * workspace first, as quant_matmul_i8 does.
 * Errors: MICONV_ERR_NULL, MICONV_ERR_SHAPE (M < 0, N or K < 1, a stride below
 * its row), MICONV_ERR_UNSUPPORTED (out_dtype), MICONV_ERR_ALIGN,
 * MICONV_ERR_TOO_LARGE (K > 2^23 - 16; M or N > 2^31 - 256; so many outputs that
 * a grid does not hold them, or 2^35 bytes of rows to copy),
 * MICONV_ERR_WORKSPACE. */
long quant_matmul_f8_workspace_bytes(long M, long N, long K, const void *a, long a_stride, const void *w,
                                     long w_stride);
int quant_matmul_f8(long M, long N, long K, const void *a, long a_stride, const uint8_t *a_exps, long a_exps_stride,
                    const float *a_scale, const void *w, long w_stride, const uint8_t *w_exps, long w_exps_stride,
                    const float *bias, const void *residual, long residual_stride, int out_dtype, void *y,
                    long y_stride, int relu, void *ws, size_t ws_bytes, void *stream);
/* The kernels of a call, as quant_matmul_describe names them, whose exponents' rows lie less than 2^23 bytes apart. */
int quant_matmul_f8_describe(long M, long N, long K, const void *a, long a_stride, const void *w, long w_stride,
                             int out_dtype, char *buf, int buflen, int *launches);

/* A paged cache of keys and values in 8 bits: e4m3 [pages][heads][page_size]
 * [head_dim] and exponents uint8 [pages][heads][page_size / block], for keys and
 * for values: `block` places of a page that follow one another share a power of
 * two in each head.  block divides page_size and is 256 at most.
 * A token whose keys or values of a head hold a NaN or an infinity is held with
 * NaN for its keys there and 0 for its values, and counts nothing to the
 * exponents.  An exponent byte above 246 is never written, nor a code of values
 * that is no number.  A cache that is filled by other means has to keep to that:
 * what attention makes of rows that see such a code is NaN in some tiles and
 * finite in others.
 * head_dim: 32, 64, 96, 128, 192 or 256.  Codes are 16-byte aligned. */
typedef struct quant_kv8 {
    void *k_codes, *k_exps, *v_codes, *v_exps;
    long pages;
    int heads, page_size, head_dim, block;
} quant_kv8;

/* Writes the new tokens of sequences to the cache.  Sequence s has lens[s]
 * tokens, the new ones among them, at the places of quant_attention_kv8; its new
 * ones are rows starts[s] .. starts[s + 1] of k and v ([heads][head_dim] of dtype
 * at k + i * k_stride, v + i * v_stride; starts NULL: row s alone), rows past
 * max_new not written, nor places before 0, past the table's end, or in a page
 * outside the cache.
 * The places of a block before the first new one are held: where the new
 * tokens need a larger exponent than the block has, the values held are rounded
 * again to the new one.  A block whose first place is new begins anew, whatever
 * it held; what lies behind the last token stays as it is.
 * No two sequences of a call may write to the same page.
 * Errors: MICONV_ERR_NULL, MICONV_ERR_SHAPE (max_new or table_stride < 1, a
 * stride below its row, page_size no multiple of block), MICONV_ERR_UNSUPPORTED
 * (dtype, head_dim, block), MICONV_ERR_ALIGN, MICONV_ERR_TOO_LARGE (2^31 slots
 * or tokens, 2^16 sequences or heads, 2^31 rows of heads in a page, so many
 * blocks that a grid does not hold them). */
int quant_kv8_write(const quant_kv8 *cache, int seqs, long tokens, int dtype, const void *k, long k_stride,
                    const void *v, long v_stride, const int32_t *starts, const int32_t *lens, const int32_t *table,
                    int table_stride, int max_new, void *stream);

/* Reads tokens back: the values at slots[i] (page * page_size + place in the
 * page) into k + i * k_stride and v + i * v_stride, of dtype (each is exact in
 * bf16); zeros for a slot outside the cache.  Errors as quant_kv4_read. */
int quant_kv8_read(const quant_kv8 *cache, long tokens, const int32_t *slots, int dtype, void *k, long k_stride,
                   void *v, long v_stride, void *stream);

/* Attention of new tokens over the 8-bit cache, which holds them already: as
 * quant_attention_kv4 in every argument, place, mask, result, rounding and
 * error.  A row that sees a token that was written with keys or values that are
 * not finite is NaN. */
long quant_attention_kv8_workspace_bytes(const quant_kv8 *cache, int seqs, int heads, int max_new, int max_len,
                                         int causal, int window);
int quant_attention_kv8(const quant_kv8 *cache, int seqs, int heads, long tokens, const void *q, long q_stride,
                        const int32_t *starts, const int32_t *lens, const int32_t *table, int table_stride,
                        int max_new, int max_len, float scale, int causal, int window, void *out, long out_stride,
                        void *ws, size_t ws_bytes, void *stream);
/* The kernels of a call, as quant_matmul_describe names them. */
int quant_attention_kv8_describe(const quant_kv8 *cache, int seqs, int heads, int max_new, int max_len, int causal,
                                 int window, char *buf, int buflen, int *launches);

#ifdef __cplusplus
}
#endif

#pragma GCC visibility pop

#endif /* MIQUANT_H */
