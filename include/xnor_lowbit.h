/*
 * libxnor — the real layers around a network's binary blocks, in few bits.
 *
 * XNOR-Net leaves a network's first and last layers real (sec. 4.1).  These calls run what stands there: the residual's addition
 * and the root-mean-square norm with 8-bit outputs, products with 4-bit weights under group scales, and the log probabilities of
 * the answer; in 8 bits the products, activation functions that keep their input for the backward pass, the gradients of weights, and
 * tokens drawn from the answer.  The conventions are those of xnor.h (device pointers that the caller owns, 16-byte aligned; enqueued on hip_stream
 * without synchronising; nothing is allocated or kept; an xnor_status comes back, arguments are checked before anything is
 * launched), with these additions:
 *  - Real tensors hold one xnor_dtype; sums, norms and statistics are held in float32 whatever it is, and a result is rounded
 *    once, to nearest even.
 *  - Rows that a call only reads may lie apart: `..._stride` is the distance of two rows in elements, at least their width.
 *    Everything else is densely packed.  Rows need no alignment of their own.
 *  - Sizes go up to rows = 65535 * 64, in = out = 2^24, vocab = 2^30 (the backward pass of logprobs: rows * ceil(vocab / 8192) < 2^24);
 *    beyond them and below 1 (rows: 0): XNOR_ERR_SHAPE.
 *  - rows = 0 is a call without work: XNOR_OK, nothing is launched and no pointer is looked at.
 *  - Where two kernels are enqueued, the first may be when the second reports XNOR_ERR_HIP; it writes that call's own outputs or
 *    workspace only.  A workspace's contents are undefined afterwards, and nothing in it has to be cleared before.
 *  - What a ..._workspace_bytes call says never falls as rows grows: a workspace for more rows serves fewer rows of the same other sizes.
 */
#ifndef XNOR_LOWBIT_H
#define XNOR_LOWBIT_H

#include "xnor.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    XNOR_F32 = 0,
    XNOR_BF16 = 1,
    XNOR_F16 = 2
} xnor_dtype;

/*
 * Residual addition, root-mean-square norm and 8-bit rounding of rows:
 *     h = x + residual                                  float32 (residual NULL: h = x);  sum_out = h in `type`
 *     rstd = 1 / sqrt(mean_j h_j^2 + eps)
 *     t = h * weight                                    (weight NULL: t = h)
 *     per row and group of neighbouring columns:        top = max |t|
 *         q = round(t * (127 / top)), halves to even;   scale = top * rstd / 127
 *     values = q * scale, in `type`                     what the 8 bits stand for: h * rstd * weight to half a scale
 * q depends on no sum: it is the same integer whatever order the mean was added in.
 *   x, residual  in   `type` [rows][cols], apart by x_stride and residual_stride (ignored without residual)
 *   weight       in   (nullable) float32 [cols]
 *   sum_out      out  (nullable) `type` [rows][cols]; may be x or residual itself where that is dense
 *   q            out  (nullable) int8 [rows][cols]
 *   scale        out  float32 [rows][groups], groups = ceil(cols / group) (1 where group is 0); may be NULL without q
 *   values       out  (nullable) `type` [rows][cols]
 *   rstd         out  (nullable) float32 [rows]
 *   group             0 (one scale for the whole row), 32, 64 or 128 columns; the last group of a row may be shorter
 *   eps               > 0 and finite
 * One of q and values is required.  A group whose top is below 2^-100 is q = 0 with scale 0; one that holds an infinity or a NaN
 * is q = 0 with scale NaN, and so are all groups of a row that holds a NaN.  An infinity elsewhere in the row makes rstd, and so
 * the scale, 0 (so does a sum of squares beyond float32's range).  cols <= 32768, XNOR_ERR_UNSUPPORTED otherwise.
 */
XNOR_API int xnor_rmsnorm_q8(const void *x, int64_t x_stride, const void *residual, int64_t residual_stride, const float *weight,
                             void *sum_out, int8_t *q, float *scale, void *values, float *rstd, int rows, int cols, int group,
                             int type, float eps, void *hip_stream);

/*
 * Backward pass of the norm, straight through the rounding to 8 bits (as sec. 3.1 does for sign): with n = h * rstd
 *     g_h = rstd * (w * g_values - n * mean_j(w_j * g_values_j * n_j)) + g_sum,     g_weight = sum over rows of g_values * n
 * g_h is the gradient of x and of residual alike.
 *   h          in   `type` [rows][cols], apart by h_stride: sum_out of the forward pass (x, where there was no residual)
 *   rstd       in   float32 [rows], of the forward pass
 *   weight     in   (nullable) float32 [cols]
 *   g_values   in   `type` [rows][cols], apart by g_stride
 *   g_sum      in   (nullable) `type` [rows][cols], apart by g_sum_stride: the gradient that reaches sum_out by itself
 *   g_h        out  `type` [rows][cols]; may be g_sum or g_values itself where that is dense
 *   g_weight   out  (nullable) float32 [cols]; the rows are added in an order that the sizes alone decide
 *   workspace       xnor_rmsnorm_backward_workspace_bytes(rows, cols) bytes, required with g_weight
 * With rows = 0 g_weight is written (zeros).
 */
XNOR_API size_t xnor_rmsnorm_backward_workspace_bytes(int rows, int cols);
XNOR_API int xnor_rmsnorm_backward(const void *h, int64_t h_stride, const float *rstd, const float *weight, const void *g_values,
                                   int64_t g_stride, const void *g_sum, int64_t g_sum_stride, void *g_h, float *g_weight,
                                   void *workspace, int rows, int cols, int type, void *hip_stream);

/*
 * 4-bit weights: output o's weights are w[o][k] = scale[o][g] * (u[o][k] - zero[o][g]), u and zero in 0..15, g = k / group.
 *   codes  uint8 [out][16 * ceil(in / 32)]: two to a byte, the even input in the low half; what is past `in` counts as nothing
 *   scale  float32 [out][ceil(in / group)]     zero  (nullable: 8 everywhere) uint8 [out][ceil(in / group)]
 *   group  32, 64 or 128 inputs; the last group of a row may be shorter
 * xnor_w4_quantize  w `type` [out][in], apart by w_stride, finite  ->  codes and scale, and zero where it is given.  Without zero:
 *     scale = max|w| / 7, u = round(w * (7 / max|w|)) + 8.  With it: lo = min(w, 0), hi = max(w, 0), scale = (hi - lo) / 15,
 *     zero = round(-lo * (15 / (hi - lo))), u = round(w * (15 / (hi - lo))) + zero within 0..15.  Halves to even; a group whose
 *     range is below 2^-100 has scale 0.
 * xnor_w4_pack      codes, scale, zero  ->  wimg, xnor_w4_wimg_bytes(out, in, group) bytes (opaque; 0: invalid sizes): what the
 *     products read.  Once per layer.
 */
XNOR_API int xnor_w4_quantize(const void *w, int64_t w_stride, uint8_t *codes, float *scale, uint8_t *zero, int out, int in, int group,
                              int type, void *hip_stream);
XNOR_API size_t xnor_w4_wimg_bytes(int out, int in, int group);
XNOR_API int xnor_w4_pack(const uint8_t *codes, const float *scale, const uint8_t *zero, void *wimg, int out, int in, int group,
                          void *hip_stream);

/*
 * Products of rows with 4-bit weights:  y[r][o] = sum_k x[r][k] w[o][k], summed in float32, rounded once.  A real row's sums hold 16 + u in place of
 * u - zero, and what that adds is taken out group by group, or four groups at a time: roundings are relative to sum |x| 32 scale over four groups.
 *   xnor_w4_linear      x `type` [rows][in], apart by x_stride  ->  y `type` [rows][out].  The products are exact (16-bit rows as they
 *       are, float32 rows as three bfloat16 numbers); a row that holds an infinity or a NaN gives NaN.  Finite rows of
 *       any size do not, where sum |x| scale over four groups is below 2^134 (float16: 2^122); an infinity is then a result beyond the type's range
 *   xnor_w4_linear_q8   q int8 [rows][in] with x_scale float32 [rows][ceil(in / x_group)] (one per row where x_group is 0), as
 *       xnor_rmsnorm_q8 writes them: x = q * x_scale  ->  y `type` [rows][out].  The sums of a group are exact integers.
 *       x_group is 0, 32, 64 or 128, and not below group otherwise (XNOR_ERR_UNSUPPORTED)
 *   wimg        in   from xnor_w4_pack with the same out, in and group
 *   workspace        xnor_w4_linear_workspace_bytes(rows, in, out, group) bytes, may be NULL where that is 0
 * The order of the sums follows from the sizes alone: the same call gives the same bits.
 */
XNOR_API size_t xnor_w4_linear_workspace_bytes(int rows, int in, int out, int group);
XNOR_API int xnor_w4_linear(const void *x, int64_t x_stride, const void *wimg, void *y, void *workspace, int rows, int in, int out,
                            int group, int type, void *hip_stream);
XNOR_API int xnor_w4_linear_q8(const int8_t *q, const float *x_scale, const void *wimg, void *y, void *workspace, int rows, int in,
                               int out, int group, int x_group, int type, void *hip_stream);

/*
 * Log probabilities of given tokens, entropy and the likeliest alternatives of rows of logits, which are read once:
 *     lse = log sum_j exp(l_j),   logprob[i] = l_token[i] - lse,   entropy = -sum_j p_j log p_j with p_j = exp(l_j - lse)
 *   logits       in   `type` [rows][vocab], apart by stride; -inf marks what is masked
 *   tokens       in   int32 or int64 (token_bytes 4 or 8) [rows][given]; one outside 0..vocab-1 is no token: its logprob is 0
 *   logprob      out  float32 [rows][given]; tokens and logprob may be NULL where given is 0
 *   lse          out  (nullable) float32 [rows]
 *   shift        out  (nullable) float32 [rows][2]: the largest logit m and log sum_j exp(l_j - m), whose sum is lse.  The backward pass
 *                     takes both: a float32 lse of large magnitude (all logits at a type's lowest value) would not hold the second
 *   entropy      out  (nullable) float32 [rows]
 *   top_index    out  int32 [rows][top], the largest logits first, of equal ones the lowest index first
 *   top_logprob  out  float32 [rows][top]; both may be NULL where top is 0
 *   workspace         xnor_logprobs_workspace_bytes(rows, vocab, top) bytes, may be NULL where that is 0
 *   given             0 .. 1024;  top  0 .. 32
 * Where fewer than top logits are above -inf, the rest are index -1 and logprob -inf.  A row without any has lse -inf, shift (-inf, 0), entropy 0
 * and logprobs of -inf.  A row that holds a NaN or +inf has NaN statistics and alternatives of index -1 and logprob NaN.
 */
XNOR_API size_t xnor_logprobs_workspace_bytes(int rows, int vocab, int top);
XNOR_API int xnor_logprobs(const void *logits, int64_t stride, const void *tokens, int token_bytes, float *logprob, float *lse, float *shift,
                           float *entropy, int32_t *top_index, float *top_logprob, void *workspace, int rows, int vocab, int given,
                           int top, int type, void *hip_stream);

/*
 * Backward pass of logprob and entropy:
 *     g_logits_j = sum_i g_logprob[i] ([token[i] = j] - p_j) - g_entropy p_j (log p_j + entropy)
 * A masked logit (-inf) has gradient 0, and so has all of a row without any other; what is no token takes no part.  A p below 2^-126 counts
 * as 0.
 *   logits, tokens             in   as above
 *   shift, entropy             in   of the forward pass; entropy may be NULL without g_entropy
 *   g_logprob                  in   (nullable) float32 [rows][given]
 *   g_entropy                  in   (nullable) float32 [rows]; one of the two is required
 *   g_logits                   out  `type` [rows][vocab]; may be logits itself where that is dense
 */
XNOR_API int xnor_logprobs_backward(const void *logits, int64_t stride, const void *tokens, int token_bytes, const float *shift,
                                    const float *entropy, const float *g_logprob, const float *g_entropy, void *g_logits, int rows,
                                    int vocab, int given, int type, void *hip_stream);

/*
 * Rows to 8 bits:  per row and group of neighbouring columns  top = max |x|,  q = round(x * (127 / top)), halves to even,  scale = top / 127
 *   x      in   `type` [rows][cols], apart by x_stride; cols up to 2^24
 *   q      out  int8 [rows][cols]
 *   scale  out  float32 [rows][groups], groups = ceil(cols / group) (1 where group is 0: one scale for the whole row)
 *   group       0, 32, 64 or 128 columns; the last group of a row may be shorter
 * A group whose top is below 2^-100 is q = 0 with scale 0; one that holds an infinity or a NaN is q = 0 with scale NaN.
 * Rows of weights [out][in] with group 0 give what xnor_w8_linear takes as w and w_scale.
 */
XNOR_API int xnor_q8_rows(const void *x, int64_t x_stride, int8_t *q, float *scale, int rows, int cols, int group, int type, void *hip_stream);

/*
 * Products of 8-bit rows with 8-bit weights, a scale for each row and output:
 *     y[r][o] = (sum_k q[r][k] w[o][k]) * (x_scale[r] * w_scale[o]) + bias[o]
 * The sums are exact integers; a result is finite where it is within float32's range, whatever the scales, and one product of the scales is rounded to
 * float32 before the sum is multiplied by it.
 *   q        in   int8 [rows][in] with x_scale float32 [rows]: as xnor_q8_rows, xnor_rmsnorm_q8 and xnor_activation_q8 write them with group 0
 *   w        in   int8 [out][in] with w_scale float32 [out]
 *   bias     in   (nullable) float32 [out]
 *   y        out  `type` [rows][out]
 *   workspace     xnor_w8_linear_workspace_bytes(rows, in, out) bytes, may be NULL where that is 0
 * in <= 131071 (sums within 32 bits), XNOR_ERR_UNSUPPORTED otherwise.  From 2^23 tiles of 256 x 256 results on (2^39 of them, more than the memory holds): XNOR_ERR_SHAPE.
 */
XNOR_API size_t xnor_w8_linear_workspace_bytes(int rows, int in, int out);
XNOR_API int xnor_w8_linear(const int8_t *q, const float *x_scale, const int8_t *w, const float *w_scale, const float *bias, void *y, void *workspace,
                            int rows, int in, int out, int type, void *hip_stream);

/*
 * Activation functions, whose input is kept in 8 bits for the backward pass and whose values may go to the next product in 8 bits:
 *     a = f(x)                                    gated 0: x [rows][cols]
 *     a = f(x[:, :cols]) * x[:, cols:]            gated 1: x [rows][2 cols]
 *     f: XNOR_RELU max(x, 0);  XNOR_GELU x Phi(x), Phi the normal distribution;  XNOR_SILU x / (1 + exp(-x));  in float32
 *   x           in   `type` [rows][cols or 2 cols], apart by x_stride
 *   y           out  (nullable) `type` [rows][cols]: a
 *   q, scale    out  (nullable) int8 [rows][cols], float32 [rows][ceil(cols / group) or 1]: what xnor_q8_rows makes of a in float32
 *   kept, kept_scale
 *               out  (nullable) int8 [rows][cols or 2 cols], float32 [rows][groups of kept_group of those columns, or 1]: what xnor_q8_rows makes of x
 *   group, kept_group   0, 32, 64 or 128 columns
 * One of y, q and kept is required.  cols <= 2^23; in the backward pass rows * ceil(cols / 2048) < 2^24 - 1, XNOR_ERR_SHAPE otherwise.
 *
 * Backward pass, from what was kept: with x^ = kept * kept_scale
 *     g_x = g_y f'(x^),  f'(0) = 0 for XNOR_RELU;     gated: g_x[:, :cols] = g_y x^[:, cols:] f'(x^[:, :cols]),  g_x[:, cols:] = g_y f(x^[:, :cols])
 *   g_y         in   `type` [rows][cols], apart by g_stride
 *   g_x         out  `type` [rows][cols or 2 cols]; may be g_y itself where that is dense and gated is 0
 */
typedef enum {
    XNOR_RELU = 0,
    XNOR_GELU = 1,
    XNOR_SILU = 2
} xnor_function;

XNOR_API int xnor_activation_q8(const void *x, int64_t x_stride, void *y, int8_t *q, float *scale, int8_t *kept, float *kept_scale, int rows, int cols,
                                int group, int kept_group, int function, int gated, int type, void *hip_stream);
XNOR_API int xnor_activation_backward(const int8_t *kept, const float *kept_scale, const void *g_y, int64_t g_stride, void *g_x, int rows, int cols,
                                      int kept_group, int function, int gated, int type, void *hip_stream);

/*
 * Gradients of a product's weights and bias from the 8-bit rows that it read:
 *     g_w[o][k] = sum_r g_y[r][o] q[r][k] scale[r][k / group],     g_bias[o] = sum_r g_y[r][o]
 *   q, scale    in   int8 [rows][in], float32 [rows][ceil(in / group)] (one per row where group is 0)
 *   g_y         in   `type` [rows][out], apart by g_stride
 *   g_w         out  `w_type` [out][in]; accumulate 1: added to what it holds, in float32, and rounded once more
 *   g_bias      out  (nullable) float32 [out]; accumulate as above
 *   workspace        xnor_q8_weight_gradient_workspace_bytes(rows, in, out, group, type, w_type) bytes
 * Few products run in float32 throughout; the others on the 16-bit matrix instructions with float32 sums.  There a row's value q * scale and a float32
 * gradient enter as two 11-bit floats (22 bits), 16-bit gradients as they are; with group 0 q enters as it is and g_y * scale as two such floats.  For XNOR_BF16 results one takes the
 * place of two, but for float32 gradients (and their products with the scales of rows).  Both sides are first
 * multiplied by powers of two that bring each column's largest (of a group: what its largest scale makes of a code of 128) to between 2^14 and 2^15; what is then below 2^-14 keeps its
 * value to 2^-25, at most 2^-39 of that largest.  A scale may be any finite number: only its products with gradients have to be within float32's range.  A row of g_w whose gradients hold an
 * infinity or a NaN is not finite; neither are a group's columns with a scale that is not.  The order of the sums follows from the sizes alone.
 * With rows = 0 the results are zeros (accumulate: left as they are).  in * out <= 2^35, XNOR_ERR_SHAPE otherwise.
 */
XNOR_API size_t xnor_q8_weight_gradient_workspace_bytes(int rows, int in, int out, int group, int type, int w_type);
XNOR_API int xnor_q8_weight_gradient(const int8_t *q, const float *scale, const void *g_y, int64_t g_stride, void *g_w, float *g_bias, int accumulate,
                                     void *workspace, int rows, int in, int out, int group, int type, int w_type, void *hip_stream);

/*
 * Draws a token for each row of logits, with random numbers that are given.  The tokens of a row are ordered by their logits, the largest first, of equal ones the
 * lowest index first, and have weights exp((l - largest) / temperature).  Drawn from are
 *     the first top_k;  of these the shortest run from the first on whose weights reach top_p of theirs;  of these the ones whose weight is min_p or more
 * and drawn is the first of them whose weights, added up in that order, exceed uniform times their sum.
 *   logits       in   `type` [rows][vocab], apart by stride; -inf marks what is masked, and is never drawn
 *   temperature  in   (nullable: 1) float32 [rows], >= 0; 0 draws the first token
 *   top_k        in   (nullable) int32 [rows]; 0 and below: all
 *   top_p        in   (nullable) float32 [rows]; 1 and above: all; always one token at least
 *   min_p        in   (nullable) float32 [rows]; 0 and below: all; above 1 as 1
 *   uniform      in   float32 [rows], within [0, 1): below counts as 0, above as the largest number below 1
 *   token        out  int32 [rows]
 *   logprob      out  (nullable) float32 [rows]: log of the token's weight over the sum that it was drawn from
 *   kept         out  (nullable) int32 [rows]: how many tokens it was drawn from
 *   workspace         xnor_sample_workspace_bytes(rows, vocab) bytes, may be NULL where that is 0 and with top_k
 * Weights are computed to 1.5e-13 of themselves, held as multiples of 2^-44 of the largest (of 2^(b - 62) for a vocabulary of 2^b > 2^18) and added as integers, so that
 * a draw depends on no order of additions: it is the formula's but for a uniform, a top_p or a min_p that close to a border.  Tokens whose weight rounds to 0 are
 * counted, never drawn.
 * A row without any logit above -inf has token -1, logprob -inf and kept 0; one that holds a NaN or +inf, or whose temperature (NaN or below 0),
 * top_p, min_p or uniform is none (NaN), token -1, logprob NaN and kept 0.
 */
XNOR_API size_t xnor_sample_workspace_bytes(int rows, int vocab);
XNOR_API int xnor_sample(const void *logits, int64_t stride, const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p,
                         const float *uniform, int32_t *token, float *logprob, int32_t *kept, void *workspace, int rows, int vocab, int type, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* XNOR_LOWBIT_H */
