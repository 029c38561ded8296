// C ABI of xnor_lowbit.h: argument validation and dispatch.
#include "xnor_internal.h"
#include "lowbit.h"
#include "real8.h"
#include <math.h>

using namespace xnor;

namespace {

constexpr int MAX_ROWS = 65535 * 64, MAX_WIDTH = 1 << 24, MAX_VOCAB = 1 << 30, MAX_COLS = 32768, MAX_GIVEN = 1024, MAX_TOP = 32;
constexpr int MAX_W8_IN = 131071;          // 128 * 128 products within 31 bits
constexpr long long MAX_WEIGHTS = 1LL << 35;    // of a gradient: tiles within one launch

template <class... P> bool aligned16(P... p) { return ((reinterpret_cast<uintptr_t>(p) | ... | 0) & 15u) == 0; }
bool w4_group(int g) { return g == 32 || g == 64 || g == 128; }

xnor_status check_w4(int out, int in, int group)
{
    if (out <= 0 || in <= 0 || out > MAX_WIDTH || in > MAX_WIDTH) return XNOR_ERR_SHAPE;
    return w4_group(group) ? XNOR_OK : XNOR_ERR_UNSUPPORTED;
}
xnor_status check_logprobs(int token_bytes, int rows, int vocab, int given, int top, int type)
{
    if (rows < 0 || rows > MAX_ROWS || vocab <= 0 || vocab > MAX_VOCAB || given < 0 || top < 0) return XNOR_ERR_SHAPE;
    if (given > MAX_GIVEN || top > MAX_TOP || !known_type(type) || (given && token_bytes != 4 && token_bytes != 8)) return XNOR_ERR_UNSUPPORTED;
    return XNOR_OK;
}

bool row_group(int g) { return g == 0 || w4_group(g); }
xnor_status check_w8(int rows, int in, int out)
{
    if (rows < 0 || rows > MAX_ROWS || in <= 0 || out <= 0 || in > MAX_WIDTH || out > MAX_WIDTH) return XNOR_ERR_SHAPE;
    return in > MAX_W8_IN ? XNOR_ERR_UNSUPPORTED : XNOR_OK;
}
xnor_status check_activation(int rows, int cols, int kept_group, int function, int gated, int type)
{
    if (rows < 0 || rows > MAX_ROWS || cols <= 0 || cols > MAX_WIDTH / 2) return XNOR_ERR_SHAPE;
    if (!row_group(kept_group) || function < XNOR_RELU || function > XNOR_SILU || (gated & ~1) || !known_type(type)) return XNOR_ERR_UNSUPPORTED;
    return XNOR_OK;
}
xnor_status check_gradient(int rows, int in, int out, int group, int type, int w_type)
{
    if (rows < 0 || rows > MAX_ROWS || in <= 0 || out <= 0 || in > MAX_WIDTH || out > MAX_WIDTH || (long long)in * out > MAX_WEIGHTS) return XNOR_ERR_SHAPE;
    return row_group(group) && known_type(type) && known_type(w_type) ? XNOR_OK : XNOR_ERR_UNSUPPORTED;
}

}  // namespace

extern "C" {

int xnor_rmsnorm_q8(const void *x, int64_t x_stride, const void *residual, int64_t residual_stride, const float *weight, void *sum_out, int8_t *q,
                    float *scale, void *values, float *rstd, int rows, int cols, int group, int type, float eps, void *hip_stream)
{
    if (rows < 0 || rows > MAX_ROWS || cols <= 0 || !(eps > 0.0f) || isinf(eps)) return XNOR_ERR_SHAPE;
    if (cols > MAX_COLS || !known_type(type) || (group != 0 && !w4_group(group))) return XNOR_ERR_UNSUPPORTED;
    if (rows == 0) return XNOR_OK;
    if (!x || (!q && !values) || (q && !scale)) return XNOR_ERR_NULL;
    if (x_stride < cols || (residual && residual_stride < cols)) return XNOR_ERR_SHAPE;
    if (!aligned16(x, residual, weight, sum_out, q, scale, values, rstd)) return XNOR_ERR_ALIGN;
    return launch_rmsnorm_q8(x, x_stride, residual, residual_stride, weight, sum_out, q, scale, values, rstd, rows, cols, group, type, eps,
                             (hipStream_t)hip_stream);
}

size_t xnor_rmsnorm_backward_workspace_bytes(int rows, int cols)
{
    if (rows <= 0 || rows > MAX_ROWS || cols <= 0 || cols > MAX_COLS) return 0;
    return rmsnorm_grad_workspace_bytes(rows, cols);
}

int xnor_rmsnorm_backward(const void *h, int64_t h_stride, const float *rstd, const float *weight, const void *g_values, int64_t g_stride,
                          const void *g_sum, int64_t g_sum_stride, void *g_h, float *g_weight, void *workspace, int rows, int cols, int type,
                          void *hip_stream)
{
    if (rows < 0 || rows > MAX_ROWS || cols <= 0) return XNOR_ERR_SHAPE;
    if (cols > MAX_COLS || !known_type(type)) return XNOR_ERR_UNSUPPORTED;
    if (rows == 0 && !g_weight) return XNOR_OK;
    if (rows && (!h || !rstd || !g_values || !g_h || (g_weight && !workspace))) return XNOR_ERR_NULL;
    if (rows && (h_stride < cols || g_stride < cols || (g_sum && g_sum_stride < cols))) return XNOR_ERR_SHAPE;
    if (!aligned16(g_weight) || (rows && !aligned16(h, rstd, weight, g_values, g_sum, g_h, workspace))) return XNOR_ERR_ALIGN;
    return launch_rmsnorm_backward(h, h_stride, rstd, weight, g_values, g_stride, g_sum, g_sum_stride, g_h, g_weight, workspace, rows, cols, type,
                                   (hipStream_t)hip_stream);
}

int xnor_w4_quantize(const void *w, int64_t w_stride, uint8_t *codes, float *scale, uint8_t *zero, int out, int in, int group, int type,
                     void *hip_stream)
{
    if (xnor_status s = check_w4(out, in, group)) return s;
    if (!known_type(type)) return XNOR_ERR_UNSUPPORTED;
    if (!w || !codes || !scale) return XNOR_ERR_NULL;
    if (w_stride < in) return XNOR_ERR_SHAPE;
    if (!aligned16(w, codes, scale, zero)) return XNOR_ERR_ALIGN;
    return launch_w4_quantize(w, w_stride, codes, scale, zero, out, in, group, type, (hipStream_t)hip_stream);
}

size_t xnor_w4_wimg_bytes(int out, int in, int group) { return check_w4(out, in, group) ? 0 : w4_wimg_bytes(out, in, group); }

int xnor_w4_pack(const uint8_t *codes, const float *scale, const uint8_t *zero, void *wimg, int out, int in, int group, void *hip_stream)
{
    if (xnor_status s = check_w4(out, in, group)) return s;
    if (!codes || !scale || !wimg) return XNOR_ERR_NULL;
    if (!aligned16(codes, scale, zero, wimg)) return XNOR_ERR_ALIGN;
    return launch_w4_pack(codes, scale, zero, wimg, out, in, group, (hipStream_t)hip_stream);
}

size_t xnor_w4_linear_workspace_bytes(int rows, int in, int out, int group)
{
    return rows <= 0 || rows > MAX_ROWS || check_w4(out, in, group) ? 0 : w4_linear_workspace_bytes(rows, in, out, group);
}

int xnor_w4_linear(const void *x, int64_t x_stride, const void *wimg, void *y, void *workspace, int rows, int in, int out, int group, int type,
                   void *hip_stream)
{
    if (rows < 0 || rows > MAX_ROWS) return XNOR_ERR_SHAPE;
    if (xnor_status s = check_w4(out, in, group)) return s;
    if (!known_type(type)) return XNOR_ERR_UNSUPPORTED;
    if (rows == 0) return XNOR_OK;
    if (!x || !wimg || !y || (!workspace && w4_linear_needs(rows, in, out, group, type))) return XNOR_ERR_NULL;
    if (x_stride < in) return XNOR_ERR_SHAPE;
    if (!aligned16(x, wimg, y, workspace)) return XNOR_ERR_ALIGN;
    return launch_w4_linear(x, x_stride, wimg, y, workspace, rows, in, out, group, type, (hipStream_t)hip_stream);
}

int xnor_w4_linear_q8(const int8_t *q, const float *x_scale, const void *wimg, void *y, void *workspace, int rows, int in, int out, int group,
                      int x_group, int type, void *hip_stream)
{
    if (rows < 0 || rows > MAX_ROWS) return XNOR_ERR_SHAPE;
    if (xnor_status s = check_w4(out, in, group)) return s;
    if (!known_type(type) || (x_group != 0 && (!w4_group(x_group) || x_group < group))) return XNOR_ERR_UNSUPPORTED;
    if (rows == 0) return XNOR_OK;
    if (!q || !x_scale || !wimg || !y || (!workspace && w4_linear_needs(rows, in, out, group, W4_8_BITS))) return XNOR_ERR_NULL;
    if (!aligned16(q, x_scale, wimg, y, workspace)) return XNOR_ERR_ALIGN;
    return launch_w4_linear_q8(q, x_scale, wimg, y, workspace, rows, in, out, group, x_group, type, (hipStream_t)hip_stream);
}

size_t xnor_logprobs_workspace_bytes(int rows, int vocab, int top)
{
    return rows <= 0 || check_logprobs(4, rows, vocab, 0, top, XNOR_F32) ? 0 : logprobs_workspace_bytes(rows, vocab, top);
}

int xnor_logprobs(const void *logits, int64_t stride, const void *tokens, int token_bytes, float *logprob, float *lse, float *shift, float *entropy,
                  int32_t *top_index, float *top_logprob, void *workspace, int rows, int vocab, int given, int top, int type, void *hip_stream)
{
    if (xnor_status s = check_logprobs(token_bytes, rows, vocab, given, top, type)) return s;
    if (rows == 0) return XNOR_OK;
    if (!logits || (given && (!tokens || !logprob)) || (top && (!top_index || !top_logprob)) ||
        (!workspace && logprobs_needs(rows, vocab, top)))
        return XNOR_ERR_NULL;
    if (stride < vocab) return XNOR_ERR_SHAPE;
    if (!aligned16(logits, tokens, logprob, lse, shift, entropy, top_index, top_logprob, workspace)) return XNOR_ERR_ALIGN;
    return launch_logprobs(logits, stride, tokens, token_bytes, logprob, lse, shift, entropy, top_index, top_logprob, workspace, rows, vocab, given, top, type,
                           (hipStream_t)hip_stream);
}

int xnor_logprobs_backward(const void *logits, int64_t stride, const void *tokens, int token_bytes, const float *shift, const float *entropy,
                           const float *g_logprob, const float *g_entropy, void *g_logits, int rows, int vocab, int given, int type, void *hip_stream)
{
    if (xnor_status s = check_logprobs(token_bytes, rows, vocab, given, 0, type)) return s;
    if (rows == 0) return XNOR_OK;
    if (!logits || !shift || !g_logits || (!g_logprob && !g_entropy) || (g_entropy && !entropy) || (g_logprob && given && !tokens)) return XNOR_ERR_NULL;
    if (stride < vocab) return XNOR_ERR_SHAPE;
    if (!aligned16(logits, tokens, shift, entropy, g_logprob, g_entropy, g_logits)) return XNOR_ERR_ALIGN;
    return launch_logprobs_backward(logits, stride, tokens, token_bytes, shift, entropy, g_logprob, g_entropy, g_logits, rows, vocab, given, type,
                                    (hipStream_t)hip_stream);
}

int xnor_q8_rows(const void *x, int64_t x_stride, int8_t *q, float *scale, int rows, int cols, int group, int type, void *hip_stream)
{
    if (rows < 0 || rows > MAX_ROWS || cols <= 0 || cols > MAX_WIDTH) return XNOR_ERR_SHAPE;
    if (!row_group(group) || !known_type(type)) return XNOR_ERR_UNSUPPORTED;
    if (rows == 0) return XNOR_OK;
    if (!x || !q || !scale) return XNOR_ERR_NULL;
    if (x_stride < cols) return XNOR_ERR_SHAPE;
    if (!aligned16(x, q, scale)) return XNOR_ERR_ALIGN;
    return launch_q8_rows(x, x_stride, q, scale, rows, cols, group, type, (hipStream_t)hip_stream);
}

size_t xnor_w8_linear_workspace_bytes(int rows, int in, int out) { return rows <= 0 || check_w8(rows, in, out) ? 0 : w8_linear_workspace_bytes(rows, in, out); }

int xnor_w8_linear(const int8_t *q, const float *x_scale, const int8_t *w, const float *w_scale, const float *bias, void *y, void *workspace, int rows,
                   int in, int out, int type, void *hip_stream)
{
    if (xnor_status s = check_w8(rows, in, out)) return s;
    if (!known_type(type)) return XNOR_ERR_UNSUPPORTED;
    if (rows == 0) return XNOR_OK;
    if (!q || !x_scale || !w || !w_scale || !y || (!workspace && w8_linear_needs(rows, in, out))) return XNOR_ERR_NULL;
    if (!aligned16(q, x_scale, w, w_scale, bias, y, workspace)) return XNOR_ERR_ALIGN;
    return launch_w8_linear(q, x_scale, w, w_scale, bias, y, workspace, rows, in, out, type, (hipStream_t)hip_stream);
}

int xnor_activation_q8(const void *x, int64_t x_stride, void *y, int8_t *q, float *scale, int8_t *kept, float *kept_scale, int rows, int cols, int group,
                       int kept_group, int function, int gated, int type, void *hip_stream)
{
    if (xnor_status s = check_activation(rows, cols, kept_group, function, gated, type)) return s;
    if (!row_group(group)) return XNOR_ERR_UNSUPPORTED;
    if (rows == 0) return XNOR_OK;
    if (!x || (!y && !q && !kept) || (q && !scale) || (kept && !kept_scale)) return XNOR_ERR_NULL;
    if (x_stride < (int64_t)cols << gated) return XNOR_ERR_SHAPE;
    if (!aligned16(x, y, q, scale, kept, kept_scale)) return XNOR_ERR_ALIGN;
    return launch_activation_q8(x, x_stride, y, q, scale, kept, kept_scale, rows, cols, group, kept_group, function, gated, type, (hipStream_t)hip_stream);
}

int xnor_activation_backward(const int8_t *kept, const float *kept_scale, const void *g_y, int64_t g_stride, void *g_x, int rows, int cols, int kept_group,
                             int function, int gated, int type, void *hip_stream)
{
    if (xnor_status s = check_activation(rows, cols, kept_group, function, gated, type)) return s;
    if (rows == 0) return XNOR_OK;
    if (!kept || !kept_scale || !g_y || !g_x) return XNOR_ERR_NULL;
    if (g_stride < cols) return XNOR_ERR_SHAPE;
    if (!aligned16(kept, kept_scale, g_y, g_x)) return XNOR_ERR_ALIGN;
    return launch_activation_backward(kept, kept_scale, g_y, g_stride, g_x, rows, cols, kept_group, function, gated, type, (hipStream_t)hip_stream);
}

size_t xnor_q8_weight_gradient_workspace_bytes(int rows, int in, int out, int group, int type, int w_type)
{
    return rows <= 0 || check_gradient(rows, in, out, group, type, w_type) ? 0 : weight_gradient_workspace_bytes(rows, in, out, group, type, w_type);
}

int xnor_q8_weight_gradient(const int8_t *q, const float *scale, const void *g_y, int64_t g_stride, void *g_w, float *g_bias, int accumulate, void *workspace,
                            int rows, int in, int out, int group, int type, int w_type, void *hip_stream)
{
    if (xnor_status s = check_gradient(rows, in, out, group, type, w_type)) return s;
    if (accumulate & ~1) return XNOR_ERR_UNSUPPORTED;
    if (rows == 0 && accumulate) return XNOR_OK;
    if (!g_w || (rows && (!q || !scale || !g_y || !workspace))) return XNOR_ERR_NULL;
    if (rows && g_stride < out) return XNOR_ERR_SHAPE;
    if (!aligned16(g_w, g_bias) || (rows && !aligned16(q, scale, g_y, workspace))) return XNOR_ERR_ALIGN;
    return launch_weight_gradient(q, scale, g_y, g_stride, g_w, g_bias, accumulate, workspace, rows, in, out, group, type, w_type, (hipStream_t)hip_stream);
}

size_t xnor_sample_workspace_bytes(int rows, int vocab)
{
    return rows <= 0 || rows > MAX_ROWS || vocab <= 0 || vocab > MAX_VOCAB ? 0 : sample_workspace_bytes(rows, vocab);
}

int xnor_sample(const void *logits, int64_t stride, const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p, const float *uniform,
                int32_t *token, float *logprob, int32_t *kept, void *workspace, int rows, int vocab, int type, void *hip_stream)
{
    if (rows < 0 || rows > MAX_ROWS || vocab <= 0 || vocab > MAX_VOCAB) return XNOR_ERR_SHAPE;
    if (!known_type(type)) return XNOR_ERR_UNSUPPORTED;
    if (rows == 0) return XNOR_OK;
    if (!logits || !uniform || !token || (!workspace && sample_needs(rows, vocab, top_k != nullptr))) return XNOR_ERR_NULL;
    if (stride < vocab) return XNOR_ERR_SHAPE;
    if (!aligned16(logits, temperature, top_k, top_p, min_p, uniform, token, logprob, kept, workspace)) return XNOR_ERR_ALIGN;
    return launch_sample(logits, stride, temperature, top_k, top_p, min_p, uniform, token, logprob, kept, workspace, rows, vocab, type,
                         (hipStream_t)hip_stream);
}

}  // extern "C"
