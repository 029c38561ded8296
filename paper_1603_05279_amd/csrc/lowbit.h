// Launchers of the calls of xnor_lowbit.h (arguments checked by lowbit_api.hip; rows = 0 reaches none but rmsnorm's backward pass).
#pragma once
#include <hip/hip_runtime.h>
#include "xnor_lowbit.h"

namespace xnor {

// What the ..._workspace_bytes of xnor_lowbit.h say never falls as rows grows, so it serves fewer rows too; a call may need less (..._needs: whether any)
size_t rmsnorm_grad_workspace_bytes(int rows, int cols);        // shares of g_weight, [parts][cols] floats
xnor_status launch_rmsnorm_q8(const void *x, long long x_stride, const void *residual, long long residual_stride, const float *weight,
                              void *sum_out, int8_t *q, float *scale, void *values, float *rstd, int rows, int cols, int group, int type,
                              float eps, hipStream_t stream);
xnor_status launch_rmsnorm_backward(const void *h, long long h_stride, const float *rstd, const float *weight, const void *g, long long g_stride,
                                    const void *g_sum, long long g_sum_stride, void *g_h, float *g_weight, void *workspace, int rows, int cols,
                                    int type, hipStream_t stream);
constexpr int W4_8_BITS = 3;
size_t w4_wimg_bytes(int out, int in, int group);
xnor_status launch_w4_quantize(const void *w, long long stride, uint8_t *codes, float *scale, uint8_t *zero, int out, int in, int group, int type,
                               hipStream_t stream);
xnor_status launch_w4_pack(const uint8_t *codes, const float *scale, const uint8_t *zero, void *wimg, int out, int in, int group, hipStream_t stream);
size_t w4_linear_workspace_bytes(int rows, int in, int out, int group);
bool w4_linear_needs(int rows, int in, int out, int group, int form);
xnor_status launch_w4_linear(const void *x, long long x_stride, const void *wimg, void *y, void *workspace, int rows, int in, int out, int group, int type,
                             hipStream_t stream);
xnor_status launch_w4_linear_q8(const int8_t *q, const float *x_scale, const void *wimg, void *y, void *workspace, int rows, int in, int out, int group,
                                int x_group, int type, hipStream_t stream);
// products (form: the rows' xnor_dtype, or W4_8_BITS): w4_rows_kernel, or the kernels of w4_tiles.hip on staged rows
enum W4Kernel { W4_ROWS, W4_WAVES, W4_TILES };
struct W4Choice {
    W4Kernel kernel;
    int tiles;              // of 16 outputs per workgroup of w4_rows_kernel
    double time;            // us, expected
};
W4Choice w4_choice(int rows, int in, int out, int group, int form);
xnor_status launch_w4_staged(W4Kernel kernel, const void *x, long long x_stride, const float *x_scale, const void *wimg, void *y, void *workspace, int rows,
                             int in, int out, int group, int x_group, int form, int type, hipStream_t stream);
size_t logprobs_workspace_bytes(int rows, int vocab, int top);
bool logprobs_needs(int rows, int vocab, int top);
xnor_status launch_logprobs(const void *logits, long long stride, const void *tokens, int token_bytes, float *logprob, float *lse, float *shift, float *entropy,
                            int32_t *top_index, float *top_logprob, void *workspace, int rows, int vocab, int given, int top, int type,
                            hipStream_t stream);
xnor_status launch_logprobs_backward(const void *logits, long long stride, const void *tokens, int token_bytes, const float *shift,
                                     const float *entropy, const float *g_logprob, const float *g_entropy, void *g_logits, int rows, int vocab,
                                     int given, int type, hipStream_t stream);

}  // namespace xnor
