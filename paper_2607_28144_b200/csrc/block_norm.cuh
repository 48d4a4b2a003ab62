// Parameters of the block-norm kernels (block_norm.cu), shared with the entry points (block_ops.cu).
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>

namespace regenvc {

constexpr int kNormMaxChannels = 8192;   // sixteen columns per thread, at most 512 threads
constexpr int kNormMaxCtas = 760;        // the backward pass's grid never exceeds this: it bounds the workspace
constexpr int kNormLayer = 1, kNormRms = 2;

struct BlockNormParams {
    int n_tokens, channels, tokens_per_mod;
    int norm, post_norm;          // 0 none, kNormLayer, kNormRms
    float eps, post_eps, residual_scale;
    long long mod_stride;         // elements between the modulation rows of scale, shift and gate
    long long x_stride, y_stride, x_out_stride, h_stride, dx_out_stride, dx_stride, dy_stride;
    const void* x;                // forward: residual stream; backward: the saved x'
    const void* y;
    const float *gate, *post_weight, *weight, *bias, *scale, *shift;
    // forward results
    void *x_out, *h;
    // backward: incoming and outgoing gradients
    const void *dh, *dx_out;
    void *dx, *dy;
    float *dgate, *dpost_weight, *dweight, *dbias, *dscale, *dshift;
    float* partials;              // backward workspace
    int rows_per_cta;             // set by the launcher
};

inline size_t block_norm_workspace_bytes(long long n_tokens, long long channels) {
    const long long ctas = n_tokens < kNormMaxCtas ? n_tokens : kNormMaxCtas;
    return (size_t)ctas * 9 * (size_t)channels * sizeof(float);
}

// x_type / io_type as in regenvc_type; `vec`: channels, strides and addresses allow 16-byte accesses.
cudaError_t launch_block_norm_forward(BlockNormParams p, int x_type, int io_type, bool vec, int sm_count,
                                      cudaStream_t stream);
// *launches: how many kernels were enqueued.
cudaError_t launch_block_norm_backward(BlockNormParams p, int x_type, int io_type, bool vec, int sm_count, int* launches,
                                       cudaStream_t stream);

}  // namespace regenvc
