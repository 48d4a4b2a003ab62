// Parameters of the multi-axis rotation kernel (rope_axes.cu), shared with its entry point (block_ops.cu).
#pragma once
#include <cuda_runtime.h>

namespace regenvc {

constexpr int kRopeMaxPairs = 128;   // head_dim up to 256
constexpr int kRopeMaxAxes = 4;

struct RopeAxesParams {
    const void* in[2];                 // q, k
    void* out[2];
    long long in_token[2], in_head[2], out_token[2], out_head[2];   // strides in elements
    int heads[2];                      // heads of q, of k (0: no k)
    int n_tokens, head_dim, n_pairs;   // 2 * n_pairs elements of a head are rotated, the rest is copied
    int n_axes, axis_end[kRopeMaxAxes];   // pairs below axis_end[a] (and not of an earlier axis) turn with axis a
    const void* positions;             // [n_axes][n_tokens] int32 or fp32
    long long pos_stride;
    int pos_float, inverse, halves;
    int tokens_per_cta;                // set by the launcher
    double turns[kRopeMaxPairs];       // frequency / (2 pi) of a pair: whole turns per unit of position
};

cudaError_t launch_rope_axes(RopeAxesParams p, int type, bool vec, int sm_count, cudaStream_t stream);

}  // namespace regenvc
