// Parameters of the kernels that normalise and rotate the heads of queries and keys (head_rows.cu, head_rows_grad.cu), into
// rows or into a paged cache, shared with their entry points (cache_ops.cu).
#pragma once
#include <cuda_runtime.h>

#include "rope_axes.cuh"

namespace regenvc {

// Where an operand's vectors lie, strides in bytes, for the kernels on units: an address is then two multiply-adds.
struct HeadRowsView {
    const char *from, *dy;
    char* to;
    int from_token, from_head, dy_token, dy_head, to_token, to_head;
};

struct HeadRowsParams {
    const void* in[3];                 // q, k, v: [tokens][heads][head_dim]
    void* out[3];                      // q, k: rows; paged: k, v: the caches
    long long in_token[3], in_head[3], out_token[3], out_head[3];   // strides in elements (paged: between slots of a page)
    int heads[3];                      // heads of q, k, v (0: absent)
    int n_tokens, head_dim, n_pairs;   // 2 * n_pairs elements of a head are rotated, the rest is not
    int n_axes, axis_end[kRopeMaxAxes];
    const void* positions;             // [n_axes][n_tokens] int32 or fp32
    long long pos_stride;
    int pos_float, halves, norm;       // norm: 0 none, 1 root mean square
    float eps;
    const float* weight[2];            // gains of q, of k [head_dim], or nullptr
    // paged: where the new tokens of a sequence go
    int paged;
    const int* row_starts;             // [n_sequences + 1]
    const int* lengths;                // [n_sequences] cached tokens, the new ones among them
    const int* table;                  // [n_sequences][pages of a sequence]
    long long table_stride, page_stride[2];
    int n_sequences, page_size, n_pages;
    int most_tokens;                   // that a sequence's row of the table can hold
    int* status;
    // gradients: in[] = x, grad[] = dy, out[] = dx
    const void* grad[2];
    long long grad_token[2], grad_head[2];
    float* dweight[2];
    float* partial;                    // [blocks][2][head_dim]
    int tokens_per_cta;                // set by the launchers, as is:
    HeadRowsView view[3];
    double turns[kRopeMaxPairs];       // frequency / (2 pi) of a pair: whole turns per unit of position
};

cudaError_t launch_head_rows(HeadRowsParams p, int type, bool vec, int sm_count, cudaStream_t stream);
// The gradients' grid has at most this many blocks, which sizes their workspace.
constexpr int kHeadGradMaxBlocks = 1184;
inline size_t head_grad_workspace_bytes(int head_dim) { return (size_t)kHeadGradMaxBlocks * 2 * head_dim * sizeof(float); }
cudaError_t launch_head_rows_grad(HeadRowsParams p, int type, bool vec, int sm_count, int* launches, cudaStream_t stream);

}  // namespace regenvc
