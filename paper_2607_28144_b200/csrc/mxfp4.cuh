// Packed form of a matrix in microscaled 4-bit floating point, and the parameters of the kernels on it (mxfp4.cu,
// mxfp4_project.cu), shared with the entry points (block_ops.cu).
//
// cols are rounded up to cols_pad, a multiple of 128 (padding codes and scales are 0, which stand for 0.0).
//   codes  : [rows][cols_pad / 2] bytes; byte b of a row holds element 2b in its low and 2b + 1 in its high half (e2m1:
//            sign, two exponent bits, one mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6)
//   scales : one byte (e8m0: 2^(byte - 127), 255 is NaN) per row and 32 columns, at the next multiple of 512 bytes, in
//            tiles of 128 rows x 4 blocks = 512 bytes, tiles of a row block one after the other; inside a tile the byte of
//            (row r, block b) is at (r % 32) * 16 + (r % 128) / 32 * 4 + b % 4 -- the order in which one tensor-memory
//            copy of 32 rows x 16 bytes puts them where the block-scaled tensor instruction reads them.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace regenvc {

struct MxLayout {
    long long rows, cols, cols_pad, scale_at, bytes;
    __host__ __device__ MxLayout(long long r, long long c)
        : rows(r), cols(c), cols_pad((c + 127) / 128 * 128), scale_at((r * (cols_pad / 2) + 511) / 512 * 512),
          bytes(scale_at + (r + 127) / 128 * (cols_pad / 128) * 512) {}
    __host__ __device__ long long scale_tiles() const { return (rows + 127) / 128 * (cols_pad / 128); }
};

struct MxConvertParams {
    const void* src;      // quantise: values; dequantise: packed
    void* dst;
    long long row_stride; // of the values, in elements
    int rows, cols;
    int vec;              // the values' address and stride allow accesses of 32 bytes (2), 16 bytes (1) or neither (0)
};
cudaError_t launch_mxfp4_quantize(const MxConvertParams& p, int type, int sm_count, cudaStream_t stream);
cudaError_t launch_mxfp4_dequantize(const MxConvertParams& p, int type, int sm_count, cudaStream_t stream);

struct MxProjectParams {
    const float* bias;    // [features] or nullptr
    int n_tokens, features, k_blocks;   // k_blocks: cols_pad / 128
    int y_f16;            // y is fp16 (else bf16)
    int* status;
};
// The tensor-core product.  A plan says which build runs and what its tensor maps look like.
struct MxProjectPlan {
    int pair;             // 1: on pairs of CTAs
    int tile_features;    // output features per work item
    int w_box_rows;       // rows of one weight load
};
MxProjectPlan plan_mxfp4_project(int n_tokens, int features, int in_features, int sm_count);
cudaError_t configure_mxfp4_project();
// early: the launch before it on `stream` is launch_mxfp4_quantize() of this x, whose end the set-up may overlap (the kernel
// waits for it before it reads x).
cudaError_t launch_mxfp4_project(const MxProjectPlan& plan, const CUtensorMap& x, const CUtensorMap& xs, const CUtensorMap& w,
                                 const CUtensorMap& ws, const CUtensorMap& y, const MxProjectParams& p, bool early,
                                 int sm_count, cudaStream_t stream);

// The product for a few tokens (mxfp4_rows.cu), from x of any type or packed.
constexpr int kMxFewRows = 4;
struct MxRowsParams {
    const void* x;
    long long x_stride;       // elements between rows (not packed)
    const uint8_t* w;         // packed
    const float* bias;        // [features] or nullptr
    void* y;                  // [n_tokens][features] 16-bit
    long long cols_pad, x_scale_at, w_scale_at;
    int n_tokens, features, cols;
    int vec;                  // x's address and stride allow 16-byte accesses
    int y_f16;
};
bool mxfp4_rows_fits(int n_tokens, int features, long long cols_pad);
cudaError_t launch_mxfp4_rows(const MxRowsParams& p, int type, bool packed, int sm_count, cudaStream_t stream);

}  // namespace regenvc
