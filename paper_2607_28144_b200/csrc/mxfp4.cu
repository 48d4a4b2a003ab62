// To and from microscaled 4-bit floating point (blocks of 32 along a row share a power-of-two scale; layout in
// mxfp4.cuh).  Bound: HBM.  Sixteen threads take 128 columns of a row, eight each: four threads hold one block, so the
// largest magnitude is two exchanges away, reads are 16 bytes per thread and writes 64 contiguous bytes per row.
#include "mx_convert.cuh"
#include "mxfp4.cuh"
#include "row_io.cuh"

namespace regenvc {
namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;

template <typename T>
__device__ __forceinline__ void load_eight(const T* row, int c, int cols, bool vec, float* v) {
    if (vec && c + 8 <= cols) {
        widen8(load_raw8(row + c), v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c + i < cols ? to_f32(row[c + i]) : 0.0f;
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) mxfp4_quantize_kernel(const MxConvertParams p) {
    const MxLayout lay(p.rows, p.cols);
    const int groups = (int)(lay.cols_pad / 128);
    const long long units = (long long)(p.rows + 127) / 128 * 128 * groups;   // rows past the last: scales only
    const int lane = threadIdx.x & 15;
    const long long step = (long long)gridDim.x * (kThreads / 16);
    uint8_t* codes = reinterpret_cast<uint8_t*>(p.dst);
    uint8_t* scales = codes + lay.scale_at;
    // whole warps take part in the exchanges: the trip count is that of the warp's first half
    const long long first = (long long)blockIdx.x * (kThreads / 16) + (threadIdx.x >> 4);
    for (long long base = first; base - ((threadIdx.x >> 4) & 1) < units; base += step * kUnroll) {
        float v[kUnroll][8];
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) {
            const long long u = base + k * step;
            const long long row = u / groups;
            const int c = (int)(u - row * groups) * 128 + lane * 8;
            if (u < units && row < p.rows) {
                load_eight(reinterpret_cast<const T*>(p.src) + row * p.row_stride, c, p.cols, p.vec != 0, v[k]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[k][i] = 0.0f;
            }
        }
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) {
            const long long u = base + k * step;
            const long long row = u / groups;
            const int g = (int)(u - row * groups);
            uint32_t top = 0;   // magnitudes compare as their bit patterns, NaN above infinity
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[k][i]) & 0x7FFFFFFFu);
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const uint32_t byte = mx_scale_byte(top);
            const float inv = mx_inverse_scale(byte);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] = byte == 255u ? 0.0f : v[k][i] * inv;
            // the four scales of these 128 columns side by side
            uint32_t word = byte << (lane >> 2) * 8;
            word |= __shfl_xor_sync(0xffffffffu, word, 4);
            word |= __shfl_xor_sync(0xffffffffu, word, 8);
            if (u < units) {
                if (row < p.rows)
                    *reinterpret_cast<uint32_t*>(codes + row * (lay.cols_pad / 2) + g * 64 + lane * 4) = mx_codes8(v[k]);
                if (lane == 0)
                    *reinterpret_cast<uint32_t*>(scales + (row / 128 * groups + g) * 512 + row % 32 * 16 + row % 128 / 32 * 4) = word;
            }
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) mxfp4_dequantize_kernel(const MxConvertParams p) {
    const MxLayout lay(p.rows, p.cols);
    const int eights = (p.cols + 7) / 8;
    const long long units = (long long)p.rows * eights;
    const long long step = (long long)gridDim.x * kThreads;
    const uint8_t* codes = reinterpret_cast<const uint8_t*>(p.src);
    const uint8_t* scales = codes + lay.scale_at;
    for (long long base = (long long)blockIdx.x * kThreads + threadIdx.x; base < units; base += step * kUnroll) {
        uint32_t q[kUnroll];
        uint32_t s[kUnroll];
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) {
            const long long u = base + k * step;
            if (u >= units) continue;
            const long long row = u / eights;
            const int c = (int)(u - row * eights) * 8;
            q[k] = *reinterpret_cast<const uint32_t*>(codes + row * (lay.cols_pad / 2) + c / 2);
            s[k] = scales[(row / 128 * (lay.cols_pad / 128) + c / 128) * 512 + row % 32 * 16 + row % 128 / 32 * 4 + c / 32 % 4];
        }
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) {
            const long long u = base + k * step;
            if (u >= units) continue;
            const long long row = u / eights;
            const int c = (int)(u - row * eights) * 8;
            uint32_t h2[4];
            float v[8];
            mx_values8(q[k], h2);
            const float scale = mx_scale_value(s[k]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                widen2(h2[i], v[2 * i], v[2 * i + 1], (const __half*)nullptr);
                v[2 * i] *= scale;
                v[2 * i + 1] *= scale;
            }
            T* out = reinterpret_cast<T*>(p.dst) + row * p.row_stride + c;
            if (p.vec && c + 8 <= p.cols) {
                store8(out, v);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c + i < p.cols) from_f32(v[i], out[i]);
            }
        }
    }
}

unsigned grid_for(long long units, int per_block, int sm_count) {
    long long blocks = (units + (long long)per_block * kUnroll - 1) / ((long long)per_block * kUnroll);
    if (blocks < sm_count) blocks = (units + per_block - 1) / per_block < sm_count ? (units + per_block - 1) / per_block : sm_count;
    if (blocks > 8ll * sm_count) blocks = 8ll * sm_count;
    return (unsigned)blocks;
}

}  // namespace

cudaError_t launch_mxfp4_quantize(const MxConvertParams& p, int type, int sm_count, cudaStream_t stream) {
    const long long units = (long long)(p.rows + 127) / 128 * 128 * ((p.cols + 127) / 128);
    const unsigned grid = grid_for(units, kThreads / 16, sm_count);
    if (type == kTypeBf16) mxfp4_quantize_kernel<__nv_bfloat16><<<grid, kThreads, 0, stream>>>(p);
    else if (type == kTypeF16) mxfp4_quantize_kernel<__half><<<grid, kThreads, 0, stream>>>(p);
    else mxfp4_quantize_kernel<float><<<grid, kThreads, 0, stream>>>(p);
    return cudaGetLastError();
}

cudaError_t launch_mxfp4_dequantize(const MxConvertParams& p, int type, int sm_count, cudaStream_t stream) {
    const long long units = (long long)p.rows * ((p.cols + 7) / 8);
    const unsigned grid = grid_for(units, kThreads, sm_count);
    if (type == kTypeBf16) mxfp4_dequantize_kernel<__nv_bfloat16><<<grid, kThreads, 0, stream>>>(p);
    else if (type == kTypeF16) mxfp4_dequantize_kernel<__half><<<grid, kThreads, 0, stream>>>(p);
    else mxfp4_dequantize_kernel<float><<<grid, kThreads, 0, stream>>>(p);
    return cudaGetLastError();
}

}  // namespace regenvc
