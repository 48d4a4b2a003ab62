// To and from microscaled 4-bit floating point (blocks of 32 along a row share a power-of-two scale; layout in
// mxfp4.cuh).  Bound: HBM.  Sixteen threads take 128 columns of a row, eight each: four threads hold one block, so the
// largest magnitude is two exchanges away, reads are 16 bytes per thread and writes 64 contiguous bytes per row.
#include "mx_convert.cuh"
#include "mxfp4.cuh"
#include "row_io.cuh"

namespace regenvc {
namespace {

constexpr int kThreads = 256;
constexpr int kGroups = kThreads / 16;   // half warps: groups of 128 columns in hand at a time
constexpr int kUnroll = 4;

// A half warp's 128 values where rows do not allow 16-byte accesses: lane l reads elements l, l + 16, ... (neighbouring
// lanes neighbouring elements), and an exchange through shared memory gives it elements 8l .. 8l + 7.
template <typename T>
__device__ __forceinline__ void load_spread(const T* row, int c, int cols, int lane, float* buf, float* v) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i * 16 + lane < cols ? to_f32(row[c + i * 16 + lane]) : 0.0f;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 8; ++i) buf[i * 16 + lane] = v[i];
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float4 q = reinterpret_cast<const float4*>(buf)[lane * 2 + i];
        v[4 * i] = q.x, v[4 * i + 1] = q.y, v[4 * i + 2] = q.z, v[4 * i + 3] = q.w;
    }
}

// One thread's eight values of 128 columns: codes, and the scales of the four blocks as one word (in every lane).
__device__ __forceinline__ uint32_t quantise_eight(float* v, int lane, uint32_t* scale_word) {
    uint32_t top = 0;   // magnitudes compare as their bit patterns, NaN above infinity
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const uint32_t byte = mx_scale_byte(top);
    const float inv = mx_inverse_scale(byte);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = byte == 255u ? 0.0f : v[i] * inv;
    uint32_t word = byte << (lane >> 2) * 8;
    word |= __shfl_xor_sync(0xffffffffu, word, 4);
    *scale_word = word | __shfl_xor_sync(0xffffffffu, word, 8);
    return mx_codes8(v);
}

// A thread block takes `rows_per_block` rows (of the rows rounded up to whole scale tiles: behind the last row only scales
// are written); a half warp takes 128 columns of one of them at a time.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) mxfp4_quantize_kernel(const MxConvertParams p, const int rows_per_block) {
    __shared__ alignas(16) float spread[VEC ? 1 : kGroups][VEC ? 4 : 128];
    const MxLayout lay(p.rows, p.cols);
    const unsigned groups = (unsigned)(lay.cols_pad / 128);
    const long long row0 = (long long)blockIdx.x * rows_per_block;
    const unsigned total = rows_per_block * groups;
    const int lane = threadIdx.x & 15;
    const unsigned half = threadIdx.x >> 4;
    uint8_t* codes = reinterpret_cast<uint8_t*>(p.dst) + row0 * (lay.cols_pad / 2);
    uint8_t* scales = reinterpret_cast<uint8_t*>(p.dst) + lay.scale_at;
    const T* src = reinterpret_cast<const T*>(p.src) + row0 * p.row_stride;
    const int live = (int)(p.rows - row0 < rows_per_block ? (p.rows - row0 > 0 ? p.rows - row0 : 0) : rows_per_block);
    constexpr int kBatch = VEC ? kUnroll : 1;
    // whole warps take part in the exchanges: the trip count is that of the block's first half warp
    for (unsigned base = 0; base < total; base += kGroups * kBatch) {
        Raw8<T> raw[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const unsigned u = base + k * kGroups + half, r = u / groups;
            const int c = (int)(u - r * groups) * 128 + lane * 8;
            if (VEC && (int)r < live && c + 8 <= p.cols) raw[k] = load_raw8(src + (long long)r * p.row_stride + c);
        }
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const unsigned u = base + k * kGroups + half, r = u / groups, g = u - r * groups;
            const int c = (int)g * 128 + lane * 8;
            float v[8];
            const T* row = src + (long long)r * p.row_stride;
            if constexpr (VEC) {
                if ((int)r < live && c + 8 <= p.cols) {
                    widen8(raw[k], v);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = (int)r < live && c + i < p.cols ? to_f32(row[c + i]) : 0.0f;
                }
            } else {
                load_spread(row, (int)g * 128, (int)r < live ? p.cols : 0, lane, spread[half], v);
            }
            uint32_t word;
            const uint32_t eight = quantise_eight(v, lane, &word);
            if (u >= total) continue;
            if ((int)r < live) *reinterpret_cast<uint32_t*>(codes + (long long)r * (lay.cols_pad / 2) + g * 64 + lane * 4) = eight;
            const long long row_at = row0 + r;
            if (lane == 0)
                *reinterpret_cast<uint32_t*>(scales + (row_at / 128 * groups + g) * 512 + row_at % 32 * 16 + row_at % 128 / 32 * 4) = word;
        }
    }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) mxfp4_dequantize_kernel(const MxConvertParams p, const int rows_per_block) {
    __shared__ alignas(16) float spread[VEC ? 1 : kGroups][VEC ? 4 : 128];
    const MxLayout lay(p.rows, p.cols);
    const unsigned groups = (unsigned)(lay.cols_pad / 128);
    const long long row0 = (long long)blockIdx.x * rows_per_block;
    const int live = (int)(p.rows - row0 < rows_per_block ? p.rows - row0 : rows_per_block);
    const unsigned total = live * groups;
    const int lane = threadIdx.x & 15;
    const unsigned half = threadIdx.x >> 4;
    const uint8_t* codes = reinterpret_cast<const uint8_t*>(p.src) + row0 * (lay.cols_pad / 2);
    const uint8_t* scales = reinterpret_cast<const uint8_t*>(p.src) + lay.scale_at;
    T* dst = reinterpret_cast<T*>(p.dst) + row0 * p.row_stride;
    for (unsigned base = 0; base < total; base += kGroups * kUnroll) {
        uint32_t q[kUnroll], s[kUnroll];
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) {
            const unsigned u = base + k * kGroups + half, r = u / groups, g = u - r * groups;
            if (u >= total) continue;
            const long long row_at = row0 + r;
            q[k] = *reinterpret_cast<const uint32_t*>(codes + (long long)r * (lay.cols_pad / 2) + g * 64 + lane * 4);
            s[k] = scales[(row_at / 128 * groups + g) * 512 + row_at % 32 * 16 + row_at % 128 / 32 * 4 + lane / 4];
        }
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) {
            const unsigned u = base + k * kGroups + half, r = u / groups, g = u - r * groups;
            const int c = (int)g * 128 + lane * 8;
            T* out = dst + (long long)r * p.row_stride;
            uint32_t h2[4];
            float v[8];
            mx_values8(u < total ? q[k] : 0u, h2);
            const float scale = mx_scale_value(u < total ? s[k] : 0u);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                widen2(h2[i], v[2 * i], v[2 * i + 1], (const __half*)nullptr);
                v[2 * i] *= scale;
                v[2 * i + 1] *= scale;
            }
            if constexpr (VEC) {
                if (u >= total) continue;
                if (c + 8 <= p.cols) {
                    store8(out + c, v);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (c + i < p.cols) from_f32(v[i], out[c + i]);
                }
            } else {
                // the exchange of load_spread() the other way round
                float* buf = spread[half];
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    reinterpret_cast<float4*>(buf)[lane * 2 + i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int e = (int)g * 128 + i * 16 + lane;
                    if (u < total && e < p.cols) from_f32(buf[i * 16 + lane], out[e]);
                }
            }
        }
    }
}

// Rows per thread block: one while that leaves no more blocks than the device holds at a time, at most eight.
int rows_per_block(long long rows, int sm_count) {
    long long r = rows / (8ll * sm_count);
    return (int)(r < 1 ? 1 : (r > 8 ? 8 : r));
}

template <typename T>
cudaError_t quantize_typed(const MxConvertParams& p, int sm_count, cudaStream_t stream) {
    const long long rows = ((long long)p.rows + 127) / 128 * 128;
    const int per = rows_per_block(rows, sm_count);
    const unsigned grid = (unsigned)((rows + per - 1) / per);
    if (p.vec) mxfp4_quantize_kernel<T, true><<<grid, kThreads, 0, stream>>>(p, per);
    else mxfp4_quantize_kernel<T, false><<<grid, kThreads, 0, stream>>>(p, per);
    return cudaGetLastError();
}
template <typename T>
cudaError_t dequantize_typed(const MxConvertParams& p, int sm_count, cudaStream_t stream) {
    const int per = rows_per_block(p.rows, sm_count);
    const unsigned grid = (unsigned)(((long long)p.rows + per - 1) / per);
    if (p.vec) mxfp4_dequantize_kernel<T, true><<<grid, kThreads, 0, stream>>>(p, per);
    else mxfp4_dequantize_kernel<T, false><<<grid, kThreads, 0, stream>>>(p, per);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_mxfp4_quantize(const MxConvertParams& p, int type, int sm_count, cudaStream_t stream) {
    if (type == kTypeBf16) return quantize_typed<__nv_bfloat16>(p, sm_count, stream);
    if (type == kTypeF16) return quantize_typed<__half>(p, sm_count, stream);
    return quantize_typed<float>(p, sm_count, stream);
}

cudaError_t launch_mxfp4_dequantize(const MxConvertParams& p, int type, int sm_count, cudaStream_t stream) {
    if (type == kTypeBf16) return dequantize_typed<__nv_bfloat16>(p, sm_count, stream);
    if (type == kTypeF16) return dequantize_typed<__half>(p, sm_count, stream);
    return dequantize_typed<float>(p, sm_count, stream);
}

}  // namespace regenvc
