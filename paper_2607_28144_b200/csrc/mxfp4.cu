// To and from microscaled 4-bit floating point (blocks of 32 along a row share a power-of-two scale; layout in
// mxfp4.cuh).  Bound: HBM.  Sixteen threads take 128 columns of a row, eight each: four threads hold one block, so the
// largest magnitude is two exchanges away, reads are 16 bytes per thread and writes 64 contiguous bytes per row.  A
// thread keeps its columns and walks down a range of rows, four rows of loads in flight at a time: no division per
// element group (with a unit number split into row and column a 31200 x 5120 quantisation took 265 us in 64-bit and 123 us
// in 32-bit arithmetic).
#include "mx_convert.cuh"
#include "mxfp4.cuh"
#include "row_io.cuh"

namespace regenvc {
namespace {

constexpr int kMaxThreads = 256;
constexpr int kRowsAhead = 4;

// Largest magnitude of eight values as an fp32 bit pattern (magnitudes compare as their bits, NaN above infinity).
__device__ __forceinline__ uint32_t top_of(const float* v) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    return top;
}
// The same from packed 16-bit values: the bit patterns of magnitudes compare as unsigned halves.
__device__ __forceinline__ uint32_t top16_of(const uint4& r) {
    const uint32_t m = __vmaxu2(__vmaxu2(r.x & 0x7FFF7FFFu, r.y & 0x7FFF7FFFu), __vmaxu2(r.z & 0x7FFF7FFFu, r.w & 0x7FFF7FFFu));
    return max(m >> 16, m & 0xFFFFu);
}
template <typename T>
__device__ __forceinline__ uint32_t top_raw(const Raw8<T>& r) {
    if constexpr (sizeof(T) == 4) {
        float v[8];
        widen8(r, v);
        return top_of(v);
    } else {
        const uint32_t h = top16_of(r.w[0]);
        float a, b;
        widen2(h, a, b, (const T*)nullptr);
        return __float_as_uint(a);
    }
}

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

// Place of the scale word (four blocks) of a row in the tiles of one column group, `groups` tiles per 128 rows.
__device__ __forceinline__ long long scale_word(long long row, unsigned groups, unsigned g) {
    return (row / 128 * groups + g) * 512 + (row & 31) * 16 + (row & 127) / 32 * 4;
}

// Thread block (x: range of rows, y: column groups of 128, two per warp).  Rows behind the last one, up to a whole scale
// tile, get scales of 0.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kMaxThreads) mxfp4_quantize_kernel(const MxConvertParams p, const int rows_per_block) {
    __shared__ alignas(16) float spread[VEC ? 1 : kMaxThreads / 16][VEC ? 4 : 128];
    const MxLayout lay(p.rows, p.cols);
    const unsigned groups = (unsigned)(lay.cols_pad / 128);
    const int lane = threadIdx.x & 15, half = threadIdx.x >> 4;
    const unsigned g = blockIdx.y * (blockDim.x / 16) + half;   // may lie behind the last group: the warp stays whole
    const int c = (int)g * 128 + lane * 8;
    const long long row0 = (long long)blockIdx.x * rows_per_block;
    const long long rows_pad = (lay.rows + 127) / 128 * 128;
    const int rows = (int)(rows_pad - row0 < rows_per_block ? rows_pad - row0 : rows_per_block);
    const int live = (int)(lay.rows - row0 < 0 ? 0 : (lay.rows - row0 < rows ? lay.rows - row0 : rows));
    uint8_t* codes = reinterpret_cast<uint8_t*>(p.dst) + row0 * (lay.cols_pad / 2) + g * 64 + lane * 4;
    uint8_t* scales = reinterpret_cast<uint8_t*>(p.dst) + lay.scale_at;
    const T* src = reinterpret_cast<const T*>(p.src) + row0 * p.row_stride;
    const bool mine = g < groups, whole = mine && c + 8 <= p.cols;
    for (int r = 0; r < rows; r += kRowsAhead) {
        Raw8<T> raw[kRowsAhead];
        if constexpr (VEC) {
#pragma unroll
            for (int k = 0; k < kRowsAhead; ++k)
                if (whole && r + k < live) raw[k] = load_raw8(src + (r + k) * p.row_stride + c);
        }
#pragma unroll
        for (int k = 0; k < kRowsAhead; ++k) {
            float v[8];
            uint32_t top;
            const T* row = src + (r + k) * p.row_stride;
            const bool on = r + k < live;
            if constexpr (VEC) {
                if (whole && on) {
                    widen8(raw[k], v);
                    top = top_raw(raw[k]);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = mine && on && c + i < p.cols ? to_f32(row[c + i]) : 0.0f;
                    top = top_of(v);
                }
            } else {
                load_spread(row, (int)g * 128, mine && on ? p.cols : 0, lane, spread[half], v);
                top = top_of(v);
            }
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const uint32_t byte = mx_scale_byte(top);
            const float inv = mx_inverse_scale(byte);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= inv;
            const uint32_t eight = byte == 255u ? 0u : mx_codes8(v);
            // the four scales of these 128 columns side by side
            uint32_t word = byte << (lane >> 2) * 8;
            word |= __shfl_xor_sync(0xffffffffu, word, 4);
            word |= __shfl_xor_sync(0xffffffffu, word, 8);
            if (mine && on) *reinterpret_cast<uint32_t*>(codes + (r + k) * (lay.cols_pad / 2)) = eight;
            if (mine && lane == 0 && r + k < rows) *reinterpret_cast<uint32_t*>(scales + scale_word(row0 + r + k, groups, g)) = word;
        }
    }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kMaxThreads) mxfp4_dequantize_kernel(const MxConvertParams p, const int rows_per_block) {
    __shared__ alignas(16) float spread[VEC ? 1 : kMaxThreads / 16][VEC ? 4 : 128];
    const MxLayout lay(p.rows, p.cols);
    const unsigned groups = (unsigned)(lay.cols_pad / 128);
    const int lane = threadIdx.x & 15, half = threadIdx.x >> 4;
    const unsigned g = blockIdx.y * (blockDim.x / 16) + half;
    const int c = (int)g * 128 + lane * 8;
    const long long row0 = (long long)blockIdx.x * rows_per_block;
    const int rows = (int)(lay.rows - row0 < rows_per_block ? lay.rows - row0 : rows_per_block);
    const uint8_t* codes = reinterpret_cast<const uint8_t*>(p.src) + row0 * (lay.cols_pad / 2) + g * 64 + lane * 4;
    const uint8_t* scales = reinterpret_cast<const uint8_t*>(p.src) + lay.scale_at + lane / 4;
    T* dst = reinterpret_cast<T*>(p.dst) + row0 * p.row_stride;
    const bool mine = g < groups;
    for (int r = 0; r < rows; r += kRowsAhead) {
        uint32_t q[kRowsAhead], s[kRowsAhead];
#pragma unroll
        for (int k = 0; k < kRowsAhead; ++k) {
            q[k] = s[k] = 0;
            if (mine && r + k < rows) {
                q[k] = *reinterpret_cast<const uint32_t*>(codes + (r + k) * (lay.cols_pad / 2));
                s[k] = scales[scale_word(row0 + r + k, groups, g)];
            }
        }
#pragma unroll
        for (int k = 0; k < kRowsAhead; ++k) {
            const bool on = mine && r + k < rows;
            T* out = dst + (r + k) * p.row_stride;
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
            if constexpr (VEC) {
                if (on && c + 8 <= p.cols) {
                    store8(out + c, v);
                } else if (on) {
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
                    if (on && e < p.cols) from_f32(buf[i * 16 + lane], out[e]);
                }
            }
        }
    }
}

// Threads: two column groups per warp, at most eight warps; rows per block: a multiple of kRowsAhead, about five blocks of
// 256 threads per SM in all.
struct ConvertPlan {
    dim3 grid;
    int threads, rows;
};
ConvertPlan plan_convert(long long rows, long long groups, int sm_count) {
    ConvertPlan c;
    c.threads = (int)(groups >= 16 ? 256 : (groups + 1) / 2 * 32);
    const long long across = (groups + c.threads / 16 - 1) / (c.threads / 16);
    long long down = 5ll * sm_count * (256 / c.threads) / across;
    if (down < 1) down = 1;
    long long per = (rows + down - 1) / down;
    per = (per + kRowsAhead - 1) / kRowsAhead * kRowsAhead;
    if (per > 4096) per = 4096;
    c.rows = (int)per;
    c.grid = dim3((unsigned)((rows + per - 1) / per), (unsigned)across);
    return c;
}

template <typename T>
cudaError_t quantize_typed(const MxConvertParams& p, int sm_count, cudaStream_t stream) {
    const ConvertPlan c = plan_convert(((long long)p.rows + 127) / 128 * 128, ((long long)p.cols + 127) / 128, sm_count);
    if (p.vec) mxfp4_quantize_kernel<T, true><<<c.grid, c.threads, 0, stream>>>(p, c.rows);
    else mxfp4_quantize_kernel<T, false><<<c.grid, c.threads, 0, stream>>>(p, c.rows);
    return cudaGetLastError();
}
template <typename T>
cudaError_t dequantize_typed(const MxConvertParams& p, int sm_count, cudaStream_t stream) {
    const ConvertPlan c = plan_convert(p.rows, ((long long)p.cols + 127) / 128, sm_count);
    if (p.vec) mxfp4_dequantize_kernel<T, true><<<c.grid, c.threads, 0, stream>>>(p, c.rows);
    else mxfp4_dequantize_kernel<T, false><<<c.grid, c.threads, 0, stream>>>(p, c.rows);
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
