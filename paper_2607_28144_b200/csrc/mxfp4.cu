// To and from microscaled 4-bit floating point (blocks of 32 along a row share a power-of-two scale; layout in
// mxfp4.cuh).  Bound: HBM in bytes, instructions in practice: with eight values per thread the quantisation issued 110
// instructions per thread and row and kept the schedulers busy for 65 % of its time.  Hence sixteen values per thread --
// two threads hold one block, so its largest magnitude is one exchange away; 32-byte reads, 8-byte codes --, magnitudes
// compared as packed 16-bit patterns, and threads that keep their columns and walk down a range of rows by adding strides,
// several rows of loads in flight at a time.  Measured: quantisation of 31200 x 5120 bf16 80 us (5.0 TB/s), of 10920 x 1536
// 12.8 us; 5120 x 13825 fp32 there and back, element by element, 134 us (4.8 TB/s).
#include "mx_convert.cuh"
#include "mxfp4.cuh"
#include "row_io.cuh"

namespace regenvc {
namespace {

constexpr int kMaxThreads = 256;
constexpr int kWarpCols = 512;            // columns of a warp: four groups of 128
constexpr int kSpread = kWarpCols + kWarpCols / 4;

// Sixteen elements as they lie in memory.
template <typename T>
struct Raw16 {
    uint32_t w[4 * sizeof(T)];
};
// wide: 32-byte accesses are allowed, else 16-byte ones
template <typename T>
__device__ __forceinline__ void load16(Raw16<T>& r, const T* p, bool wide) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
        uint32_t* w = r.w + 8 * i;
        const T* q = p + i * (32 / (int)sizeof(T));
        if (wide) {
            asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(q));
        } else {
            const uint4 a = reinterpret_cast<const uint4*>(q)[0], b = reinterpret_cast<const uint4*>(q)[1];
            w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
        }
    }
}
template <typename T>
__device__ __forceinline__ void store16(T* p, const Raw16<T>& r, bool wide) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
        const uint32_t* w = r.w + 8 * i;
        T* q = p + i * (32 / (int)sizeof(T));
        if (wide) {
            asm volatile("st.global.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                         ::"r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]), "l"(q) : "memory");
        } else {
            reinterpret_cast<uint4*>(q)[0] = make_uint4(w[0], w[1], w[2], w[3]);
            reinterpret_cast<uint4*>(q)[1] = make_uint4(w[4], w[5], w[6], w[7]);
        }
    }
}
template <typename T>
__device__ __forceinline__ void widen16(const Raw16<T>& r, float* v) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r.w[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) widen2(r.w[i], v[2 * i], v[2 * i + 1], (const T*)nullptr);
    }
}
// Largest magnitude as an fp32 bit pattern (magnitudes compare as their bits, NaN above infinity; 16-bit ones as
// unsigned halves).
template <typename T>
__device__ __forceinline__ uint32_t top_of(const Raw16<T>& r) {
    if constexpr (sizeof(T) == 4) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) top = max(top, r.w[i] & 0x7FFFFFFFu);
        return top;
    } else {
        uint32_t m = r.w[0] & 0x7FFF7FFFu;
#pragma unroll
        for (int i = 1; i < 8; ++i) m = __vmaxu2(m, r.w[i] & 0x7FFF7FFFu);
        float a, b;
        widen2(max(m >> 16, m & 0xFFFFu), a, b, (const T*)nullptr);
        return __float_as_uint(a);
    }
}
// Element by element, for rows that do not allow wide accesses: a warp's 512 columns are read with neighbouring lanes on
// neighbouring elements and exchanged through shared memory (16 elements every 20 words, off each other's banks).
__device__ __forceinline__ int spread_at(int e) { return e + (e >> 4) * 4; }
template <typename T>
__device__ __forceinline__ void load_spread(const T* row, int c, int cols, int lane, float* buf, Raw16<float>& r) {
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 16; ++i) buf[spread_at(i * 32 + lane)] = c + i * 32 + lane < cols ? to_f32(row[c + i * 32 + lane]) : 0.0f;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float4 q = *reinterpret_cast<const float4*>(buf + lane * 20 + 4 * i);
        r.w[4 * i] = __float_as_uint(q.x), r.w[4 * i + 1] = __float_as_uint(q.y);
        r.w[4 * i + 2] = __float_as_uint(q.z), r.w[4 * i + 3] = __float_as_uint(q.w);
    }
}

// Place of the scale word (four blocks) of a row in the tiles of one column group, `groups` tiles per 128 rows.
__device__ __forceinline__ long long scale_place(long long row, unsigned groups, unsigned g) {
    return (row / 128 * groups + g) * 512 + (row & 31) * 16 + (row & 127) / 32 * 4;
}

// Codes (eight bytes) and the scales of the 128 columns around, from sixteen values in a thread.
template <typename T>
__device__ __forceinline__ uint2 quantise16(const Raw16<T>& r, int lane, uint32_t* scale_word) {
    uint32_t top = top_of<T>(r);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    const uint32_t byte = mx_scale_byte(top);
    const float inv = mx_inverse_scale(byte);
    float v[16];
    widen16<T>(r, v);
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] *= inv;
    uint2 codes = make_uint2(mx_codes8(v), mx_codes8(v + 8));
    if (byte == 255u) codes = make_uint2(0, 0);
    uint32_t word = byte << (lane >> 1 & 3) * 8;
    word |= __shfl_xor_sync(0xffffffffu, word, 2);
    *scale_word = word | __shfl_xor_sync(0xffffffffu, word, 4);
    return codes;
}

// Thread block (x: range of rows, y: warps' columns).  Rows behind the last one, up to a whole scale tile, get scales of 0.
template <typename T, bool VEC>
__global__ void __launch_bounds__(kMaxThreads) mxfp4_quantize_kernel(const MxConvertParams p, const int rows_per_block) {
    __shared__ alignas(16) float spread[VEC ? 1 : kMaxThreads / 32][VEC ? 4 : kSpread];
    constexpr int kAhead = !VEC ? 1 : (sizeof(T) == 4 ? 2 : 4);   // rows of loads in flight
    // a product launched behind this may set itself up from here on (it starts once every block of this grid has)
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const MxLayout lay(p.rows, p.cols);
    const unsigned groups = (unsigned)(lay.cols_pad / 128);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c0 = (int)(blockIdx.y * (blockDim.x / 32) + warp) * kWarpCols, c = c0 + lane * 16;
    const unsigned g = (unsigned)c / 128;                       // may lie behind the last group: the warp stays whole
    const long long row0 = (long long)blockIdx.x * rows_per_block;
    const long long rows_pad = (lay.rows + 127) / 128 * 128;
    const int rows = (int)(rows_pad - row0 < rows_per_block ? rows_pad - row0 : rows_per_block);
    const int live = (int)(lay.rows - row0 < 0 ? 0 : (lay.rows - row0 < rows ? lay.rows - row0 : rows));
    const long long code_row = lay.cols_pad / 2;
    uint8_t* codes = reinterpret_cast<uint8_t*>(p.dst) + row0 * code_row + c / 2;
    uint8_t* scales = reinterpret_cast<uint8_t*>(p.dst) + lay.scale_at;
    const T* src = reinterpret_cast<const T*>(p.src) + row0 * p.row_stride;
    const bool mine = g < groups, whole = c + 16 <= p.cols, wide = p.vec > 1;
    for (int r = 0; r < rows; r += kAhead) {
        Raw16<T> raw[kAhead];
        if constexpr (VEC) {
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                if (whole && r + k < live) load16(raw[k], src + k * p.row_stride + c, wide);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const bool on = r + k < live;
            const T* row = src + k * p.row_stride;
            uint32_t word;
            uint2 eight;
            if constexpr (VEC) {
                if (!(whole && on)) {   // the last columns of a row, or none
                    Raw16<T> part;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        float f = on && c + i < p.cols ? to_f32(row[c + i]) : 0.0f;
                        T e;
                        from_f32(f, e);
                        if constexpr (sizeof(T) == 4) {
                            part.w[i] = __float_as_uint(e);
                        } else {
                            const uint32_t bits = *reinterpret_cast<const uint16_t*>(&e);
                            part.w[i / 2] = i % 2 ? part.w[i / 2] | bits << 16 : bits;
                        }
                    }
                    raw[k] = part;
                }
                eight = quantise16<T>(raw[k], lane, &word);
            } else {
                Raw16<float> f;
                load_spread(row, c0, on ? p.cols : 0, lane, spread[warp], f);
                eight = quantise16<float>(f, lane, &word);
            }
            if (mine && on) *reinterpret_cast<uint2*>(codes + k * code_row) = eight;
            if (mine && (lane & 7) == 0 && r + k < rows) *reinterpret_cast<uint32_t*>(scales + scale_place(row0 + r + k, groups, g)) = word;
        }
        src += kAhead * p.row_stride;
        codes += kAhead * code_row;
    }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kMaxThreads) mxfp4_dequantize_kernel(const MxConvertParams p, const int rows_per_block) {
    __shared__ alignas(16) float spread[VEC ? 1 : kMaxThreads / 32][VEC ? 4 : kSpread];
    constexpr int kAhead = 4;
    const MxLayout lay(p.rows, p.cols);
    const unsigned groups = (unsigned)(lay.cols_pad / 128);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c0 = (int)(blockIdx.y * (blockDim.x / 32) + warp) * kWarpCols, c = c0 + lane * 16;
    const unsigned g = (unsigned)c / 128;
    const long long row0 = (long long)blockIdx.x * rows_per_block;
    const int rows = (int)(lay.rows - row0 < rows_per_block ? lay.rows - row0 : rows_per_block);
    const long long code_row = lay.cols_pad / 2;
    const uint8_t* codes = reinterpret_cast<const uint8_t*>(p.src) + row0 * code_row + c / 2;
    const uint8_t* scales = reinterpret_cast<const uint8_t*>(p.src) + lay.scale_at + (lane >> 1 & 3);
    T* dst = reinterpret_cast<T*>(p.dst) + row0 * p.row_stride;
    const bool mine = g < groups, whole = c + 16 <= p.cols, wide = p.vec > 1;
    for (int r = 0; r < rows; r += kAhead) {
        uint2 q[kAhead];
        uint32_t s[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            q[k] = make_uint2(0, 0);
            s[k] = 0;
            if (mine && r + k < rows) {
                q[k] = *reinterpret_cast<const uint2*>(codes + k * code_row);
                s[k] = scales[scale_place(row0 + r + k, groups, g)];
            }
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const bool on = mine && r + k < rows;
            T* out = dst + k * p.row_stride;
            uint32_t h2[8];
            float v[16];
            mx_values8(q[k].x, h2);
            mx_values8(q[k].y, h2 + 4);
            const float scale = mx_scale_value(s[k]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                widen2(h2[i], v[2 * i], v[2 * i + 1], (const __half*)nullptr);
                v[2 * i] *= scale;
                v[2 * i + 1] *= scale;
            }
            if constexpr (VEC) {
                if (on && whole) {
                    Raw16<T> w;
                    if constexpr (sizeof(T) == 4) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) w.w[i] = __float_as_uint(v[i]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i) w.w[i] = narrow2(v[2 * i], v[2 * i + 1], (const T*)nullptr);
                    }
                    store16(out + c, w, wide);
                } else if (on) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (c + i < p.cols) from_f32(v[i], out[c + i]);
                }
            } else {
                // the exchange of load_spread() the other way round
                float* buf = spread[warp];
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<float4*>(buf + lane * 20 + 4 * i) = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int e = i * 32 + lane;
                    if (r + k < rows && c0 + e < p.cols) from_f32(buf[spread_at(e)], out[c0 + e]);
                }
            }
        }
        codes += kAhead * code_row;
        dst += kAhead * p.row_stride;
    }
}

// A thread block is up to eight warps side by side; rows per block: a multiple of four, about 1280 threads per SM in all.
struct ConvertPlan {
    dim3 grid;
    int threads, rows;
};
ConvertPlan plan_convert(long long rows, long long cols, int sm_count) {
    ConvertPlan c;
    const long long warps = (cols + kWarpCols - 1) / kWarpCols, across = (warps + 7) / 8;
    const long long each = (warps + across - 1) / across;
    c.threads = (int)each * 32;
    long long down = 40ll * sm_count / (each * across);
    if (down < 1) down = 1;
    long long per = (rows + down - 1) / down;
    per = (per + 3) / 4 * 4;
    if (per > 4096) per = 4096;
    c.rows = (int)per;
    c.grid = dim3((unsigned)((rows + per - 1) / per), (unsigned)across);
    return c;
}

template <typename T>
cudaError_t quantize_typed(const MxConvertParams& p, int sm_count, cudaStream_t stream) {
    const ConvertPlan c = plan_convert(((long long)p.rows + 127) / 128 * 128, p.cols, sm_count);
    if (p.vec) mxfp4_quantize_kernel<T, true><<<c.grid, c.threads, 0, stream>>>(p, c.rows);
    else mxfp4_quantize_kernel<T, false><<<c.grid, c.threads, 0, stream>>>(p, c.rows);
    return cudaGetLastError();
}
template <typename T>
cudaError_t dequantize_typed(const MxConvertParams& p, int sm_count, cudaStream_t stream) {
    const ConvertPlan c = plan_convert(p.rows, p.cols, sm_count);
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
