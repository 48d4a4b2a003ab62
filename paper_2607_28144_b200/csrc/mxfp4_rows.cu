// Product of a few rows with a 4-bit matrix, y = Q(x) w^T + b: the modulation row of a denoising step, embeddings, single
// tokens (and up to four where the matrix is small).  x is quantised in the kernel (or read packed), so such a call is one
// launch.
//
// Bound: the weights' bytes from HBM (17 / 32 byte per weight), and at small sizes the launch itself.  For more than one
// token and 2^24 weights or more the tensor-core product takes over, although it computes 128 rows (2 x 5120 -> 15360: 20.5
// against 46 us; 4 x 5120 -> 5120: 19 against 21 us).  Every thread block first takes all of x to e2m1 values (as fp16,
// which holds them) in shared memory, while its first weights are on their way.  A half warp then walks over groups of FP
// output features: a lane reads 16 bytes = one block of 32 weights per feature, up to eight of them in flight at a time.  Sixteen products are summed in packed fp16 -- exactly:
// products of two e2m1 values are multiples of 1/4 up to 36, and eight of them in one half of a pair stay below 2^11
// quarters -- then joined in fp32 and scaled by the two blocks' powers of two.  Measured, one token: 1536 -> 9216 6.3 us,
// 10240 -> 15360 29 us (84 MB, 2.9 TB/s).
#include "common.cuh"
#include "mx_convert.cuh"
#include "mxfp4.cuh"
#include "row_io.cuh"

namespace regenvc {
namespace {

constexpr int kThreads = 256;
constexpr int kHalfWarps = kThreads / 16;
constexpr int kMostShared = 160 * 1024;   // dynamic shared memory of a thread block, at most
struct Packed {};   // source type of x that is in 4-bit form already

__device__ __forceinline__ float2 sum_pairs(const uint4& a, const uint4& b, const uint4& c, const uint4& d, const uint32_t* w) {
    const uint32_t x[16] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w, c.x, c.y, c.z, c.w, d.x, d.y, d.z, d.w};
    const __half2* xs = reinterpret_cast<const __half2*>(x);
    const __half2* ws = reinterpret_cast<const __half2*>(w);
    __half2 s = __hmul2(xs[0], ws[0]), t = __hmul2(xs[8], ws[8]);
#pragma unroll
    for (int i = 1; i < 8; ++i) {
        s = __hfma2(xs[i], ws[i], s);
        t = __hfma2(xs[i + 8], ws[i + 8], t);
    }
    const float2 f = __half22float2(s), g = __half22float2(t);
    return make_float2(f.x + g.x, f.y + g.y);
}

// sum * 2^(a + b - 254) for scale bytes a and b, without overflow on the way; NaN if either is
__device__ __forceinline__ float scaled(float sum, uint32_t a, uint32_t b) {
    const int e = (int)(a + b) - 254;
    if (e >= -126 && e <= 116 && max(a, b) < 255u) return sum * __uint_as_float((uint32_t)(e + 127) << 23);
    if (a == 255u || b == 255u) return __uint_as_float(0x7FC00000u);
    const int h = e >> 1;
    return sum * __uint_as_float((uint32_t)(h + 127) << 23) * __uint_as_float((uint32_t)(e - h + 127) << 23);
}

// T: element type of x, or Packed.  MR: rows computed (rows past n_tokens are zero and not written).
template <typename T, int MR, int FP>
__global__ void __launch_bounds__(kThreads) mxfp4_rows_kernel(const MxRowsParams p) {
    extern __shared__ uint4 smem4[];
    // [MR][4 pieces][blocks] 16 bytes = 8 values: lanes with neighbouring blocks read neighbouring words
    const int blocks = (int)(p.cols_pad / 32);
    uint4* xv = smem4;
    uint8_t* xscale = reinterpret_cast<uint8_t*>(smem4 + (size_t)MR * 4 * blocks);   // [MR][blocks]
    const int lane = threadIdx.x & 15;

    constexpr int kAhead = 8 / FP;   // blocks per lane and feature in flight
    uint4 q[kAhead][FP];
    uint32_t s[kAhead][FP];
    int f0 = (blockIdx.x * kHalfWarps + (threadIdx.x >> 4)) * FP;   // features is a multiple of 8, so of FP
    auto load = [&](int b0) {
        const uint8_t* codes = p.w + (long long)f0 * (p.cols_pad / 2);
        const uint8_t* scales = p.w + p.w_scale_at + (long long)(f0 / 128) * (p.cols_pad / 128) * 512 + f0 % 32 * 16 + f0 % 128 / 32 * 4;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int b = b0 + 16 * k;
            if (b < blocks)
#pragma unroll
                for (int f = 0; f < FP; ++f) {   // the FP rows lie in one tile of scales: f0 is a multiple of FP
                    q[k][f] = __ldg(reinterpret_cast<const uint4*>(codes + (long long)f * (p.cols_pad / 2)) + b);
                    s[k][f] = __ldg(scales + (long long)(b / 4) * 512 + f * 16 + b % 4);
                }
        }
    };
    if (f0 < p.features) load(lane);

    if constexpr (sizeof(T) == 1) {   // Packed
        const uint8_t* codes = reinterpret_cast<const uint8_t*>(p.x);
        for (int i = threadIdx.x; i < MR * 4 * blocks; i += kThreads) {
            const int m = i / (4 * blocks), j = i - m * 4 * blocks, b = j >> 2, piece = j & 3;
            uint32_t h2[4];
            mx_values8(m < p.n_tokens ? *reinterpret_cast<const uint32_t*>(codes + (long long)m * (p.cols_pad / 2) + j * 4) : 0u, h2);
            xv[(m * 4 + piece) * blocks + b] = make_uint4(h2[0], h2[1], h2[2], h2[3]);
            if (piece == 0) xscale[m * blocks + b] = m < p.n_tokens ? codes[p.x_scale_at + (long long)(b / 4) * 512 + m * 16 + b % 4] : 0;
        }
    } else {
        const int total = MR * blocks * 4;   // a multiple of 16: half warps stay whole
        for (int base = 0; base < total; base += kThreads) {
            const int i = base + threadIdx.x;
            const int m = i / (4 * blocks), j = i - m * 4 * blocks, b = j >> 2, piece = j & 3, c = j * 8;
            float v[8];
            if (i < total && m < p.n_tokens) {
                const T* row = reinterpret_cast<const T*>(p.x) + m * p.x_stride;
                if (p.vec && c + 8 <= p.cols) {
                    widen8(load_raw8(row + c), v);
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = c + k < p.cols ? to_f32(row[c + k]) : 0.0f;
                }
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = 0.0f;
            }
            uint32_t top = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) top = max(top, __float_as_uint(v[k]) & 0x7FFFFFFFu);
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const uint32_t byte = mx_scale_byte(top);
            const float inv = mx_inverse_scale(byte);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = byte == 255u ? 0.0f : v[k] * inv;
            uint32_t h2[4];
            mx_round8(v, h2);
            if (i < total) {
                xv[(m * 4 + piece) * blocks + b] = make_uint4(h2[0], h2[1], h2[2], h2[3]);
                if (piece == 0) xscale[m * blocks + b] = (uint8_t)byte;
            }
        }
    }
    __syncthreads();

    while (f0 < p.features) {
        float acc[FP][MR];
#pragma unroll
        for (int f = 0; f < FP; ++f)
#pragma unroll
            for (int m = 0; m < MR; ++m) acc[f][m] = 0.0f;
        for (int b0 = lane; b0 - lane < blocks; b0 += 16 * kAhead) {
            if (b0 != lane) load(b0);
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int b = b0 + 16 * k;
                if (b < blocks) {
                    uint32_t w[FP][16];
#pragma unroll
                    for (int f = 0; f < FP; ++f) {
                        mx_values8(q[k][f].x, w[f]);
                        mx_values8(q[k][f].y, w[f] + 4);
                        mx_values8(q[k][f].z, w[f] + 8);
                        mx_values8(q[k][f].w, w[f] + 12);
                    }
#pragma unroll
                    for (int m = 0; m < MR; ++m) {
                        const uint4* x = xv + m * 4 * blocks + b;
                        const uint4 x0 = x[0], x1 = x[blocks], x2 = x[2 * blocks], x3 = x[3 * blocks];
                        const uint32_t sx = xscale[m * blocks + b];
#pragma unroll
                        for (int f = 0; f < FP; ++f) {
                            const float2 t = sum_pairs(x0, x1, x2, x3, w[f]);
                            acc[f][m] += scaled(t.x + t.y, s[k][f], sx);
                        }
                    }
                }
            }
        }
        const int done = f0;
        f0 += gridDim.x * kHalfWarps * FP;
        if (f0 < p.features) load(lane);   // the next features' first weights, in flight during the sums
        // (the sixteen lanes of a half warp are here together; the other half may have left the loop)
        const uint32_t mates = 0xFFFFu << (threadIdx.x & 16);
#pragma unroll
        for (int o = 8; o > 0; o >>= 1)
#pragma unroll
            for (int f = 0; f < FP; ++f)
#pragma unroll
                for (int m = 0; m < MR; ++m) acc[f][m] += __shfl_xor_sync(mates, acc[f][m], o);
        if (lane != 0) continue;
#pragma unroll
        for (int m = 0; m < MR; ++m) {
            if (m >= p.n_tokens) continue;
#pragma unroll
            for (int f = 0; f < FP; ++f) {
                const float r = acc[f][m] + (p.bias ? p.bias[done + f] : 0.0f);
                const long long at = (long long)m * p.features + done + f;
                if (p.y_f16) reinterpret_cast<__half*>(p.y)[at] = __float2half_rn(r);
                else reinterpret_cast<__nv_bfloat16*>(p.y)[at] = __float2bfloat16_rn(r);
            }
        }
    }
}

template <typename T, int MR, int FP>
cudaError_t launch_one(const MxRowsParams& p, int sm_count, cudaStream_t stream) {
    const size_t smem = (size_t)MR * (p.cols_pad * 2 + p.cols_pad / 32);
    if (smem > 48000) {
        // always the most that any call takes: the limit is the kernel's, and other host threads launch it at other sizes
        const cudaError_t e = cudaFuncSetAttribute(mxfp4_rows_kernel<T, MR, FP>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostShared);
        if (e != cudaSuccess) return e;
    }
    const int per_block = kHalfWarps * FP;
    int blocks = (p.features + per_block - 1) / per_block;
    if (blocks > sm_count) {   // no more than the device holds at a time: every block quantises x once
        int per_sm = 1;
        const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, mxfp4_rows_kernel<T, MR, FP>, kThreads, smem);
        if (e != cudaSuccess) return e;
        if (per_sm < 1) per_sm = 1;
        if (blocks > per_sm * sm_count) blocks = per_sm * sm_count;
    }
    mxfp4_rows_kernel<T, MR, FP><<<(unsigned)blocks, kThreads, smem, stream>>>(p);
    return cudaGetLastError();
}
template <typename T>
cudaError_t launch_typed(const MxRowsParams& p, int sm_count, cudaStream_t stream) {
    if (p.n_tokens > 1) return launch_one<T, 4, 1>(p, sm_count, stream);
    // two features per half warp once that still gives every SM a block
    if (p.features >= 2 * kHalfWarps * sm_count) return launch_one<T, 1, 2>(p, sm_count, stream);
    return launch_one<T, 1, 1>(p, sm_count, stream);
}

}  // namespace

bool mxfp4_rows_fits(int n_tokens, int features, long long cols_pad) {
    if (n_tokens > kMxFewRows || (n_tokens > 1 && features * cols_pad >= 1ll << 24)) return false;
    return (n_tokens == 1 ? 1 : 4) * (cols_pad * 2 + cols_pad / 32) <= kMostShared;
}

cudaError_t launch_mxfp4_rows(const MxRowsParams& p, int type, bool packed, int sm_count, cudaStream_t stream) {
    if (packed) return launch_typed<Packed>(p, sm_count, stream);
    if (type == kTypeBf16) return launch_typed<__nv_bfloat16>(p, sm_count, stream);
    if (type == kTypeF16) return launch_typed<__half>(p, sm_count, stream);
    return launch_typed<float>(p, sm_count, stream);
}

}  // namespace regenvc
