// Norms before and after a transformer block, fused with the block's gate and residual scale, and their gradients.
//
//     z  = N2(y) pw  (or y)          x' = a x + g z          h = (N1(x') w + b) (1 + s) + t
//
// N is layer norm ((v - mean) r, r = 1 / sqrt(var + eps)) or RMS norm (v r, r = 1 / sqrt(mean v^2 + eps)); g, s, t are
// rows of a modulation table shared by tokens_per_mod consecutive tokens.  With xhat = N1(x'), yhat = N2(y):
//
//     d  = dh (1 + s) w                                dx' = r (d - [layer] mean(d) - xhat mean(d xhat)) + dx'_in
//     dt = S0,  ds = w S1 + b S0,                      dw = sum_rows (1 + s) S1,  db = sum_rows (1 + s) S0
//     dz = g dx',  dy = N2's gradient of dz pw         dg = pw S2,  dpw = sum_rows g S2,    dx = a dx'
//     S0 = sum dh,  S1 = sum dh xhat,  S2 = sum dx' yhat  over the tokens of one modulation row
//
// Bound: HBM (every tensor is read or written once; 8 bytes per element forward in bf16).  A thread block owns a
// contiguous range of tokens and a thread eight fixed columns, for two reasons: the modulation, weight and bias values
// of a column stay in registers over all tokens that share them (read per token they would be 12 bytes of fp32 against
// 8 bytes of tokens), and the backward pass can sum over tokens in registers too, without atomics, in an order that
// depends on the shape alone.  Statistics take two passes over registers (mean, then centred squares) in fp32.
#include "block_norm.cuh"
#include "row_io.cuh"

namespace regenvc {
namespace {

// One thread's eight columns of a row: neighbouring (one or two 16-byte words) or, where sizes, strides or addresses
// do not allow that, `threads` apart and element by element.
template <typename T, bool VEC>
struct Cols;
template <typename T>
struct Cols<T, true> {
    Raw8<T> r;
    __device__ __forceinline__ void load(const void* base, long long row, long long stride, int c0, int, unsigned live) {
        if (live) r = load_raw8(reinterpret_cast<const T*>(base) + row * stride + c0);
    }
    __device__ __forceinline__ void widen(float* v, unsigned live) const {
        if (live) {
            widen8(r, v);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.0f;
        }
    }
    static __device__ __forceinline__ void store(void* base, long long row, long long stride, int c0, int, unsigned live,
                                                 const float* v) {
        if (live) store8(reinterpret_cast<T*>(base) + row * stride + c0, v);
    }
};
template <typename T>
struct Cols<T, false> {
    T e[8];
    __device__ __forceinline__ void load(const void* base, long long row, long long stride, int c0, int step, unsigned live) {
        const T* p = reinterpret_cast<const T*>(base) + row * stride + c0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (live >> i & 1) e[i] = p[i * step];
    }
    __device__ __forceinline__ void widen(float* v, unsigned live) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (live >> i & 1) ? to_f32(e[i]) : 0.0f;
    }
    static __device__ __forceinline__ void store(void* base, long long row, long long stride, int c0, int step, unsigned live,
                                                 const float* v) {
        T* p = reinterpret_cast<T*>(base) + row * stride + c0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (live >> i & 1) from_f32(v[i], p[i * step]);
    }
};

template <bool VEC>
__device__ __forceinline__ void vector8(const float* base, float absent, int c0, int step, unsigned live, float* v) {
    if (base == nullptr || !live) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = absent;
    } else if constexpr (VEC) {
        const float4 a = __ldg(reinterpret_cast<const float4*>(base + c0)), b = __ldg(reinterpret_cast<const float4*>(base + c0) + 1);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (live >> i & 1) ? __ldg(base + c0 + i * step) : absent;
    }
}

// Sums over the thread block, the same value in every thread, in a fixed order.  Two buffers used in turn make one
// barrier per sum enough: a buffer is written again only behind the next sum's barrier.
struct BlockSum {
    float (*buf)[2][32];   // [2 buffers][2 values][warp]
    int warps, turn;
    template <int N>
    __device__ __forceinline__ void run(float* v) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
#pragma unroll
            for (int n = 0; n < N; ++n) v[n] += __shfl_xor_sync(0xffffffffu, v[n], o);
        if (warps == 1) return;
        float (*b)[32] = buf[turn];
        turn ^= 1;
        if ((threadIdx.x & 31) == 0)
#pragma unroll
            for (int n = 0; n < N; ++n) b[n][threadIdx.x >> 5] = v[n];
        __syncthreads();
#pragma unroll
        for (int n = 0; n < N; ++n) {
            float s = 0.0f;
            for (int w = 0; w < warps; w += 4) {
                const float4 q = *reinterpret_cast<const float4*>(&b[n][w]);
                s += (q.x + q.y) + (q.z + q.w);
            }
            v[n] = s;
        }
    }
};
__device__ __forceinline__ BlockSum block_sum_init(float (*buf)[2][32]) {
    for (int i = threadIdx.x; i < 128; i += blockDim.x) (&buf[0][0][0])[i] = 0.0f;   // entries past the last warp stay 0
    __syncthreads();
    return BlockSum{buf, (int)(blockDim.x + 31) / 32, 0};
}

// v -> normalised v (dead columns hold and keep 0); returns the reciprocal deviation.
__device__ __forceinline__ float normalise(float* v, int kind, float eps, float channels, unsigned live, bool vec, BlockSum& sum) {
    float s[1];
    if (kind == kNormLayer) {
        s[0] = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s[0] += v[i];
        sum.run<1>(s);
        const float mean = s[0] / channels;   // (a product with 1 / channels would leave a constant row a mean off by an ulp)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (vec ? live != 0 : (live >> i & 1) != 0) ? v[i] - mean : 0.0f;
    }
    s[0] = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s[0] = fmaf(v[i], v[i], s[0]);
    sum.run<1>(s);
    const float r = rsqrtf(s[0] / channels + eps);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= r;
    return r;
}

__device__ __forceinline__ unsigned live_columns(int channels, bool vec, int* c0, int* step) {
    const int tid = threadIdx.x, threads = blockDim.x;
    unsigned live = 0;
    if (vec) {
        *c0 = tid * 8;
        *step = 1;
        live = *c0 < channels ? 0xFFu : 0u;
    } else {
        *c0 = tid;
        *step = threads;
#pragma unroll
        for (int i = 0; i < 8; ++i) live |= (tid + i * threads < channels ? 1u : 0u) << i;
    }
    return live;
}

template <typename TX, typename TIO, bool VEC, int MAXT>
__global__ void __launch_bounds__(MAXT) block_norm_forward_kernel(const BlockNormParams p) {
    __shared__ alignas(16) float buf[2][2][32];
    BlockSum sum = block_sum_init(buf);
    int c0, step;
    const unsigned live = live_columns(p.channels, VEC, &c0, &step);
    const float channels = (float)p.channels;
    const int row0 = blockIdx.x * p.rows_per_cta;
    const int row1 = min(p.n_tokens, row0 + p.rows_per_cta);
    int mod = -1, mod_end = row0;   // modulation row held in registers, and its first token behind
    float w[8], b[8], g[8];
    Cols<TX, VEC> nx;
    Cols<TIO, VEC> ny;
    nx.load(p.x, row0, p.x_stride, c0, step, live);
    if (p.y) ny.load(p.y, row0, p.y_stride, c0, step, live);
    for (int row = row0; row < row1; ++row) {
        float v[8], z[8];
        nx.widen(v, live);
        if (p.y) ny.widen(z, live);
        // the next row's loads are in flight during this row's sums
        if (row + 1 < row1) {
            nx.load(p.x, row + 1, p.x_stride, c0, step, live);
            if (p.y) ny.load(p.y, row + 1, p.y_stride, c0, step, live);
        }
        if (row >= mod_end) {
            mod = row / p.tokens_per_mod;
            mod_end = p.tokens_per_mod < p.n_tokens - mod * p.tokens_per_mod ? (mod + 1) * p.tokens_per_mod : p.n_tokens;
            const long long at = mod * p.mod_stride;
            float t[8];
            vector8<VEC>(p.weight, 1.0f, c0, step, live, w);
            vector8<VEC>(p.bias, 0.0f, c0, step, live, b);
            vector8<VEC>(p.scale ? p.scale + at : nullptr, 0.0f, c0, step, live, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[i] = fmaf(w[i], t[i], w[i]);
                b[i] = fmaf(b[i], t[i], b[i]);
            }
            vector8<VEC>(p.shift ? p.shift + at : nullptr, 0.0f, c0, step, live, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) b[i] += t[i];
            vector8<VEC>(p.gate ? p.gate + at : nullptr, 1.0f, c0, step, live, g);
            vector8<VEC>(p.post_weight, 1.0f, c0, step, live, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) g[i] *= t[i];
        }
        if (p.y) {
            if (p.post_norm) normalise(z, p.post_norm, p.post_eps, channels, live, VEC, sum);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = fmaf(g[i], z[i], p.residual_scale * v[i]);
            if (p.x_out) Cols<TX, VEC>::store(p.x_out, row, p.x_out_stride, c0, step, live, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (VEC ? live != 0 : (live >> i & 1) != 0) ? v[i] : 0.0f;
        }
        if (p.norm) {   // on x' before its rounding to the residual stream's type
            normalise(v, p.norm, p.eps, channels, live, VEC, sum);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = fmaf(v[i], w[i], b[i]);
            Cols<TIO, VEC>::store(p.h, row, p.h_stride, c0, step, live, v);
        }
    }
}

// Results of a modulation row from its three sums, for one column.
__device__ __forceinline__ void write_mod_grads(const BlockNormParams& p, long long mod, int c, float s0, float s1, float s2) {
    const long long at = mod * p.channels + c;
    if (p.dshift) p.dshift[at] = s0;
    if (p.dscale) p.dscale[at] = fmaf(p.weight ? p.weight[c] : 1.0f, s1, (p.bias ? p.bias[c] : 0.0f) * s0);
    if (p.dgate) p.dgate[at] = (p.post_weight ? p.post_weight[c] : 1.0f) * s2;
}

// Workspace: per thread block two slots of [3][channels] sums (its first modulation row, and its last one where that is
// another) that are not complete inside the block, then [3][channels] of sums for the weights' gradients.
__device__ __forceinline__ float* slot_of(const BlockNormParams& p, int cta, int which) {
    return p.partials + ((long long)cta * 9 + which * 3) * p.channels;
}

template <typename TX, typename TIO, bool VEC, int MAXT>
__global__ void __launch_bounds__(MAXT) block_norm_backward_kernel(const BlockNormParams p) {
    __shared__ alignas(16) float buf[2][2][32];
    extern __shared__ float wsum[];   // [3][channels] if a weight's gradient is wanted; every column has one owner
    BlockSum sum = block_sum_init(buf);
    int c0, step;
    const unsigned live = live_columns(p.channels, VEC, &c0, &step);
    const float channels = (float)p.channels;
    const int row0 = blockIdx.x * p.rows_per_cta;
    const int row1 = min(p.n_tokens, row0 + p.rows_per_cta);
    const int first_mod = row0 / p.tokens_per_mod;
    const bool want_w = p.dweight || p.dbias || p.dpost_weight;
    const bool want_mod = p.dscale || p.dshift || p.dgate;
    if (want_w)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (live >> i & 1)
#pragma unroll
                for (int k = 0; k < 3; ++k) wsum[k * p.channels + c0 + i * step] = 0.0f;

    float s0[8], s1[8], s2[8], w[8], g[8];
    for (int row = row0; row < row1;) {
        const int mod = row / p.tokens_per_mod;
        const int begin = mod * p.tokens_per_mod;
        const int whole_end = p.tokens_per_mod < p.n_tokens - begin ? begin + p.tokens_per_mod : p.n_tokens;
        const int end = min(row1, whole_end);
        const bool complete = row == begin && end == whole_end;
        const long long at = mod * p.mod_stride;
        {
            float t[8];
            vector8<VEC>(p.weight, 1.0f, c0, step, live, w);
            vector8<VEC>(p.scale ? p.scale + at : nullptr, 0.0f, c0, step, live, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = fmaf(w[i], t[i], w[i]);
            vector8<VEC>(p.gate ? p.gate + at : nullptr, 1.0f, c0, step, live, g);
            vector8<VEC>(p.post_weight, 1.0f, c0, step, live, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                g[i] *= t[i];
                s0[i] = s1[i] = s2[i] = 0.0f;
            }
        }
        for (; row < end; ++row) {
            float xh[8], d[8];
            Cols<TX, VEC> rx, rdx;
            Cols<TIO, VEC> rdh, ry;
            if (p.norm) {
                rx.load(p.x, row, p.x_stride, c0, step, live);
                rdh.load(p.dh, row, p.h_stride, c0, step, live);
            }
            if (p.dx_out) rdx.load(p.dx_out, row, p.dx_out_stride, c0, step, live);
            if (p.y) ry.load(p.y, row, p.y_stride, c0, step, live);
            if (p.norm) {
                float t[2] = {0.0f, 0.0f};
                rx.widen(xh, live);
                rdh.widen(d, live);
                const float r = normalise(xh, p.norm, p.eps, channels, live, VEC, sum);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    s0[i] += d[i];
                    s1[i] = fmaf(d[i], xh[i], s1[i]);
                    d[i] *= w[i];
                    t[0] += d[i];
                    t[1] = fmaf(d[i], xh[i], t[1]);
                }
                sum.run<2>(t);
                const float m0 = p.norm == kNormLayer ? t[0] / channels : 0.0f, m1 = t[1] / channels;
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] = r * (d[i] - fmaf(xh[i], m1, m0));
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] = 0.0f;
            }
            if (p.dx_out) {
                rdx.widen(xh, live);
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] += xh[i];
            }
            if (p.dx) {
#pragma unroll
                for (int i = 0; i < 8; ++i) xh[i] = p.residual_scale * d[i];
                Cols<TX, VEC>::store(p.dx, row, p.dx_stride, c0, step, live, xh);
            }
            if (p.y) {
                float yh[8];
                ry.widen(yh, live);
                float r = 1.0f;
                if (p.post_norm) r = normalise(yh, p.post_norm, p.post_eps, channels, live, VEC, sum);
                float t[2] = {0.0f, 0.0f};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const bool on = VEC ? live != 0 : (live >> i & 1) != 0;
                    s2[i] = fmaf(d[i], yh[i], s2[i]);
                    d[i] = on ? d[i] * g[i] : 0.0f;
                    t[0] += d[i];
                    t[1] = fmaf(d[i], yh[i], t[1]);
                }
                if (p.post_norm) {
                    sum.run<2>(t);
                    const float m0 = p.post_norm == kNormLayer ? t[0] / channels : 0.0f, m1 = t[1] / channels;
#pragma unroll
                    for (int i = 0; i < 8; ++i) d[i] = r * (d[i] - fmaf(yh[i], m1, m0));
                }
                if (p.dy) Cols<TIO, VEC>::store(p.dy, row, p.dy_stride, c0, step, live, d);
            }
        }
        // the modulation row's sums: final where all of its tokens are this block's, else a slot of the workspace
        if (want_w || want_mod) {
            float* slot = slot_of(p, blockIdx.x, mod == first_mod ? 0 : 1);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (!(live >> i & 1)) continue;
                const int c = c0 + i * step;
                if (want_w) {
                    const float s = p.scale ? 1.0f + p.scale[at + c] : 1.0f;
                    wsum[c] = fmaf(s, s1[i], wsum[c]);
                    wsum[p.channels + c] = fmaf(s, s0[i], wsum[p.channels + c]);
                    wsum[2 * p.channels + c] = fmaf(p.gate ? p.gate[at + c] : 1.0f, s2[i], wsum[2 * p.channels + c]);
                }
                if (!want_mod) continue;
                if (complete) {
                    write_mod_grads(p, mod, c, s0[i], s1[i], s2[i]);
                } else {
                    slot[c] = s0[i];
                    slot[p.channels + c] = s1[i];
                    slot[2 * p.channels + c] = s2[i];
                }
            }
        }
    }
    if (want_w) {
        float* out = slot_of(p, blockIdx.x, 2);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (live >> i & 1)
#pragma unroll
                for (int k = 0; k < 3; ++k) out[k * p.channels + c0 + i * step] = wsum[k * p.channels + c0 + i * step];
    }
}

// Joins the slots.  Thread block (32 columns, job): 32 lanes of threads take every 32nd slot each, then one of them
// adds the 32 sums.  Jobs below n_jobs are modulation rows that no single thread block of the first kernel held whole;
// job n_jobs is the weights' gradients.
__global__ void __launch_bounds__(1024) block_norm_join_kernel(const BlockNormParams p, const int n_ctas, const int n_jobs,
                                                              const int by_boundary) {
    __shared__ float part[3][32][33];
    const int c = blockIdx.x * 32 + threadIdx.x, lane = threadIdx.y, job = blockIdx.y;
    const bool weights = job == n_jobs;
    int mod = job, a = 0, b = n_ctas;
    if (!weights) {
        if (by_boundary) {
            // the modulation row, if any, that runs over the end of thread block `job` (rows shorter than a block's
            // range: at most two blocks hold one)
            const long long token = (long long)(job + 1) * p.rows_per_cta;
            mod = (int)(token / p.tokens_per_mod);
            if (token % p.tokens_per_mod == 0) return;
        }
        const long long t0 = (long long)mod * p.tokens_per_mod;
        const long long t1 = t0 + p.tokens_per_mod < p.n_tokens ? t0 + p.tokens_per_mod : p.n_tokens;
        a = (int)(t0 / p.rows_per_cta);
        b = (int)((t1 - 1) / p.rows_per_cta) + 1;
        if (b - a < 2) return;   // complete already
    }
    float s[3] = {0.0f, 0.0f, 0.0f};
    if (c < p.channels)
        for (int cta = a + lane; cta < b; cta += 32) {
            const int which = weights ? 2 : ((long long)cta * p.rows_per_cta / p.tokens_per_mod == mod ? 0 : 1);
            const float* slot = slot_of(p, cta, which) + c;
#pragma unroll
            for (int k = 0; k < 3; ++k) s[k] += slot[(long long)k * p.channels];
        }
#pragma unroll
    for (int k = 0; k < 3; ++k) part[k][lane][threadIdx.x] = s[k];
    __syncthreads();
    if (lane != 0 || c >= p.channels) return;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        s[k] = 0.0f;
        for (int i = 0; i < 32; ++i) s[k] += part[k][i][threadIdx.x];
    }
    if (weights) {
        if (p.dweight) p.dweight[c] = s[0];
        if (p.dbias) p.dbias[c] = s[1];
        if (p.dpost_weight) p.dpost_weight[c] = s[2];
    } else {
        write_mod_grads(p, mod, c, s[0], s[1], s[2]);
    }
}

int threads_for(int channels) { return (channels + 255) / 256 * 32; }

// Thread blocks and rows per thread block: about `per_sm_threads` threads per SM, at most kNormMaxCtas blocks.
int plan_rows(BlockNormParams* p, int per_sm_threads, int sm_count) {
    int per_sm = per_sm_threads / threads_for(p->channels);
    if (per_sm < 1) per_sm = 1;
    int most = per_sm * sm_count;
    if (most > kNormMaxCtas) most = kNormMaxCtas;
    if (most > p->n_tokens) most = p->n_tokens;
    p->rows_per_cta = (p->n_tokens + most - 1) / most;
    return (p->n_tokens + p->rows_per_cta - 1) / p->rows_per_cta;
}

template <typename TX, typename TIO, bool VEC>
cudaError_t forward_sized(const BlockNormParams& p, int ctas, cudaStream_t stream) {
    const int threads = threads_for(p.channels);
    if constexpr (!VEC) {   // element by element: one build for every size
        block_norm_forward_kernel<TX, TIO, VEC, 1024><<<ctas, threads, 0, stream>>>(p);
        return cudaGetLastError();
    }
    if (threads <= 256) block_norm_forward_kernel<TX, TIO, VEC, 256><<<ctas, threads, 0, stream>>>(p);
    else if (threads <= 640) block_norm_forward_kernel<TX, TIO, VEC, 640><<<ctas, threads, 0, stream>>>(p);
    else block_norm_forward_kernel<TX, TIO, VEC, 1024><<<ctas, threads, 0, stream>>>(p);
    return cudaGetLastError();
}
template <typename TX, typename TIO, bool VEC, int MAXT>
cudaError_t backward_one(const BlockNormParams& p, int ctas, cudaStream_t stream) {
    const bool want_w = p.dweight || p.dbias || p.dpost_weight;
    const size_t smem = want_w ? 3 * (size_t)p.channels * sizeof(float) : 0;
    if (smem > 40000) {   // static and dynamic shared memory together past the default limit of 48 KB
        cudaError_t e = cudaFuncSetAttribute(block_norm_backward_kernel<TX, TIO, VEC, MAXT>,
                                             cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    block_norm_backward_kernel<TX, TIO, VEC, MAXT><<<ctas, threads_for(p.channels), smem, stream>>>(p);
    return cudaGetLastError();
}
template <typename TX, typename TIO, bool VEC>
cudaError_t backward_sized(const BlockNormParams& p, int ctas, cudaStream_t stream) {
    const int threads = threads_for(p.channels);
    if constexpr (!VEC) return backward_one<TX, TIO, VEC, 1024>(p, ctas, stream);
    if (threads <= 256) return backward_one<TX, TIO, VEC, 256>(p, ctas, stream);
    if (threads <= 640) return backward_one<TX, TIO, VEC, 640>(p, ctas, stream);
    return backward_one<TX, TIO, VEC, 1024>(p, ctas, stream);
}

}  // namespace

#define REGENVC_BY_TYPE(call)                                                                           \
    if (x_type == kTypeBf16) return vec ? call<__nv_bfloat16, __nv_bfloat16, true> : call<__nv_bfloat16, __nv_bfloat16, false>; \
    if (x_type == kTypeF16) return vec ? call<__half, __half, true> : call<__half, __half, false>;        \
    if (io_type == kTypeBf16) return vec ? call<float, __nv_bfloat16, true> : call<float, __nv_bfloat16, false>; \
    if (io_type == kTypeF16) return vec ? call<float, __half, true> : call<float, __half, false>;         \
    return vec ? call<float, float, true> : call<float, float, false>;

typedef cudaError_t (*NormLaunch)(const BlockNormParams&, int, cudaStream_t);
static NormLaunch pick_forward(int x_type, int io_type, bool vec) { REGENVC_BY_TYPE(forward_sized) }
static NormLaunch pick_backward(int x_type, int io_type, bool vec) { REGENVC_BY_TYPE(backward_sized) }

cudaError_t launch_block_norm_forward(BlockNormParams p, int x_type, int io_type, bool vec, int sm_count,
                                      cudaStream_t stream) {
    const int ctas = plan_rows(&p, 1280, sm_count);
    return pick_forward(x_type, io_type, vec)(p, ctas, stream);
}

cudaError_t launch_block_norm_backward(BlockNormParams p, int x_type, int io_type, bool vec, int sm_count, int* launches,
                                       cudaStream_t stream) {
    const int ctas = plan_rows(&p, 768, sm_count);
    *launches = 0;
    cudaError_t e = pick_backward(x_type, io_type, vec)(p, ctas, stream);
    if (e != cudaSuccess) return e;
    *launches = 1;
    const bool want_w = p.dweight || p.dbias || p.dpost_weight;
    const bool want_mod = p.dscale || p.dshift || p.dgate;
    const bool by_boundary = p.tokens_per_mod < p.rows_per_cta;
    const int n_mods = (int)(((long long)p.n_tokens + p.tokens_per_mod - 1) / p.tokens_per_mod);
    const int jobs = !want_mod || ctas == 1 ? 0 : (by_boundary ? ctas - 1 : n_mods);   // at most `ctas` either way
    if (jobs + (want_w ? 1 : 0) == 0) return cudaSuccess;
    block_norm_join_kernel<<<dim3((p.channels + 31) / 32, jobs + (want_w ? 1 : 0)), dim3(32, 32), 0, stream>>>(p, ctas, jobs,
                                                                                                          by_boundary ? 1 : 0);
    e = cudaGetLastError();
    if (e == cudaSuccess) *launches = 2;
    return e;
}

}  // namespace regenvc
