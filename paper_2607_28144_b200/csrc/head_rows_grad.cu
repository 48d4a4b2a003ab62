// Gradients of the norm and rotation of queries and keys, from the operands themselves: nothing is kept between the passes.
//
//     x the operand, n = x r, r = 1 / sqrt(mean(x^2) + eps), y = R (n w)
//     g = R^T dy,   dw = sum over tokens and heads of g n,   dx = r (g w - n mean(g w n))
//
// Bound: HBM, x and dy are read once and dx is written once.  Both sums over a head, of x^2 and of g w x, run side by side.
// 128 registers hold two vectors of operands, their products and the sums of both gains, so two blocks fill an SM (three spill:
// 59 us instead of 44); what a block keeps in flight is then one vector a group, which is what bounds it.  Loads and stores are
// marked as touched once (50 instead of 51 us, fp32 60 instead of 62 before the walk over one token's heads).
// Measured, 10920 tokens, 12 + 12 heads of 128: bf16 44.3 us, 4.5 TB/s; fp32, 4097 tokens, 40 + 8 heads, 61.5 us, 4.9 TB/s (whose
// build spills 48 to 76 bytes at 128 registers).
// The sums of dw have a fixed order: a thread adds up what its own vectors give, a block joins its threads, a second kernel
// joins the blocks, each over the same vectors in every call of a shape; no atomics.
#include "head_rows_core.cuh"

namespace regenvc {
namespace {

template <typename T>
struct Vector {
    const T *x, *dy;
    T* dx;
};
template <typename T>
__device__ __forceinline__ Vector<T> locate(const HeadRowsParams& p, int token, int h, int& w) {
    w = h < p.heads[0] ? 0 : 1;
    const long long n = token, hh = w ? h - p.heads[0] : h;
    return {reinterpret_cast<const T*>(p.in[w]) + n * p.in_token[w] + hh * p.in_head[w],
            reinterpret_cast<const T*>(p.grad[w]) + n * p.grad_token[w] + hh * p.grad_head[w],
            reinterpret_cast<T*>(p.out[w]) + n * p.out_token[w] + hh * p.out_head[w]};
}

template <typename T, bool HALVES, bool SOME>   // SOME: adjacent pairs of which the head's last do not turn
__global__ void __launch_bounds__(kHeadThreads, 2) head_rows_grad_kernel(const __grid_constant__ HeadRowsParams p, const int width) {
    extern __shared__ float4 shared_raw[];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // the join sets itself up and waits for this grid
    const int pitch = table_pitch(p), units = p.head_dim / 16, turning = table_units<HALVES ? kHalfUnits : kAdjacentUnits>(p);
    float2* table = reinterpret_cast<float2*>(shared_raw);
    float* gains = reinterpret_cast<float*>(table + p.tokens_per_cta * pitch);
    // a group of lanes has one token of those at hand, and every so many of its vectors
    const int u = threadIdx.x & (width - 1), group = threadIdx.x / width, step = blockDim.x / width / p.tokens_per_cta;
    const int t = group / step, all = p.heads[0] + p.heads[1], rounds = (all + step - 1) / step;
    const bool active = u < units;
    const Pieces at = pieces_of<HALVES>(p, active ? u : 0);
    const float inv_d = 1.0f / (float)p.head_dim;
    const bool sums = p.partial != nullptr;
    const int lo_bytes = at.lo * (int)sizeof(T), hi_from_lo = at.hi - at.lo;
    const ulonglong2* words = reinterpret_cast<const ulonglong2*>(table + t * pitch) + u;
    const ulonglong2* gain_words = reinterpret_cast<const ulonglong2*>(gains) + u;
    Unit dw[2] = {};

    struct Item {
        Raw8<T> xl, xh, yl, yh;
        T* to;                                              // nullptr: nothing to do
        int of;                                             // 0 q, 1 k
    };
    for (long long token0 = (long long)blockIdx.x * p.tokens_per_cta; token0 < p.n_tokens; token0 += (long long)gridDim.x * p.tokens_per_cta) {
        const int tokens = (int)min((long long)p.tokens_per_cta, p.n_tokens - token0);
        int h = group - t * step;                           // this group's next vector
        auto fetch = [&](Item& x) {
            x.to = nullptr;
            x.of = h >= p.heads[0];
            if (active && t < tokens && h < all) {
                const int token = (int)token0 + t, head = x.of ? h - p.heads[0] : h;
                const HeadRowsView& o = p.view[x.of];
                const T* v = reinterpret_cast<const T*>(o.from + (long long)token * o.from_token + (long long)head * o.from_head + lo_bytes);
                const T* dy = reinterpret_cast<const T*>(o.dy + (long long)token * o.dy_token + (long long)head * o.dy_head + lo_bytes);
                x.to = reinterpret_cast<T*>(o.to + (long long)token * o.to_token + (long long)head * o.to_head + lo_bytes);
                x.xl = load_raw8_once(v);
                x.xh = load_raw8_once(v + hi_from_lo);
                x.yl = load_raw8_once(dy);
                x.yh = load_raw8_once(dy + hi_from_lo);
            } else {
                x.xl = x.xh = x.yl = x.yh = Raw8<T>{};
            }
            h += step;
        };
        Item next;
        fetch(next);                                        // on its way while the angles are formed
        __syncthreads();                                    // the last tokens' table has been read
        if (p.n_axes) fill_table<HALVES ? kHalfUnits : kAdjacentUnits>(p, table, pitch, (int)token0, tokens, true);
        if (token0 == (long long)blockIdx.x * p.tokens_per_cta) fill_gains<HALVES>(p, gains);
        __syncthreads();
        for (int round = 0; round < rounds; ++round) {      // the same rounds for all lanes
            const Item x = next;
            if (round + 1 < rounds) fetch(next);
            Unit v = widen<HALVES>(x.xl, x.xh), g = widen<HALVES>(x.yl, x.yh);
            if (SOME && x.to) turn_some(g, load_angles(words, turning), p.n_pairs - 4 * u, p.head_dim / 4);
            else if (at.turns && x.to) turn(g, load_angles(words, turning));
            Unit w = load_gains<HALVES>(gain_words + (active ? x.of * 4 * units : -u), units);
            uint64_t sq2 = 0, hx2 = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                w.a[e] = mul2(w.a[e], g.a[e]);
                w.b[e] = mul2(w.b[e], g.b[e]);
                sq2 = fma2(v.b[e], v.b[e], fma2(v.a[e], v.a[e], sq2));
                hx2 = fma2(w.b[e], v.b[e], fma2(w.a[e], v.a[e], hx2));
            }
            const float sq = head_sum(sum2(sq2), width), hx = head_sum(sum2(hx2), width);
            const float r = rsqrtf(sq * inv_d + p.eps);
            // mean(g w n); of a row past fp32's range n is 0, whatever the sum of g w x came to
            const float m = r == 0.0f ? 0.0f : hx * inv_d * r;
            if (x.to) {
                const uint64_t r2 = pack2(r, r), m2 = pack2(-m, -m);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v.a[e] = mul2(v.a[e], r2), v.b[e] = mul2(v.b[e], r2);   // n
                    w.a[e] = mul2(r2, fma2(v.a[e], m2, w.a[e]));
                    w.b[e] = mul2(r2, fma2(v.b[e], m2, w.b[e]));
                }
                float lo[8], hi[8];
                spread<HALVES>(w, lo, hi);
                store8_once(x.to, lo);
                store8_once(x.to + hi_from_lo, hi);
                if (sums) {
                    if (x.of == 0) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) dw[0].a[e] = fma2(g.a[e], v.a[e], dw[0].a[e]), dw[0].b[e] = fma2(g.b[e], v.b[e], dw[0].b[e]);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) dw[1].a[e] = fma2(g.a[e], v.a[e], dw[1].a[e]), dw[1].b[e] = fma2(g.b[e], v.b[e], dw[1].b[e]);
                    }
                }
            }
        }
    }
    if (!sums) return;
    // the block's sums: lanes of one warp that hold the same unit by shuffles, warps in turn through shared memory
    __shared__ float part[kHeadThreads / 32][2][kRopeMaxPairs * 2];
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int two = e >> 2, k = e >> 1 & 1, second = e & 1;
            float f[2];
            unpack2(second ? dw[w].b[two] : dw[w].a[two], f[0], f[1]);
            float s = f[k];
            s += __shfl_xor_sync(0xffffffffu, s, 16);
            if (width <= 8) s += __shfl_xor_sync(0xffffffffu, s, 8);
            if (width <= 4) s += __shfl_xor_sync(0xffffffffu, s, 4);
            if ((threadIdx.x & 31) < width && active) part[threadIdx.x >> 5][w][offset_of<HALVES>(at, two, k, second)] = s;
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * p.head_dim; i += blockDim.x) {
        const int w = i >= p.head_dim, col = w ? i - p.head_dim : i;
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < kHeadThreads / 32; ++j) s += part[j][w][col];
        p.partial[(size_t)blockIdx.x * 2 * p.head_dim + i] = s;
    }
}

// Element form: a warp holds a head, as in the forward pass.
template <typename T>
__global__ void __launch_bounds__(kHeadThreads) head_rows_grad_element_kernel(const __grid_constant__ HeadRowsParams p) {
    extern __shared__ float4 table_raw[];
    float2* table = reinterpret_cast<float2*>(table_raw);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int pitch = table_pitch(p), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int all = p.heads[0] + p.heads[1], units = p.head_dim - p.n_pairs;
    float da[2][kUnits], db[2][kUnits];
#pragma unroll
    for (int k = 0; k < kUnits; ++k) da[0][k] = da[1][k] = db[0][k] = db[1][k] = 0.0f;
    for (long long token0 = (long long)blockIdx.x * p.tokens_per_cta; token0 < p.n_tokens; token0 += (long long)gridDim.x * p.tokens_per_cta) {
        const int tokens = (int)min((long long)p.tokens_per_cta, p.n_tokens - token0);
        if (p.n_axes) {
            __syncthreads();
            fill_table<kPlain>(p, table, pitch, (int)token0, tokens, true);
            __syncthreads();
        }
        for (int i = warp; i < tokens * all; i += blockDim.x >> 5) {
            const int t = i / all;
            int w;
            const Vector<T> at = locate<T>(p, (int)token0 + t, i - t * all, w);
            const float* gain = p.weight[w];
            float xa[kUnits], xb[kUnits], ga[kUnits], gb[kUnits], sq = 0.0f, hx = 0.0f;
#pragma unroll
            for (int k = 0; k < kUnits; ++k) {
                const int u = lane + 32 * k;
                xa[k] = xb[k] = ga[k] = gb[k] = 0.0f;
                if (u >= units) continue;
                const int first = unit_first(u, p);
                xa[k] = to_f32(at.x[first]);
                ga[k] = to_f32(at.dy[first]);
                sq += xa[k] * xa[k];
                if (u < p.n_pairs) {
                    const int second = unit_second(u, p);
                    xb[k] = to_f32(at.x[second]);
                    const float d = to_f32(at.dy[second]);
                    const float2 cs = table[t * pitch + u];
                    gb[k] = d * cs.x + ga[k] * cs.y;
                    ga[k] = ga[k] * cs.x - d * cs.y;
                    sq += xb[k] * xb[k];
                    hx += gb[k] * (gain ? gain[second] : 1.0f) * xb[k];
                }
                hx += ga[k] * (gain ? gain[first] : 1.0f) * xa[k];
            }
            sq = warp_sum(sq) / (float)p.head_dim;
            hx = warp_sum(hx) / (float)p.head_dim;
            const float r = rsqrtf(sq + p.eps);
            const float m = r == 0.0f ? 0.0f : hx * r * r;  // mean(g w n) r, as above
#pragma unroll
            for (int k = 0; k < kUnits; ++k) {
                const int u = lane + 32 * k;
                if (u >= units) continue;
                const int first = unit_first(u, p);
                from_f32(r * (ga[k] * (gain ? gain[first] : 1.0f) - xa[k] * m), at.dx[first]);
                const float sa = ga[k] * (xa[k] * r), sb = gb[k] * (xb[k] * r);
                if (w) da[1][k] += sa, db[1][k] += sb;
                else da[0][k] += sa, db[0][k] += sb;
                if (u < p.n_pairs) {
                    const int second = unit_second(u, p);
                    from_f32(r * (gb[k] * (gain ? gain[second] : 1.0f) - xb[k] * m), at.dx[second]);
                }
            }
        }
    }
    if (!p.partial) return;
    __shared__ float part[kHeadThreads / 32][2][kRopeMaxPairs * 2];
#pragma unroll
    for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            const int u = lane + 32 * k;
            if (u >= units) continue;
            part[warp][w][unit_first(u, p)] = da[w][k];
            if (u < p.n_pairs) part[warp][w][unit_second(u, p)] = db[w][k];
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * p.head_dim; i += blockDim.x) {
        const int w = i >= p.head_dim, col = w ? i - p.head_dim : i;
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < kHeadThreads / 32; ++j) s += part[j][w][col];
        p.partial[(size_t)blockIdx.x * 2 * p.head_dim + i] = s;
    }
}

// Sums of the blocks' partial sums: eight columns per block, 32 threads to a column.
__global__ void __launch_bounds__(256) head_rows_join_kernel(const float* partial, int blocks, int head_dim, float* dq, float* dk) {
    __shared__ float part[32][8];
    const int col = blockIdx.x * 8 + (threadIdx.x & 7), row = threadIdx.x >> 3;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    float s = 0.0f;
    if (col < 2 * head_dim)
#pragma unroll 4
        for (int i = row; i < blocks; i += 32) s += partial[(size_t)i * 2 * head_dim + col];
    part[row][threadIdx.x & 7] = s;
    __syncthreads();
    if (threadIdx.x < 8 && col < 2 * head_dim) {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 32; ++i) sum += part[i][threadIdx.x];
        float* to = col < head_dim ? dq : dk;
        if (to) to[col < head_dim ? col : col - head_dim] = sum;
    }
}

template <typename T>
cudaError_t launch_typed(HeadRowsParams& p, bool vec, int sm_count, int* blocks, cudaStream_t stream) {
    const int all = p.heads[0] + p.heads[1];
    const bool unit = in_units(p, vec, sizeof(T));
    const int width = unit ? lanes_of_head(p) : 32;
    auto kernel = p.halves        ? head_rows_grad_kernel<T, true, false>
                  : turns_some(p) ? head_rows_grad_kernel<T, false, true>
                                  : head_rows_grad_kernel<T, false, false>;
    const size_t per_token = (size_t)table_pitch(p) * sizeof(float2), gains = 2 * (size_t)p.head_dim * sizeof(float);
    int per_sm = 1;
    const cudaError_t e = unit ? cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, kHeadThreads, kHeadTokens * per_token + gains)
                               : cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, head_rows_grad_element_kernel<T>, kHeadThreads, kHeadTokens * per_token + gains);
    if (e != cudaSuccess) return e;
    long long places = (long long)(per_sm > 0 ? per_sm : 1) * sm_count;
    if (places > kHeadGradMaxBlocks) places = kHeadGradMaxBlocks;
    p.tokens_per_cta = tokens_of_block(p.n_tokens, all, kHeadThreads / width, 8, places);
    const long long batches = ((long long)p.n_tokens + p.tokens_per_cta - 1) / p.tokens_per_cta;
    *blocks = (int)(batches < places ? batches : places);
    const size_t smem = p.tokens_per_cta * per_token + gains;
    if (unit) kernel<<<*blocks, kHeadThreads, smem, stream>>>(p, width);
    else head_rows_grad_element_kernel<T><<<*blocks, kHeadThreads, smem, stream>>>(p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_head_rows_grad(HeadRowsParams p, int type, bool vec, int sm_count, int* launches, cudaStream_t stream) {
    int blocks = 0;
    *launches = 0;
    cudaError_t e = type == kTypeBf16  ? launch_typed<__nv_bfloat16>(p, vec, sm_count, &blocks, stream)
                    : type == kTypeF16 ? launch_typed<__half>(p, vec, sm_count, &blocks, stream)
                                       : launch_typed<float>(p, vec, sm_count, &blocks, stream);
    if (e != cudaSuccess) return e;
    *launches = 1;
    if (!p.partial) return cudaSuccess;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((2 * p.head_dim + 7) / 8));
    cfg.blockDim = dim3(256);
    cfg.stream = stream;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, head_rows_join_kernel, (const float*)p.partial, blocks, p.head_dim, p.dweight[0], p.dweight[1]);
    if (e == cudaSuccess) *launches = 2;
    return e;
}

}  // namespace regenvc
