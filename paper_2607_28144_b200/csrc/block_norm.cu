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
// contiguous range of tokens and a thread sixteen fixed columns, for two reasons: the modulation, weight and bias values
// of a column stay in registers over all tokens that share them (read per token they would be 12 bytes of fp32 against
// 8 bytes of tokens), and the backward pass can sum over tokens in registers too, without atomics, in an order that
// depends on the shape alone.  Statistics take two passes over registers (mean, then centred squares) in fp32.
//
// What a row costs beside its bytes is instructions: with eight columns per thread and plain fp32 the forward kernel
// issued 299 per warp and row and kept the schedulers busy for two thirds of its 41 us (10920 x 1536 bf16, HBM at 0.27).
// Hence sixteen columns per thread, which halves the share of the sums' exchanges, arithmetic on pairs (f32x2), and
// asynchronous copies of the rows ahead into shared memory: every thread copies what it will read itself, so the ring
// needs neither barriers nor registers.
#include "block_norm.cuh"
#include "row_io.cuh"

namespace regenvc {
namespace {

constexpr int kCols = 16;            // columns per thread
constexpr int kPairs = kCols / 2;
typedef uint64_t f32x2;

__device__ __forceinline__ f32x2 both(float v) { return pack2(v, v); }
__device__ __forceinline__ float low(f32x2 v) {
    float a, b;
    unpack2(v, a, b);
    return a;
}
__device__ __forceinline__ float join(f32x2 v) {
    float a, b;
    unpack2(v, a, b);
    return a + b;
}

__device__ __forceinline__ void copy_async16(uint32_t smem, const void* global) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(global) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// Waits until at most `stages` - 1 of this thread's groups are under way.
__device__ __forceinline__ void copy_wait(int stages) {
    if (stages == 1) asm volatile("cp.async.wait_group 0;" ::: "memory");
    else if (stages == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else if (stages == 3) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else asm volatile("cp.async.wait_group 3;" ::: "memory");
}

// Where a thread's columns are.  VEC: two groups of eight neighbouring ones, `threads` groups apart (16-byte accesses of
// neighbouring threads are neighbours).  Otherwise, where sizes, strides or addresses do not allow that: sixteen columns
// `threads` apart.
template <bool VEC>
struct Place {
    int tid, threads;
    unsigned live;   // VEC: bit per group, else bit per column
    __device__ __forceinline__ explicit Place(int channels) : tid(threadIdx.x), threads(blockDim.x), live(0) {
        if constexpr (VEC) {
#pragma unroll
            for (int j = 0; j < 2; ++j) live |= (col(8 * j) < channels ? 1u : 0u) << j;
        } else {
#pragma unroll
            for (int i = 0; i < kCols; ++i) live |= (col(i) < channels ? 1u : 0u) << i;
        }
    }
    __device__ __forceinline__ int col(int i) const {
        return VEC ? ((i >> 3) * threads + tid) * 8 + (i & 7) : i * threads + tid;
    }
    __device__ __forceinline__ bool on(int i) const { return live >> (VEC ? i >> 3 : i) & 1; }
    // v in the live columns, 0 in the others
    __device__ __forceinline__ f32x2 masked(int pair, float v) const {
        if constexpr (VEC) return both(on(2 * pair) ? v : 0.0f);
        else return pack2(on(2 * pair) ? v : 0.0f, on(2 * pair + 1) ? v : 0.0f);
    }
};

// Bytes of one thread's columns of a row, and those of a row in the ring.
template <typename T>
constexpr uint32_t kMine = kCols * sizeof(T);

// One tensor's rows: through the ring (VEC) or straight from global memory.
template <typename T, bool VEC>
struct Rows {
    const T* base;
    long long stride;
    uint32_t ring;        // this thread's place in stage 0 (VEC); stages are `stage_bytes` apart
    __device__ __forceinline__ void fetch(const Place<VEC>& at, long long row, uint32_t stage) const {
        if constexpr (VEC) {
            const T* p = base + row * stride;
#pragma unroll
            for (int j = 0; j < 2; ++j)
                if (at.on(8 * j))
#pragma unroll
                    for (int k = 0; k < (int)sizeof(T) / 2; ++k)   // 16-byte pieces of eight elements
                        copy_async16(ring + stage + (j * (int)sizeof(T) / 2 + k) * at.threads * 16,
                                     p + at.col(8 * j) + k * (16 / (int)sizeof(T)));
        }
    }
    __device__ __forceinline__ void read(const Place<VEC>& at, long long row, uint32_t stage, f32x2* v) const {
        if constexpr (VEC) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                Raw8<T> r;
#pragma unroll
                for (int k = 0; k < (int)sizeof(T) / 2; ++k) {
                    const uint32_t a = ring + stage + (j * (int)sizeof(T) / 2 + k) * at.threads * 16;
                    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                                 : "=r"(r.w[k].x), "=r"(r.w[k].y), "=r"(r.w[k].z), "=r"(r.w[k].w) : "r"(a) : "memory");
                }
                float e[8];
                widen8(r, e);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[4 * j + i] = pack2(e[2 * i], e[2 * i + 1]);
            }
        } else {
            const T* p = base + row * stride;
            float e[kCols];
#pragma unroll
            for (int i = 0; i < kCols; ++i) e[i] = at.on(i) ? to_f32(p[at.col(i)]) : 0.0f;
#pragma unroll
            for (int i = 0; i < kPairs; ++i) v[i] = pack2(e[2 * i], e[2 * i + 1]);
        }
    }
};
template <typename T, bool VEC>
__device__ __forceinline__ void store_row(T* row, const Place<VEC>& at, const f32x2* v) {
    float e[kCols];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) unpack2(v[i], e[2 * i], e[2 * i + 1]);
    if constexpr (VEC) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
            if (at.on(8 * j)) store8(row + at.col(8 * j), e + 8 * j);
    } else {
#pragma unroll
        for (int i = 0; i < kCols; ++i)
            if (at.on(i)) from_f32(e[i], row[at.col(i)]);
    }
}
// A vector of parameters at this thread's columns; `absent` without one and in dead columns.
template <bool VEC>
__device__ __forceinline__ void read_vector(const float* base, float absent, const Place<VEC>& at, f32x2* v) {
#pragma unroll
    for (int i = 0; i < kPairs; ++i) v[i] = both(absent);
    if (base == nullptr) return;
    if constexpr (VEC) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
            if (at.on(8 * j))
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float4 q = __ldg(reinterpret_cast<const float4*>(base + at.col(8 * j)) + k);
                    v[4 * j + 2 * k] = pack2(q.x, q.y);
                    v[4 * j + 2 * k + 1] = pack2(q.z, q.w);
                }
    } else {
#pragma unroll
        for (int i = 0; i < kPairs; ++i)
            v[i] = pack2(at.on(2 * i) ? __ldg(base + at.col(2 * i)) : absent, at.on(2 * i + 1) ? __ldg(base + at.col(2 * i + 1)) : absent);
    }
}

// Sums over the thread block, the same value in every thread, in a fixed order.  Two buffers used in turn make one
// barrier per sum enough: a buffer is written again only behind the next sum's barrier.
struct BlockSum {
    float (*buf)[2][16];   // [2 buffers][2 values][warp]
    int warps, turn;
    template <int N>
    __device__ __forceinline__ void run(float* v) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
#pragma unroll
            for (int n = 0; n < N; ++n) v[n] += __shfl_xor_sync(0xffffffffu, v[n], o);
        if (warps == 1) return;
        float (*b)[16] = buf[turn];
        turn ^= 1;
        if ((threadIdx.x & 31) == 0)
#pragma unroll
            for (int n = 0; n < N; ++n) b[n][threadIdx.x >> 5] = v[n];
        __syncthreads();
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const float4 q = *reinterpret_cast<const float4*>(&b[n][0]);
            float s = (q.x + q.y) + (q.z + q.w);
            for (int w = 4; w < warps; w += 4) {
                const float4 r = *reinterpret_cast<const float4*>(&b[n][w]);
                s += (r.x + r.y) + (r.z + r.w);
            }
            v[n] = s;
        }
    }
};
__device__ __forceinline__ BlockSum block_sum_init(float (*buf)[2][16]) {
    for (int i = threadIdx.x; i < 64; i += blockDim.x) (&buf[0][0][0])[i] = 0.0f;   // entries past the last warp stay 0
    __syncthreads();
    return BlockSum{buf, (int)(blockDim.x + 31) / 32, 0};
}

// s / channels, rounded as a division is: the product with the reciprocal alone would leave a constant row a mean that is
// off by an ulp.
struct Channels {
    float n, inverse;
    __device__ __forceinline__ explicit Channels(int channels) : n((float)channels), inverse(1.0f / (float)channels) {}
    __device__ __forceinline__ float mean(float s) const {
        const float q = s * inverse;
        return fmaf(fmaf(-q, n, s), inverse, q);
    }
};

// v -> normalised v (dead columns hold and keep 0); returns the reciprocal deviation.
template <bool VEC>
__device__ __forceinline__ float normalise(f32x2* v, int kind, float eps, const Channels& ch, const Place<VEC>& at, BlockSum& sum) {
    float s[1];
    if (kind == kNormLayer) {
        f32x2 t = add2(v[0], v[1]), u = add2(v[2], v[3]);
#pragma unroll
        for (int i = 4; i < kPairs; i += 2) {
            t = add2(t, v[i]);
            u = add2(u, v[i + 1]);
        }
        s[0] = join(add2(t, u));
        sum.run<1>(s);
        const float mean = ch.mean(s[0]);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) v[i] = add2(v[i], at.masked(i, -mean));
    }
    f32x2 t = mul2(v[0], v[0]), u = mul2(v[1], v[1]);
#pragma unroll
    for (int i = 2; i < kPairs; i += 2) {
        t = fma2(v[i], v[i], t);
        u = fma2(v[i + 1], v[i + 1], u);
    }
    s[0] = join(add2(t, u));
    sum.run<1>(s);
    const float r = rsqrtf(ch.mean(s[0]) + eps);
    const f32x2 r2 = both(r);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) v[i] = mul2(v[i], r2);
    return r;
}

// Dead columns are never copied: their places in the ring hold 0 from the start.
__device__ __forceinline__ void clear_ring(uint4* ring, uint32_t bytes) {
    for (uint32_t i = threadIdx.x; i < bytes / 16; i += blockDim.x) ring[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
}

// The rows of up to four tensors copied ahead: `stages` rows' worth of shared memory in turn.  A stage is filled again one
// row after it was read, behind that row's barriers.
struct Ring {
    int stages;
    uint32_t bytes;      // of a stage
};

template <typename TX, typename TIO, bool VEC, int MAXT>
__global__ void __launch_bounds__(MAXT, MAXT == 512 ? 1 : 640 / MAXT) block_norm_forward_kernel(const BlockNormParams p, const Ring ring) {
    __shared__ alignas(16) float buf[2][2][16];
    extern __shared__ uint4 ring_mem[];
    BlockSum sum = block_sum_init(buf);
    const Place<VEC> at(p.channels);
    const Channels ch(p.channels);
    const int row0 = blockIdx.x * p.rows_per_cta;
    const int row1 = min(p.n_tokens, row0 + p.rows_per_cta);
    const bool residual = p.y != nullptr;
    if (VEC && p.channels < at.threads * kCols) clear_ring(ring_mem, ring.stages * ring.bytes);
    const uint32_t mine = smem_u32(ring_mem) + at.tid * 16;
    const Rows<TX, VEC> xs{reinterpret_cast<const TX*>(p.x), p.x_stride, mine};
    const Rows<TIO, VEC> ys{reinterpret_cast<const TIO*>(p.y), p.y_stride, mine + at.threads * kMine<TX>};
    auto fetch = [&](int row, int stage) {
        if constexpr (VEC) {
            if (row < row1) {
                xs.fetch(at, row, stage * ring.bytes);
                if (residual) ys.fetch(at, row, stage * ring.bytes);
            }
            copy_commit();
        }
    };
    for (int s = 0; s < ring.stages - 1; ++s) fetch(row0 + s, s);

    int mod_end = row0;   // first token behind the modulation row held in registers
    f32x2 w[kPairs], b[kPairs], g[kPairs];
    const f32x2 alpha = both(p.residual_scale);
    int stage = 0;
    for (int row = row0; row < row1; ++row) {
        if (row >= mod_end) {
            const int mod = row / p.tokens_per_mod;
            mod_end = p.tokens_per_mod < p.n_tokens - mod * p.tokens_per_mod ? (mod + 1) * p.tokens_per_mod : p.n_tokens;
            const long long from = mod * p.mod_stride;
            f32x2 t[kPairs];
            read_vector<VEC>(p.weight, 1.0f, at, w);
            read_vector<VEC>(p.bias, 0.0f, at, b);
            read_vector<VEC>(p.scale ? p.scale + from : nullptr, 0.0f, at, t);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) {
                w[i] = fma2(w[i], t[i], w[i]);
                b[i] = fma2(b[i], t[i], b[i]);
            }
            read_vector<VEC>(p.shift ? p.shift + from : nullptr, 0.0f, at, t);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) b[i] = add2(b[i], t[i]);
            read_vector<VEC>(p.gate ? p.gate + from : nullptr, 1.0f, at, g);
            read_vector<VEC>(p.post_weight, 1.0f, at, t);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) g[i] = mul2(g[i], t[i]);
        }
        fetch(row + ring.stages - 1, stage == 0 ? ring.stages - 1 : stage - 1);
        if constexpr (VEC) copy_wait(ring.stages);
        f32x2 v[kPairs];
        xs.read(at, row, stage * ring.bytes, v);
        if (residual) {
            f32x2 z[kPairs];
            ys.read(at, row, stage * ring.bytes, z);
            if (p.post_norm) normalise<VEC>(z, p.post_norm, p.post_eps, ch, at, sum);
            // (dead columns: z and x are 0, so x' is)
            if (p.residual_scale != 1.0f)
#pragma unroll
                for (int i = 0; i < kPairs; ++i) v[i] = mul2(v[i], alpha);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) v[i] = fma2(g[i], z[i], v[i]);
            if (p.x_out) store_row<TX, VEC>(reinterpret_cast<TX*>(p.x_out) + row * p.x_out_stride, at, v);
        }
        if (p.norm) {   // on x' before its rounding to the residual stream's type
            normalise<VEC>(v, p.norm, p.eps, ch, at, sum);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) v[i] = fma2(v[i], w[i], b[i]);
            store_row<TIO, VEC>(reinterpret_cast<TIO*>(p.h) + row * p.h_stride, at, v);
        }
        stage = stage + 1 == ring.stages ? 0 : stage + 1;
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
__global__ void __launch_bounds__(MAXT) block_norm_backward_kernel(const BlockNormParams p, const Ring ring) {
    __shared__ alignas(16) float buf[2][2][16];
    extern __shared__ uint4 ring_mem[];
    BlockSum sum = block_sum_init(buf);
    const Place<VEC> at(p.channels);
    const Channels ch(p.channels);
    const int row0 = blockIdx.x * p.rows_per_cta;
    const int row1 = min(p.n_tokens, row0 + p.rows_per_cta);
    const int first_mod = row0 / p.tokens_per_mod;
    const bool want_w = p.dweight || p.dbias || p.dpost_weight;
    const bool want_mod = p.dscale || p.dshift || p.dgate;
    const bool normed = p.norm != 0, branch = p.y != nullptr, more = p.dx_out != nullptr;
    if (VEC && p.channels < at.threads * kCols) clear_ring(ring_mem, ring.stages * ring.bytes);
    uint32_t mine = smem_u32(ring_mem) + at.tid * 16;
    const Rows<TX, VEC> xs{reinterpret_cast<const TX*>(p.x), p.x_stride, mine};
    const Rows<TIO, VEC> hs{reinterpret_cast<const TIO*>(p.dh), p.h_stride, mine += at.threads * kMine<TX>};
    const Rows<TX, VEC> ds{reinterpret_cast<const TX*>(p.dx_out), p.dx_out_stride, mine += at.threads * kMine<TIO>};
    const Rows<TIO, VEC> ys{reinterpret_cast<const TIO*>(p.y), p.y_stride, mine += at.threads * kMine<TX>};
    auto fetch = [&](int row, int stage) {
        if constexpr (VEC) {
            if (row < row1) {
                if (normed) {
                    xs.fetch(at, row, stage * ring.bytes);
                    hs.fetch(at, row, stage * ring.bytes);
                }
                if (more) ds.fetch(at, row, stage * ring.bytes);
                if (branch) ys.fetch(at, row, stage * ring.bytes);
            }
            copy_commit();
        }
    };
    for (int s = 0; s < ring.stages - 1; ++s) fetch(row0 + s, s);

    f32x2 s0[kPairs], s1[kPairs], s2[kPairs], w[kPairs], g[kPairs];
    const f32x2 alpha = both(p.residual_scale);
    int stage = 0;
    bool first_flush = true;
    for (int row = row0; row < row1;) {
        const int mod = row / p.tokens_per_mod;
        const int begin = mod * p.tokens_per_mod;
        const int whole_end = p.tokens_per_mod < p.n_tokens - begin ? begin + p.tokens_per_mod : p.n_tokens;
        const int end = min(row1, whole_end);
        const bool complete = row == begin && end == whole_end;
        const long long from = mod * p.mod_stride;
        {
            f32x2 t[kPairs];
            read_vector<VEC>(p.weight, 1.0f, at, w);
            read_vector<VEC>(p.scale ? p.scale + from : nullptr, 0.0f, at, t);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) w[i] = fma2(w[i], t[i], w[i]);
            read_vector<VEC>(p.gate ? p.gate + from : nullptr, 1.0f, at, g);
            read_vector<VEC>(p.post_weight, 1.0f, at, t);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) {
                g[i] = mul2(g[i], t[i]);
                s0[i] = s1[i] = s2[i] = 0ull;
            }
        }
        for (; row < end; ++row) {
            fetch(row + ring.stages - 1, stage == 0 ? ring.stages - 1 : stage - 1);
            if constexpr (VEC) copy_wait(ring.stages);
            const uint32_t here = stage * ring.bytes;
            f32x2 d[kPairs], v[kPairs];
            if (normed) {
                xs.read(at, row, here, v);
                const float r = normalise<VEC>(v, p.norm, p.eps, ch, at, sum);
                hs.read(at, row, here, d);
                f32x2 ta = 0ull, tb = 0ull;
#pragma unroll
                for (int i = 0; i < kPairs; ++i) {
                    s0[i] = add2(s0[i], d[i]);
                    s1[i] = fma2(d[i], v[i], s1[i]);
                    d[i] = mul2(d[i], w[i]);
                    ta = add2(ta, d[i]);
                    tb = fma2(d[i], v[i], tb);
                }
                float t[2] = {join(ta), join(tb)};
                sum.run<2>(t);
                // r (d - m0 - xhat m1)
                const f32x2 m0 = both(p.norm == kNormLayer ? -r * ch.mean(t[0]) : 0.0f), m1 = both(-r * ch.mean(t[1])), r2 = both(r);
#pragma unroll
                for (int i = 0; i < kPairs; ++i) d[i] = fma2(v[i], m1, fma2(d[i], r2, m0));
            } else {
#pragma unroll
                for (int i = 0; i < kPairs; ++i) d[i] = 0ull;
            }
            if (more) {
                ds.read(at, row, here, v);
#pragma unroll
                for (int i = 0; i < kPairs; ++i) d[i] = add2(d[i], v[i]);
            }
            if (p.dx) {
                if (p.residual_scale != 1.0f) {
#pragma unroll
                    for (int i = 0; i < kPairs; ++i) v[i] = mul2(d[i], alpha);
                    store_row<TX, VEC>(reinterpret_cast<TX*>(p.dx) + row * p.dx_stride, at, v);
                } else {
                    store_row<TX, VEC>(reinterpret_cast<TX*>(p.dx) + row * p.dx_stride, at, d);
                }
            }
            if (branch) {
                ys.read(at, row, here, v);
                float r = 1.0f;
                if (p.post_norm) r = normalise<VEC>(v, p.post_norm, p.post_eps, ch, at, sum);
                f32x2 ta = 0ull, tb = 0ull;
#pragma unroll
                for (int i = 0; i < kPairs; ++i) {
                    s2[i] = fma2(d[i], v[i], s2[i]);
                    d[i] = mul2(d[i], g[i]);
                }
                if (p.post_norm) {
#pragma unroll
                    for (int i = 0; i < kPairs; ++i) {
                        // (dead columns of d hold -m0 r: their terms stay out of the mean)
                        ta = add2(ta, VEC || (at.on(2 * i) && at.on(2 * i + 1)) ? (at.on(2 * i) ? d[i] : 0ull)
                                                                               : (at.on(2 * i) ? pack2(low(d[i]), 0.0f) : 0ull));
                        tb = fma2(d[i], v[i], tb);   // v is 0 there
                    }
                    float t[2] = {join(ta), join(tb)};
                    sum.run<2>(t);
                    const f32x2 m0 = both(p.post_norm == kNormLayer ? -r * ch.mean(t[0]) : 0.0f), m1 = both(-r * ch.mean(t[1])), r2 = both(r);
#pragma unroll
                    for (int i = 0; i < kPairs; ++i) d[i] = fma2(v[i], m1, fma2(d[i], r2, m0));
                }
                if (p.dy) store_row<TIO, VEC>(reinterpret_cast<TIO*>(p.dy) + row * p.dy_stride, at, d);
            }
            stage = stage + 1 == ring.stages ? 0 : stage + 1;
        }
        // the modulation row's sums: final where all of its tokens are this block's, else a slot of the workspace
        if (want_w || want_mod) {
            float* slot = slot_of(p, blockIdx.x, mod == first_mod ? 0 : 1);
            float* wslot = slot_of(p, blockIdx.x, 2);
            float e0[kCols], e1[kCols], e2[kCols];
#pragma unroll
            for (int i = 0; i < kPairs; ++i) {
                unpack2(s0[i], e0[2 * i], e0[2 * i + 1]);
                unpack2(s1[i], e1[2 * i], e1[2 * i + 1]);
                unpack2(s2[i], e2[2 * i], e2[2 * i + 1]);
            }
#pragma unroll
            for (int i = 0; i < kCols; ++i) {
                if (!at.on(i)) continue;
                const int c = at.col(i);
                if (want_w) {   // this thread's own columns of this block's own slot
                    const float s = p.scale ? 1.0f + p.scale[from + c] : 1.0f;
                    const float gate = p.gate ? p.gate[from + c] : 1.0f;
                    wslot[c] = fmaf(s, e1[i], first_flush ? 0.0f : wslot[c]);
                    wslot[p.channels + c] = fmaf(s, e0[i], first_flush ? 0.0f : wslot[p.channels + c]);
                    wslot[2 * p.channels + c] = fmaf(gate, e2[i], first_flush ? 0.0f : wslot[2 * p.channels + c]);
                }
                if (!want_mod) continue;
                if (complete) {
                    write_mod_grads(p, mod, c, e0[i], e1[i], e2[i]);
                } else {
                    slot[c] = e0[i];
                    slot[p.channels + c] = e1[i];
                    slot[2 * p.channels + c] = e2[i];
                }
            }
            first_flush = false;
        }
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

int threads_for(int channels) { return (channels + 32 * kCols - 1) / (32 * kCols) * 32; }

// A persistent grid: as many thread blocks as the device holds at a time (more would run as a second, mostly empty wave:
// 41 us instead of 33 at the window), each with an equal share of the rows; at most `cap`.
template <typename K>
cudaError_t plan(BlockNormParams* p, K kernel, int threads, size_t smem, int sm_count, int cap, int* ctas) {
    if (smem > 40000) {   // static and dynamic shared memory together past the default limit of 48 KB
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    int most = p->n_tokens;
    if (most > sm_count) {
        int per_sm = 1;
        const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, smem);
        if (e != cudaSuccess) return e;
        if (per_sm < 1) per_sm = 1;
        if (most > per_sm * sm_count) most = per_sm * sm_count;
        if (most > cap) most = cap;
    }
    p->rows_per_cta = (p->n_tokens + most - 1) / most;
    *ctas = (p->n_tokens + p->rows_per_cta - 1) / p->rows_per_cta;
    return cudaSuccess;
}

// Stages: as many as fit a share of the SM's shared memory (for about `threads_wanted` threads on it), two to four; one
// where two rows do not fit an SM (fp32 gradients of more than 7000 channels).
Ring plan_ring(bool vec, uint32_t stage_bytes, int threads, int threads_wanted) {
    if (!vec) return Ring{1, 0};
    const int blocks = threads_wanted / threads > 1 ? threads_wanted / threads : 1;
    int stages = (int)(200000u / blocks / stage_bytes);
    if (stages < 2) stages = 2 * stage_bytes <= 225000u ? 2 : 1;
    if (stages > 4) stages = 4;
    return Ring{stages, stage_bytes};
}

template <typename TX, typename TIO, bool VEC, int MAXT>
cudaError_t forward_one(BlockNormParams& p, int sm_count, int* ctas, cudaStream_t stream) {
    const int threads = threads_for(p.channels);
    const Ring ring = plan_ring(VEC, threads * (kMine<TX> + (p.y ? kMine<TIO> : 0)), threads, 640);
    const size_t smem = (size_t)ring.stages * ring.bytes;
    const cudaError_t e = plan(&p, block_norm_forward_kernel<TX, TIO, VEC, MAXT>, threads, smem, sm_count, 1 << 30, ctas);
    if (e != cudaSuccess) return e;
    block_norm_forward_kernel<TX, TIO, VEC, MAXT><<<*ctas, threads, smem, stream>>>(p, ring);
    return cudaGetLastError();
}
template <typename TX, typename TIO, bool VEC, int MAXT>
cudaError_t backward_one(BlockNormParams& p, int sm_count, int* ctas, cudaStream_t stream) {
    const int threads = threads_for(p.channels);
    // (all four tensors have their place, wanted or not)
    const Ring ring = plan_ring(VEC, threads * 2 * (kMine<TX> + kMine<TIO>), threads, 384);
    const size_t smem = (size_t)ring.stages * ring.bytes;
    const cudaError_t e = plan(&p, block_norm_backward_kernel<TX, TIO, VEC, MAXT>, threads, smem, sm_count, kNormMaxCtas, ctas);
    if (e != cudaSuccess) return e;
    block_norm_backward_kernel<TX, TIO, VEC, MAXT><<<*ctas, threads, smem, stream>>>(p, ring);
    return cudaGetLastError();
}
// Builds by the registers that a row's threads leave: up to 2048 channels (forward only), 5120, 8192.
template <typename TX, typename TIO, bool VEC>
cudaError_t forward_sized(BlockNormParams& p, int sm_count, int* ctas, cudaStream_t stream) {
    if (threads_for(p.channels) <= 128) return forward_one<TX, TIO, VEC, 128>(p, sm_count, ctas, stream);
    if (threads_for(p.channels) <= 320) return forward_one<TX, TIO, VEC, 320>(p, sm_count, ctas, stream);
    return forward_one<TX, TIO, VEC, 512>(p, sm_count, ctas, stream);
}
template <typename TX, typename TIO, bool VEC>
cudaError_t backward_sized(BlockNormParams& p, int sm_count, int* ctas, cudaStream_t stream) {
    if (threads_for(p.channels) <= 320) return backward_one<TX, TIO, VEC, 320>(p, sm_count, ctas, stream);
    return backward_one<TX, TIO, VEC, 512>(p, sm_count, ctas, stream);
}

}  // namespace

#define REGENVC_BY_TYPE(call)                                                                           \
    if (x_type == kTypeBf16) return vec ? call<__nv_bfloat16, __nv_bfloat16, true> : call<__nv_bfloat16, __nv_bfloat16, false>; \
    if (x_type == kTypeF16) return vec ? call<__half, __half, true> : call<__half, __half, false>;        \
    if (io_type == kTypeBf16) return vec ? call<float, __nv_bfloat16, true> : call<float, __nv_bfloat16, false>; \
    if (io_type == kTypeF16) return vec ? call<float, __half, true> : call<float, __half, false>;         \
    return vec ? call<float, float, true> : call<float, float, false>;

typedef cudaError_t (*NormLaunch)(BlockNormParams&, int, int*, cudaStream_t);
static NormLaunch pick_forward(int x_type, int io_type, bool vec) { REGENVC_BY_TYPE(forward_sized) }
static NormLaunch pick_backward(int x_type, int io_type, bool vec) { REGENVC_BY_TYPE(backward_sized) }

cudaError_t launch_block_norm_forward(BlockNormParams p, int x_type, int io_type, bool vec, int sm_count,
                                      cudaStream_t stream) {
    int ctas = 0;
    return pick_forward(x_type, io_type, vec)(p, sm_count, &ctas, stream);
}

cudaError_t launch_block_norm_backward(BlockNormParams p, int x_type, int io_type, bool vec, int sm_count, int* launches,
                                       cudaStream_t stream) {
    int ctas = 0;
    *launches = 0;
    cudaError_t e = pick_backward(x_type, io_type, vec)(p, sm_count, &ctas, stream);
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
