// Rotary embedding of queries and keys by explicit positions on several axes.
//
// Pair j of a head turns by position[axis(j)] * frequency(j); the pair is (2j, 2j + 1) or (j, j + n_pairs):
//     (a, b) -> (a cos - b sin, b cos + a sin),   the inverse (the gradient) with -sin.
// Angles: in whole turns, position * frequency / (2 pi) in 64 bits, its fraction taken there too (a position of 10^6 has
// lost four decimal digits of its angle in 32 bits), then sine and cosine of the fraction in 32 bits.
//
// Bound: HBM (every element is read and written once).  The angles of a token are shared by all heads of q and k, so a
// thread block computes them once per token into shared memory (a few 64-bit operations per pair against heads * 2
// elements) and then walks over its (token, head) vectors.  A thread keeps its place within a head; four vectors per
// thread are loaded before the first is used.  Measured: 31200 tokens x 80 heads x 128 bf16 207 us in a burst (6.2 TB/s of
// 6.45 measured), 215 to 219 us call after call, when the power cap takes the SM clock from 1965 to 1807 MHz (5.8 TB/s);
// 4097 x 48 heads x 128 fp16 in half pairs 22.6 us (4.5 TB/s, one round of blocks).
#include "rope_axes.cuh"
#include "row_io.cuh"

namespace regenvc {
namespace {

enum { kAdjacent = 0, kHalves = 1, kElements = 2 };
constexpr int kRopeThreads = 256;
constexpr int kBatch = 4;

// One thread's share of a head.  kAdjacent: eight neighbouring elements.  kHalves: eight of the first and the matching
// eight of the second half of the rotated part, or eight that are copied.  kElements: one pair, or one copied element.
// Place of pair j in a token's table.  A thread reads the pairs of its item as 16-byte words of two; word i of item c lies
// at i * items + c, so that neighbouring threads read neighbouring words (in the pairs' own order the reads of eight
// threads fell on two banks, and waiting for them was the kernel's largest stall).
template <int MODE>
__device__ __forceinline__ int table_place(int j, int n_pairs) {
    if constexpr (MODE == kAdjacent) return ((j >> 1 & 1) * ((n_pairs + 3) >> 2) + (j >> 2)) * 2 + (j & 1);
    if constexpr (MODE == kHalves) return ((j >> 1 & 3) * (n_pairs >> 3) + (j >> 3)) * 2 + (j & 1);
    return j;
}

template <typename T, int MODE>
struct Item;
template <typename T>
struct Item<T, kAdjacent> {
    Raw8<T> r;
    __device__ __forceinline__ void load(const T* head, int c, const RopeAxesParams&) { r = load_raw8(head + 8 * c); }
    __device__ __forceinline__ void store(T* head, int c, const float2* cs, const RopeAxesParams& p) const {
        float v[8];
        widen8(r, v);
        if (4 * c + 4 <= p.n_pairs) {
            const float4* q = reinterpret_cast<const float4*>(cs) + c;
            const int items = (p.n_pairs + 3) >> 2;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float4 t = q[i * items];
                const float a = v[4 * i], b = v[4 * i + 1], a2 = v[4 * i + 2], b2 = v[4 * i + 3];
                v[4 * i] = a * t.x - b * t.y;
                v[4 * i + 1] = b * t.x + a * t.y;
                v[4 * i + 2] = a2 * t.z - b2 * t.w;
                v[4 * i + 3] = b2 * t.z + a2 * t.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (4 * c + i < p.n_pairs) {
                    const float2 t = cs[table_place<kAdjacent>(4 * c + i, p.n_pairs)];
                    const float a = v[2 * i], b = v[2 * i + 1];
                    v[2 * i] = a * t.x - b * t.y;
                    v[2 * i + 1] = b * t.x + a * t.y;
                }
        }
        store8(head + 8 * c, v);
    }
};
template <typename T>
struct Item<T, kHalves> {
    Raw8<T> lo, hi;
    __device__ __forceinline__ void load(const T* head, int c, const RopeAxesParams& p) {
        if (8 * c < p.n_pairs) {
            lo = load_raw8(head + 8 * c);
            hi = load_raw8(head + p.n_pairs + 8 * c);
        } else {
            lo = load_raw8(head + p.n_pairs + 8 * c);   // item n_pairs / 8 is the first behind the rotated part
        }
    }
    __device__ __forceinline__ void store(T* head, int c, const float2* cs, const RopeAxesParams& p) const {
        float a[8], b[8];
        widen8(lo, a);
        if (8 * c < p.n_pairs) {
            widen8(hi, b);
            const float4* q = reinterpret_cast<const float4*>(cs) + c;
            const int items = p.n_pairs >> 3;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float4 t = q[i * items];
                const float x = a[2 * i], y = b[2 * i], x2 = a[2 * i + 1], y2 = b[2 * i + 1];
                a[2 * i] = x * t.x - y * t.y;
                b[2 * i] = y * t.x + x * t.y;
                a[2 * i + 1] = x2 * t.z - y2 * t.w;
                b[2 * i + 1] = y2 * t.z + x2 * t.w;
            }
            store8(head + 8 * c, a);
            store8(head + p.n_pairs + 8 * c, b);
        } else {
            store8(head + p.n_pairs + 8 * c, a);
        }
    }
};
template <typename T>
struct Item<T, kElements> {
    T a, b;
    static __device__ __forceinline__ int first(int c, const RopeAxesParams& p) {
        return c >= p.n_pairs ? p.n_pairs + c : (p.halves ? c : 2 * c);
    }
    static __device__ __forceinline__ int second(int c, const RopeAxesParams& p) { return p.halves ? c + p.n_pairs : 2 * c + 1; }
    __device__ __forceinline__ void load(const T* head, int c, const RopeAxesParams& p) {
        a = head[first(c, p)];
        if (c < p.n_pairs) b = head[second(c, p)];
    }
    __device__ __forceinline__ void store(T* head, int c, const float2* cs, const RopeAxesParams& p) const {
        if (c < p.n_pairs) {
            const float2 t = cs[c];
            const float x = to_f32(a), y = to_f32(b);
            from_f32(x * t.x - y * t.y, head[first(c, p)]);
            from_f32(y * t.x + x * t.y, head[second(c, p)]);
        } else {
            head[first(c, p)] = a;
        }
    }
};

template <typename T, int MODE>
__global__ void __launch_bounds__(kRopeThreads) rope_axes_kernel(const __grid_constant__ RopeAxesParams p, const int per_head) {
    extern __shared__ float4 table_raw[];
    float2* table = reinterpret_cast<float2*>(table_raw);   // [tokens_per_cta][n_pairs rounded up to 4] (cos, sin)
    const int pitch = (p.n_pairs + 3) & ~3;
    const int token0 = blockIdx.x * p.tokens_per_cta;
    const int tokens = min(p.tokens_per_cta, p.n_tokens - token0);
    const int lanes = blockDim.x / per_head;                // heads in hand at a time
    const int c = threadIdx.x % per_head, lane = threadIdx.x / per_head;
    const int all = p.heads[0] + p.heads[1];

    for (int i = threadIdx.x; i < tokens * p.n_pairs; i += blockDim.x) {
        const int t = i / p.n_pairs, j = i - t * p.n_pairs;
        int axis = 0;
        while (axis + 1 < p.n_axes && j >= p.axis_end[axis]) ++axis;
        const long long at = axis * p.pos_stride + token0 + t;
        const double pos = p.pos_float ? (double)reinterpret_cast<const float*>(p.positions)[at]
                                       : (double)reinterpret_cast<const int*>(p.positions)[at];
        const double turn = pos * p.turns[j];
        float s, k;
        sincospif(2.0f * (float)(turn - rint(turn)), &s, &k);
        table[t * pitch + table_place<MODE>(j, p.n_pairs)] = make_float2(k, p.inverse ? -s : s);
    }
    __syncthreads();
    if (lane >= lanes) return;

    int t = 0, h = lane;   // this thread's (token, head); the next one is `lanes` heads on
    while (h >= all) h -= all, ++t;
    while (t < tokens) {
        Item<T, MODE> item[kBatch];
        T* to[kBatch];
        const float2* cs[kBatch];
        int got = 0;
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            if (t < tokens) {
                const int w = h < p.heads[0] ? 0 : 1, hh = w ? h - p.heads[0] : h;
                const long long n = token0 + t;
                const T* from = reinterpret_cast<const T*>(p.in[w]) + n * p.in_token[w] + hh * p.in_head[w];
                to[i] = reinterpret_cast<T*>(p.out[w]) + n * p.out_token[w] + hh * p.out_head[w];
                cs[i] = table + t * pitch;
                item[i].load(from, c, p);
                got = i + 1;
                h += lanes;
                while (h >= all) h -= all, ++t;
            }
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
            if (i < got) item[i].store(to[i], c, cs[i], p);
    }
}

template <typename T, int MODE>
cudaError_t launch_mode(RopeAxesParams& p, int per_head, int sm_count, cudaStream_t stream) {
    const int all = p.heads[0] + p.heads[1];
    int lanes = kRopeThreads / per_head;
    const int pitch = (p.n_pairs + 3) & ~3;
    // tokens per thread block: enough vectors for about sixteen per thread; fewer where that would leave the device less
    // than one round of blocks
    int tokens = 16 * lanes / all;
    if (tokens > 16) tokens = 16;
    if (tokens > 1) {
        int per_sm = 1;
        const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, rope_axes_kernel<T, MODE>, kRopeThreads,
                                                                            (size_t)tokens * pitch * sizeof(float2));
        if (e != cudaSuccess) return e;
        const long long slots = (long long)(per_sm > 0 ? per_sm : 1) * sm_count, even = (p.n_tokens + slots - 1) / slots;
        if (tokens > even) tokens = (int)even;
    }
    if (tokens < 1) tokens = 1;
    if (lanes > all * tokens) lanes = all * tokens;
    p.tokens_per_cta = tokens;
    rope_axes_kernel<T, MODE><<<(unsigned)((p.n_tokens + tokens - 1) / tokens), lanes * per_head,
                                (size_t)tokens * pitch * sizeof(float2), stream>>>(p, per_head);
    return cudaGetLastError();
}
template <typename T>
cudaError_t launch_typed(RopeAxesParams& p, bool vec, int sm_count, cudaStream_t stream) {
    const int rest = p.head_dim - 2 * p.n_pairs;
    if (!vec || p.head_dim % 8 != 0 || (p.halves && p.n_pairs % 8 != 0))
        return launch_mode<T, kElements>(p, p.n_pairs + rest, sm_count, stream);
    if (p.halves) return launch_mode<T, kHalves>(p, (p.n_pairs + rest) / 8, sm_count, stream);
    return launch_mode<T, kAdjacent>(p, p.head_dim / 8, sm_count, stream);
}

}  // namespace

cudaError_t launch_rope_axes(RopeAxesParams p, int type, bool vec, int sm_count, cudaStream_t stream) {
    if (type == kTypeBf16) return launch_typed<__nv_bfloat16>(p, vec, sm_count, stream);
    if (type == kTypeF16) return launch_typed<__half>(p, vec, sm_count, stream);
    return launch_typed<float>(p, vec, sm_count, stream);
}

}  // namespace regenvc
