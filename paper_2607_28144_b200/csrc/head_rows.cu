// Queries and keys of every head normalised and rotated in one pass, into rows or, with the values, into a paged cache.
//
//     y = R(position) (x / sqrt(mean(x^2) + eps) * w)      over the elements of one head; values are copied
//
// R turns pair j by position[axis(j)] * frequency(j).  The normalised values never round to the rows' type in between.
// Bound: HBM, every element is read and written once (two passes, a norm and a rotation, move twice that).  The angles of
// a token are shared by all its heads, so a thread block computes them once per token into shared memory and then walks
// over its (token, head) vectors, four to eight pieces of 16 bytes per thread in flight.
// Paged: token n of the call belongs to the sequence whose rows it lies in, found by counting the row starts at or before
// it (a warp per token, all loads independent: a binary search is a chain of loads, which is what a call of a few tokens
// would wait for); its slot is the sequence's length minus the rows behind it, its page comes from the table.
#include "common.cuh"
#include "head_rows_core.cuh"

namespace regenvc {
namespace {

constexpr int kBatch = 1;
constexpr int kMaxTokens = 16;      // per thread block

// Offsets of a token's slot in the two caches; -1: the token goes nowhere (behind the last sequence, a page that is not
// there).
struct Slots {
    long long k[kMaxTokens], v[kMaxTokens];
    int rows[kMaxTokens];           // 1: the row belongs to a sequence
};

__device__ __forceinline__ void find_slots(const HeadRowsParams& p, Slots& s, int token0, int tokens) {
    const int lane = threadIdx.x & 31;
    for (int t = threadIdx.x >> 5; t < tokens; t += blockDim.x >> 5) {
        const int n = token0 + t;
        int before = 0;
#pragma unroll 4
        for (int i = lane; i <= p.n_sequences; i += 32) before += p.row_starts[i] <= n;
        before = __reduce_add_sync(0xffffffffu, before);
        if (lane == 0) {
            const int seq = before - 1;
            long long k = -1, v = -1;
            const bool row = seq >= 0 && seq < p.n_sequences;
            if (row) {
                const long long at = (long long)p.lengths[seq] - (p.row_starts[seq + 1] - n);
                bool good = at >= 0 && at < (long long)p.pages_per_sequence * p.page_size;
                if (good) {
                    const int slot = (int)(at / p.page_size), in_page = (int)(at - (long long)slot * p.page_size);
                    const int page = p.table[seq * p.table_stride + slot];
                    good = page >= 0 && page < p.n_pages;
                    if (good) {
                        k = page * p.page_stride[0] + in_page * p.out_token[1];
                        v = page * p.page_stride[1] + in_page * p.out_token[2];
                    }
                }
                if (!good) atomicCAS(p.status, 0, kStatusRange);
            }
            s.k[t] = k;
            s.v[t] = v;
            s.rows[t] = row;
        }
    }
}

// Where vector (t, h) comes from and goes to; w: 0 q, 1 k, 2 v.
template <typename T>
__device__ __forceinline__ bool locate(const HeadRowsParams& p, const Slots& s, int token0, int t, int h, int& w, const T*& from, T*& to) {
    w = 0;
    if (h >= p.heads[0]) {
        h -= p.heads[0];
        w = 1;
        if (h >= p.heads[1]) {
            h -= p.heads[1];
            w = 2;
        }
    }
    const long long n = token0 + t;
    from = reinterpret_cast<const T*>(p.in[w]) + n * p.in_token[w] + h * p.in_head[w];
    long long base = n * p.out_token[w];
    if (p.paged) {
        if (!s.rows[t]) return false;
        if (w) base = w == 1 ? s.k[t] : s.v[t];
        if (base < 0) return false;
    }
    to = reinterpret_cast<T*>(p.out[w]) + base + h * p.out_head[w];
    return true;
}

template <typename T, bool HALVES>
__global__ void __launch_bounds__(kHeadThreads, 4) head_rows_kernel(const __grid_constant__ HeadRowsParams p, const int width) {
    extern __shared__ float4 shared_raw[];
    __shared__ Slots slots;
    const int pitch = table_pitch(p), units = table_units<HALVES ? kHalfUnits : kAdjacentUnits>(p);
    float2* table = reinterpret_cast<float2*>(shared_raw);
    float* gains = reinterpret_cast<float*>(table + p.tokens_per_cta * pitch);
    const int token0 = blockIdx.x * p.tokens_per_cta, tokens = min(p.tokens_per_cta, p.n_tokens - token0);
    const int u = threadIdx.x & (width - 1), group = threadIdx.x / width, groups = blockDim.x / width;
    const bool active = u < p.head_dim / 16;
    const Pieces at = pieces_of<HALVES>(p, active ? u : 0);
    const int all = p.heads[0] + p.heads[1] + p.heads[2], total = tokens * all;
    const float inv_d = 1.0f / (float)p.head_dim;

    // One vector (token, head) per group of lanes and round, kBatch rounds at a time; the loads of the next rounds are on
    // their way while these are worked off, and the first ones while the angles are formed.
    struct Item {
        Raw8<T> lo, hi;
        T* to;                                              // nullptr: nothing to do
        int of, token;
    };
    int t = group / all, h = group - t * all;               // this group's next vector
    auto fetch = [&](Item& x) {
        x.to = nullptr;
        x.of = x.token = 0;
        x.lo = x.hi = Raw8<T>{};
        if (t < tokens) {
            const T* from;
            x.token = t;
            if (locate<T>(p, slots, token0, t, h, x.of, from, x.to) && active) {
                x.lo = load_raw8(from + at.lo);
                x.hi = load_raw8(from + at.hi);
            } else {
                x.to = nullptr;
            }
            h += groups;
            while (h >= all) h -= all, ++t;
        }
    };
    Item next[kBatch];
    if (p.paged) {
        find_slots(p, slots, token0, tokens);
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) fetch(next[i]);
    if (p.n_axes) fill_table<HALVES ? kHalfUnits : kAdjacentUnits>(p, table, pitch, token0, tokens, false);
    if (p.norm) fill_gains(p, gains);
    __syncthreads();

    for (int base = 0; base < total; base += groups * kBatch) {   // the same rounds for all lanes: sums are shuffles
        Item now[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) now[i] = next[i];
        if (base + groups * kBatch < total) {
#pragma unroll
            for (int i = 0; i < kBatch; ++i) fetch(next[i]);
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            Item& x = now[i];
            float lo[8], hi[8];
            widen8(x.lo, lo);
            widen8(x.hi, hi);
            if (p.norm) {
                float sq = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) sq += lo[e] * lo[e] + hi[e] * hi[e];
                const float r = rsqrtf(head_sum(sq, width) * inv_d + p.eps);
                if (x.of < 2) {
                    float g[8];
                    load_eight(gains + x.of * p.head_dim + at.lo, g);
#pragma unroll
                    for (int e = 0; e < 8; ++e) lo[e] *= r * g[e];
                    load_eight(gains + x.of * p.head_dim + at.hi, g);
#pragma unroll
                    for (int e = 0; e < 8; ++e) hi[e] *= r * g[e];
                }
            }
            if (!x.to) continue;
            if (x.of == 2) {                                // a copy, whatever the bits say
                store_raw8(x.to + at.lo, x.lo);
                store_raw8(x.to + at.hi, x.hi);
                continue;
            }
            if (at.turns) turn<HALVES>(lo, hi, reinterpret_cast<const float4*>(table + x.token * pitch) + u, units);
            store8(x.to + at.lo, lo);
            store8(x.to + at.hi, hi);
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kHeadThreads) head_rows_element_kernel(const __grid_constant__ HeadRowsParams p) {
    extern __shared__ float4 table_raw[];
    __shared__ Slots slots;
    float2* table = reinterpret_cast<float2*>(table_raw);
    const int pitch = table_pitch(p);
    const int token0 = blockIdx.x * p.tokens_per_cta, tokens = min(p.tokens_per_cta, p.n_tokens - token0);
    const int lane = threadIdx.x & 31, all = p.heads[0] + p.heads[1] + p.heads[2];
    const int units = p.head_dim - p.n_pairs;
    if (p.n_axes) fill_table<kPlain>(p, table, pitch, token0, tokens, false);
    if (p.paged) find_slots(p, slots, token0, tokens);
    __syncthreads();
    for (int i = threadIdx.x >> 5; i < tokens * all; i += blockDim.x >> 5) {
        const int t = i / all;
        int w;
        const T* from;
        T* to;
        if (!locate<T>(p, slots, token0, t, i - t * all, w, from, to)) continue;   // the whole warp
        T a[kUnits], b[kUnits];
        float sq = 0.0f;
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            const int u = lane + 32 * k;
            if (u < units) {
                a[k] = from[unit_first(u, p)];
                sq += to_f32(a[k]) * to_f32(a[k]);
                if (u < p.n_pairs) {
                    b[k] = from[unit_second(u, p)];
                    sq += to_f32(b[k]) * to_f32(b[k]);
                }
            }
        }
        const bool norm = p.norm && w < 2;
        const float r = norm ? rsqrtf(warp_sum(sq) / (float)p.head_dim + p.eps) : 1.0f;
        const float* gain = norm ? p.weight[w] : nullptr;
#pragma unroll
        for (int k = 0; k < kUnits; ++k) {
            const int u = lane + 32 * k;
            if (u >= units) continue;
            if (w == 2) {                                   // a copy, whatever the bits say
                to[unit_first(u, p)] = a[k];
                if (u < p.n_pairs) to[unit_second(u, p)] = b[k];
                continue;
            }
            float x = to_f32(a[k]) * r;
            if (gain) x *= gain[unit_first(u, p)];
            if (u < p.n_pairs) {
                float y = to_f32(b[k]) * r;
                if (gain) y *= gain[unit_second(u, p)];
                const float2 cs = table[t * pitch + u];
                from_f32(x * cs.x - y * cs.y, to[unit_first(u, p)]);
                from_f32(y * cs.x + x * cs.y, to[unit_second(u, p)]);
            } else {
                from_f32(x, to[unit_first(u, p)]);
            }
        }
    }
}

// Tokens per thread block: enough vectors for `rounds` per group of lanes; fewer where that would leave the device less than
// one round of blocks.
template <typename K>
cudaError_t plan_rows(K kernel, HeadRowsParams& p, int groups, int rounds, int sm_count, int* blocks, size_t* smem) {
    const int all = p.heads[0] + p.heads[1] + p.heads[2];
    int tokens = rounds * groups / all;
    if (tokens > kMaxTokens) tokens = kMaxTokens;
    const size_t per_token = (size_t)table_pitch(p) * sizeof(float2), gains = 2 * (size_t)p.head_dim * sizeof(float);
    if (p.n_tokens <= sm_count) tokens = 1;   // (and no query, which takes longer than such a call's kernel)
    if (tokens > 1) {
        int per_sm = 1;
        const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, kHeadThreads, tokens * per_token + gains);
        if (e != cudaSuccess) return e;
        const long long room = (long long)(per_sm > 0 ? per_sm : 1) * sm_count, even = (p.n_tokens + room - 1) / room;
        if (tokens > even) tokens = (int)even;
    }
    if (tokens < 1) tokens = 1;
    p.tokens_per_cta = tokens;
    *blocks = (p.n_tokens + tokens - 1) / tokens;
    *smem = tokens * per_token + gains;
    return cudaSuccess;
}

template <typename T>
cudaError_t launch_typed(HeadRowsParams& p, bool vec, int sm_count, cudaStream_t stream) {
    int blocks = 0;
    size_t smem = 0;
    if (!in_units(p, vec)) {
        const cudaError_t e = plan_rows(head_rows_element_kernel<T>, p, kHeadThreads / 32, 16, sm_count, &blocks, &smem);
        if (e != cudaSuccess) return e;
        head_rows_element_kernel<T><<<blocks, kHeadThreads, smem, stream>>>(p);
        return cudaGetLastError();
    }
    const int width = lanes_of_head(p);
    auto kernel = p.halves ? head_rows_kernel<T, true> : head_rows_kernel<T, false>;
    const cudaError_t e = plan_rows(kernel, p, kHeadThreads / width, 8, sm_count, &blocks, &smem);
    if (e != cudaSuccess) return e;
    kernel<<<blocks, kHeadThreads, smem, stream>>>(p, width);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_head_rows(HeadRowsParams p, int type, bool vec, int sm_count, cudaStream_t stream) {
    if (type == kTypeBf16) return launch_typed<__nv_bfloat16>(p, vec, sm_count, stream);
    if (type == kTypeF16) return launch_typed<__half>(p, vec, sm_count, stream);
    return launch_typed<float>(p, vec, sm_count, stream);
}

}  // namespace regenvc
