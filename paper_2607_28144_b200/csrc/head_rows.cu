// Queries and keys of every head normalised and rotated in one pass, into rows or, with the values, into a paged cache.
//
//     y = R(position) (x / sqrt(mean(x^2) + eps) * w)      over the elements of one head; values are copied
//
// R turns pair j by position[axis(j)] * frequency(j).  The normalised values never round to the rows' type in between.
// Bound: HBM, every element is read and written once (two passes, a norm and a rotation, move twice that); next to it issue
// slots and shared memory's ports.  The angles of a token are shared by all its heads, so a thread block computes them once per
// token into shared memory.  A group of lanes then has one token and walks over its heads: addresses are two multiply-adds, and
// angles and gains come in words without bank conflicts (a walk over (token, head) pairs whose lanes read gains 32 bytes apart
// took 330 instructions and 65 shared wavefronts a vector, and 32 us where this takes 26).  One vector is in flight per group
// beside the one at hand, with four blocks on an SM: angles or gains held in registers over the walk spill (31 to 55 us), three
// blocks 30 us, five 37.
// Measured, 10920 tokens, 12 + 12 heads of 128: bf16 26.0 us, 5.2 TB/s of what it has to move (27.0 with one kernel for rows and
// caches); fp32 48.5 us, 5.5 TB/s; with the values into a cache of 1560-token pages 42.8 us, 4.7 TB/s, fp32 85 us, 4.7 TB/s
// (without the norm 2 to 3 % less).  One token 2.7 us, 64 tokens appended 5 us (a chain of list, page and row behind a launch).
// Four blocks on an SM were chosen on bf16; fp32 takes 64 registers too, of which the kernel for caches spills some 110 bytes.
// Paged: token n of the call belongs to the sequence whose rows it lies in, found by counting the row starts at or before
// it (a warp per token, all loads independent: a binary search is a chain of loads, which is what a call of a few tokens
// would wait for); its slot is the sequence's length minus the rows behind it, its page comes from the table.
#include "common.cuh"
#include "head_rows_core.cuh"

namespace regenvc {
namespace {

constexpr int kMaxTokens = kHeadTokens;

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
                // (starts that do not ascend may count a row to a sequence that does not have it)
                const int first = p.row_starts[seq], end = p.row_starts[seq + 1];
                const long long at = (long long)p.lengths[seq] - ((long long)end - n);
                bool good = first <= n && n < end && end <= p.n_tokens && at >= 0 && at < p.most_tokens;
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

// Lists that contradict each other or the call's sizes, wherever the rows lie that they leave without a place: reported by the
// first block.  The last warps begin, which have no row to look up where a block has fewer than eight.
__device__ __forceinline__ void check_lists(const HeadRowsParams& p) {
    for (int s = blockDim.x - 1 - threadIdx.x; s < p.n_sequences; s += blockDim.x) {
        const int first = p.row_starts[s], end = p.row_starts[s + 1], keys = p.lengths[s];
        if (first < 0 || end < first || end > p.n_tokens || keys < end - first || keys > p.most_tokens)
            atomicCAS(p.status, 0, kStatusRange);
    }
}

// The element form's: where vector (t, h) comes from and goes to; w: 0 q, 1 k, 2 v.
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

// SOME: adjacent pairs of which the head's last do not turn.
template <typename T, bool HALVES, bool PAGED, bool SOME>
__global__ void __launch_bounds__(kHeadThreads, 4) head_rows_kernel(const __grid_constant__ HeadRowsParams p, const int width) {
    extern __shared__ float4 shared_raw[];
    __shared__ Slots slots;
    const int pitch = table_pitch(p), units = p.head_dim / 16, turning = table_units<HALVES ? kHalfUnits : kAdjacentUnits>(p);
    float2* table = reinterpret_cast<float2*>(shared_raw);
    float* gains = reinterpret_cast<float*>(table + p.tokens_per_cta * pitch);
    const int token0 = blockIdx.x * p.tokens_per_cta, tokens = min(p.tokens_per_cta, p.n_tokens - token0);
    // a group of lanes has one token, and every so many of its vectors
    const int u = threadIdx.x & (width - 1), group = threadIdx.x / width, step = blockDim.x / width / p.tokens_per_cta;
    const int t = group / step, all = p.heads[0] + p.heads[1] + p.heads[2], rounds = (all + step - 1) / step;
    bool active = u < units && t < tokens;
    const Pieces at = pieces_of<HALVES>(p, u < units ? u : 0);
    const float inv_d = 1.0f / (float)p.head_dim;
    if (PAGED) {
        find_slots(p, slots, token0, tokens);
        if (blockIdx.x == 0) check_lists(p);
        __syncthreads();
        active = active && slots.rows[t];
    }

    // The loads of the next round are on their way while this one is worked off, the first ones while the angles are formed.
    struct Item {
        Raw8<T> lo, hi;
        T* to;                                              // nullptr: nothing to do
        int of;                                             // 0 q, 1 k, 2 v
    };
    const int lo_bytes = at.lo * (int)sizeof(T), hi_from_lo = at.hi - at.lo;
    const int q_heads = p.heads[0], qk_heads = q_heads + p.heads[1];
    int h = group - t * step;                               // this group's next vector
    auto fetch = [&](Item& x) {
        x.to = nullptr;
        x.of = (h >= q_heads) + (PAGED && h >= qk_heads);
        const long long slot = !PAGED || !x.of ? 0 : (x.of == 1 ? slots.k[t] : slots.v[t]);
        if (active && h < all && slot >= 0) {
            const HeadRowsView& o = p.view[x.of];
            const int token = token0 + t, head = h - (x.of == 0 ? 0 : (!PAGED || x.of == 1 ? q_heads : qk_heads));
            const T* v = reinterpret_cast<const T*>(o.from + (long long)token * o.from_token + (long long)head * o.from_head + lo_bytes);
            x.to = reinterpret_cast<T*>(o.to + (long long)token * o.to_token + (long long)head * o.to_head + lo_bytes) + slot;
            x.lo = load_raw8_once(v);
            x.hi = load_raw8_once(v + hi_from_lo);
        } else {
            x.lo = x.hi = Raw8<T>{};
        }
        h += step;
    };
    Item next;
    fetch(next);
    if (p.n_axes) fill_table<HALVES ? kHalfUnits : kAdjacentUnits>(p, table, pitch, token0, tokens, false);
    if (p.norm) fill_gains<HALVES>(p, gains);
    __syncthreads();
    const ulonglong2* words = reinterpret_cast<const ulonglong2*>(table + t * pitch) + u;

    for (int r = 0; r < rounds; ++r) {                      // the same rounds for all lanes: sums are shuffles
        const Item x = next;
        if (r + 1 < rounds) fetch(next);
        Unit v = widen<HALVES>(x.lo, x.hi);
        if (p.norm) {
            uint64_t sq = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) sq = fma2(v.b[e], v.b[e], fma2(v.a[e], v.a[e], sq));
            const float scale = rsqrtf(head_sum(sum2(sq), width) * inv_d + p.eps);
            if ((!PAGED || x.of < 2) && x.to) {
                const Unit gain = load_gains<HALVES>(reinterpret_cast<const ulonglong2*>(gains) + x.of * 4 * units + u, units);
                const uint64_t r2 = pack2(scale, scale);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v.a[e] = mul2(v.a[e], mul2(r2, gain.a[e]));
                    v.b[e] = mul2(v.b[e], mul2(r2, gain.b[e]));
                }
            }
        }
        if (!x.to) continue;
        if (PAGED && x.of == 2) {                                    // a copy, whatever the bits say
            store_raw8(x.to, x.lo);
            store_raw8(x.to + hi_from_lo, x.hi);
            continue;
        }
        if (SOME) turn_some(v, load_angles(words, turning), p.n_pairs - 4 * u, p.head_dim / 4);
        else if (at.turns) turn(v, load_angles(words, turning));
        float lo[8], hi[8];
        spread<HALVES>(v, lo, hi);
        store8(x.to, lo);
        store8(x.to + hi_from_lo, hi);
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
    if (p.paged) {
        find_slots(p, slots, token0, tokens);
        if (blockIdx.x == 0) check_lists(p);
    }
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

size_t shared_bytes(const HeadRowsParams& p) {
    return p.tokens_per_cta * (size_t)table_pitch(p) * sizeof(float2) + 2 * (size_t)p.head_dim * sizeof(float);
}

template <typename T>
cudaError_t launch_typed(HeadRowsParams& p, bool vec, int sm_count, cudaStream_t stream) {
    const int all = p.heads[0] + p.heads[1] + p.heads[2];
    const bool unit = in_units(p, vec, sizeof(T));
    const int width = unit ? lanes_of_head(p) : 32;
    auto kernel = p.halves        ? (p.paged ? head_rows_kernel<T, true, true, false> : head_rows_kernel<T, true, false, false>)
                  : turns_some(p) ? (p.paged ? head_rows_kernel<T, false, true, true> : head_rows_kernel<T, false, false, true>)
                                  : (p.paged ? head_rows_kernel<T, false, true, false> : head_rows_kernel<T, false, false, false>);
    int per_sm = 1;
    p.tokens_per_cta = kMaxTokens;
    if (p.n_tokens > sm_count) {   // (a query takes longer than the kernel of a call of a few tokens)
        const cudaError_t e = unit ? cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, kHeadThreads, shared_bytes(p))
                                   : cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, head_rows_element_kernel<T>, kHeadThreads, shared_bytes(p));
        if (e != cudaSuccess) return e;
    }
    p.tokens_per_cta = tokens_of_block(p.n_tokens, all, kHeadThreads / width, 12, 2ll * per_sm * sm_count);
    const int blocks = (p.n_tokens + p.tokens_per_cta - 1) / p.tokens_per_cta;
    const size_t smem = shared_bytes(p);
    if (unit) kernel<<<blocks, kHeadThreads, smem, stream>>>(p, width);
    else head_rows_element_kernel<T><<<blocks, kHeadThreads, smem, stream>>>(p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_head_rows(HeadRowsParams p, int type, bool vec, int sm_count, cudaStream_t stream) {
    if (type == kTypeBf16) return launch_typed<__nv_bfloat16>(p, vec, sm_count, stream);
    if (type == kTypeF16) return launch_typed<__half>(p, vec, sm_count, stream);
    return launch_typed<float>(p, vec, sm_count, stream);
}

}  // namespace regenvc
