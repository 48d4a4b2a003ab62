// Pieces shared by the kernels on the heads of queries and keys: the table of a token group's angles and the sums over a
// head.
//
// A head's elements are worked off in chunks of eight, one lane per chunk; a group of 8, 16 or 32 lanes (the next power of
// two) holds a head, so that its sums are a few shuffles.  A lane keeps its chunk, and with it its gains, throughout.
#pragma once
#include "head_rows.cuh"
#include "row_io.cuh"

namespace regenvc {
namespace {

constexpr int kHeadThreads = 256;

// Words of a token's table: (cos, sin) of pair j where the lane that holds the pair finds it as 16-byte words of two pairs,
// word i of chunk c at i * chunks + c, so that neighbouring lanes read neighbouring words.  Adjacent pairs: four to a chunk,
// behind the last rotated pair (1, 0).  Halves: eight to a chunk of the first half, and the same for its partner's.
__device__ __forceinline__ int place_adjacent(int j, int chunks) { return ((j >> 1 & 1) * chunks + (j >> 2)) * 2 + (j & 1); }
__device__ __forceinline__ int place_halves(int j, int chunks) { return ((j >> 1 & 3) * chunks + (j >> 3)) * 2 + (j & 1); }

enum { kPlain = 0, kAdjacentChunks = 1, kHalfChunks = 2 };

// Angles in whole turns, position * frequency / (2 pi) in 64 bits, its fraction taken there too; sine and cosine of the
// fraction in 32 bits.
template <int ORDER>
__device__ __forceinline__ void fill_table(const HeadRowsParams& p, float2* table, int pitch, int token0, int tokens, bool back) {
    const int entries = ORDER == kAdjacentChunks ? p.head_dim / 2 : p.n_pairs;
    for (int i = threadIdx.x; i < tokens * entries; i += blockDim.x) {
        const int t = i / entries, j = i - t * entries;
        float s = 0.0f, k = 1.0f;
        if (j < p.n_pairs) {
            int axis = 0;
            while (axis + 1 < p.n_axes && j >= p.axis_end[axis]) ++axis;
            const long long at = axis * p.pos_stride + token0 + t;
            const double pos = p.pos_float ? (double)reinterpret_cast<const float*>(p.positions)[at]
                                           : (double)reinterpret_cast<const int*>(p.positions)[at];
            const double turn = pos * p.turns[j];
            sincospif(2.0f * (float)(turn - rint(turn)), &s, &k);
        }
        const int to = ORDER == kAdjacentChunks ? place_adjacent(j, p.head_dim / 8)
                       : ORDER == kHalfChunks   ? place_halves(j, p.n_pairs / 8)
                                                : j;
        table[t * pitch + to] = make_float2(k, back ? -s : s);
    }
}
__host__ __device__ inline int table_pitch(const HeadRowsParams& p) {
    return ((p.n_axes ? p.head_dim / 2 : 0) + 3) & ~3;   // adjacent chunks fill up to the whole head
}

// Sum over the group of `width` lanes (8, 16 or 32) that holds a head.
__device__ __forceinline__ float head_sum(float v, int width) {
    if (width >= 32) v += __shfl_xor_sync(0xffffffffu, v, 16);
    if (width >= 16) v += __shfl_xor_sync(0xffffffffu, v, 8);
    v += __shfl_xor_sync(0xffffffffu, v, 4);
    v += __shfl_xor_sync(0xffffffffu, v, 2);
    return v + __shfl_xor_sync(0xffffffffu, v, 1);
}

// (a, b) -> (a cos - b sin, b cos + a sin) for every pair of a chunk; cs: the token's table.  All lanes of a warp call it.
template <bool HALVES>
__device__ __forceinline__ void turn_chunk(float* v, const float2* cs, const HeadRowsParams& p, int c, int chunks) {
    if constexpr (!HALVES) {
        const float4* q = reinterpret_cast<const float4*>(cs) + c;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float4 t = q[i * chunks];
            const float a = v[4 * i], b = v[4 * i + 1], a2 = v[4 * i + 2], b2 = v[4 * i + 3];
            v[4 * i] = a * t.x - b * t.y;
            v[4 * i + 1] = b * t.x + a * t.y;
            v[4 * i + 2] = a2 * t.z - b2 * t.w;
            v[4 * i + 3] = b2 * t.z + a2 * t.w;
        }
    } else {
        const int half = p.n_pairs >> 3;                    // chunks of the first half
        const bool low = c < half, high = !low && c < 2 * half;
        const int lane = threadIdx.x & 31, other = low ? lane + half : (high ? lane - half : lane);
        const float4* q = reinterpret_cast<const float4*>(cs) + (low ? c : (high ? c - half : 0));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = __shfl_sync(0xffffffffu, v[2 * i], other), y = __shfl_sync(0xffffffffu, v[2 * i + 1], other);
            const float4 t = q[i * half];
            if (low | high) {
                const float s0 = low ? -t.y : t.y, s1 = low ? -t.w : t.w;
                v[2 * i] = v[2 * i] * t.x + x * s0;
                v[2 * i + 1] = v[2 * i + 1] * t.z + y * s1;
            }
        }
    }
}

__device__ __forceinline__ void load_gains(const float* w, int c, bool active, float* g) {
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = w && active ? w[8 * c + i] : 1.0f;
}

// Element form (rows without 16-byte alignment, head_dim not a multiple of 8): a warp holds a head, unit u of it is pair u
// for u < n_pairs and one unrotated element behind; up to 255 units, eight to a lane.
constexpr int kUnits = 8;
__device__ __forceinline__ int unit_first(int u, const HeadRowsParams& p) {
    return u >= p.n_pairs ? p.n_pairs + u : (p.halves ? u : 2 * u);
}
__device__ __forceinline__ int unit_second(int u, const HeadRowsParams& p) { return p.halves ? u + p.n_pairs : 2 * u + 1; }

}  // namespace
}  // namespace regenvc
