// Pieces shared by the kernels on the heads of queries and keys: the table of a token group's angles, the gains, and the
// pieces of a head.
//
// A lane holds sixteen elements of a head, as two pieces of eight: eight of the first and the matching eight of the second
// half (in half pairs: of the rotated part, and of the part that is not rotated alike).  Either way it holds both elements of
// its pairs, and neighbouring lanes read neighbouring 16-byte words (sixteen neighbours to a lane touched every sector twice,
// at twice the time).  A group of 4, 8 or 16 lanes (the next power of two) holds a head; its sums are a few shuffles.
#pragma once
#include "head_rows.cuh"
#include "row_io.cuh"

namespace regenvc {
namespace {

constexpr int kHeadThreads = 256;

enum { kPlain = 0, kAdjacentUnits = 1, kHalfUnits = 2 };

// Units of eight pairs of a table: the rotated ones, and for adjacent pairs, to the end of the head, (1, 0).
template <int ORDER>
__device__ __forceinline__ int table_units(const HeadRowsParams& p) {
    return ORDER == kAdjacentUnits ? p.head_dim / 16 : p.n_pairs / 8;
}
// Words of a token's table: (cos, sin) of pair j where the lane that holds the pair finds it as 16-byte words of two pairs,
// word i (of four) of unit u at i * units + u, so that neighbouring lanes read neighbouring words.
template <int ORDER>
__device__ __forceinline__ int place(const HeadRowsParams& p, int j) {
    const int units = table_units<ORDER>(p);
    if (ORDER == kHalfUnits) return ((j >> 1 & 3) * units + (j >> 3)) * 2 + (j & 1);
    const int half = j >= 4 * units;
    j -= half * 4 * units;
    return ((2 * half + (j >> 1 & 1)) * units + (j >> 2)) * 2 + (j & 1);
}
// Angles in whole turns, position * frequency / (2 pi) in 64 bits, its fraction taken there too; sine and cosine of the
// fraction in 32 bits.
template <int ORDER>
__device__ __forceinline__ void fill_table(const HeadRowsParams& p, float2* table, int pitch, int token0, int tokens, bool back) {
    // a thread has one pair throughout (its axis, frequency and place), and every so many tokens
    const int entries = ORDER == kAdjacentUnits ? p.head_dim / 2 : p.n_pairs;
    const int at_a_time = blockDim.x / entries, first = threadIdx.x / entries, j = threadIdx.x - first * entries;
    if (first >= at_a_time) return;
    float2* to = table + (ORDER == kPlain ? j : place<ORDER>(p, j));
    if (j >= p.n_pairs) {
        for (int t = first; t < tokens; t += at_a_time) to[t * pitch] = make_float2(1.0f, 0.0f);
        return;
    }
    int axis = 0;
    while (axis + 1 < p.n_axes && j >= p.axis_end[axis]) ++axis;
    const long long at = axis * p.pos_stride + token0;
    const double turns = p.turns[j];
#pragma unroll 4
    for (int t = first; t < tokens; t += at_a_time) {
        const double pos = p.pos_float ? (double)reinterpret_cast<const float*>(p.positions)[at + t]
                                       : (double)reinterpret_cast<const int*>(p.positions)[at + t];
        const double turn = pos * turns;
        float s, k;
        sincospif(2.0f * (float)(turn - rint(turn)), &s, &k);
        to[t * pitch] = make_float2(k, back ? -s : s);
    }
}
__host__ __device__ inline int table_pitch(const HeadRowsParams& p) {
    return ((p.n_axes ? p.head_dim / 2 : 0) + 3) & ~3;
}
// Gains of q and k [2][head_dim] (ones where there are none).
__device__ __forceinline__ void fill_gains(const HeadRowsParams& p, float* gains) {
    for (int i = threadIdx.x; i < 2 * p.head_dim; i += blockDim.x) {
        const int w = i >= p.head_dim;
        gains[i] = p.weight[w] ? p.weight[w][i - w * p.head_dim] : 1.0f;
    }
}

// Sum over the group of `width` lanes (4, 8 or 16) that holds a head.
__device__ __forceinline__ float head_sum(float v, int width) {
    if (width >= 16) v += __shfl_xor_sync(0xffffffffu, v, 8);
    if (width >= 8) v += __shfl_xor_sync(0xffffffffu, v, 4);
    v += __shfl_xor_sync(0xffffffffu, v, 2);
    return v + __shfl_xor_sync(0xffffffffu, v, 1);
}
__device__ __forceinline__ float warp_sum(float v) { return head_sum(v + __shfl_xor_sync(0xffffffffu, v, 16), 16); }

// Where unit u's two pieces of eight lie in a head.
struct Pieces {
    int lo, hi;
    bool turns;     // (half pairs: a unit behind the rotated part does not turn)
};
template <bool HALVES>
__device__ __forceinline__ Pieces pieces_of(const HeadRowsParams& p, int u) {
    if (!HALVES) return {8 * u, p.head_dim / 2 + 8 * u, p.n_axes > 0};
    const int units = p.n_pairs / 8;
    if (u < units) return {8 * u, p.n_pairs + 8 * u, p.n_axes > 0};
    const int at = 2 * p.n_pairs + 8 * (u - units);
    return {at, at + p.head_dim / 2 - p.n_pairs, false};
}

// (a, b) -> (a cos - b sin, b cos + a sin) for the eight pairs of a unit; words: the token's table from the unit's word on.
template <bool HALVES>
__device__ __forceinline__ void turn(float* lo, float* hi, const float4* words, int units) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float4 t = words[i * units];
        if (HALVES) {
            const float a = lo[2 * i], b = hi[2 * i], a2 = lo[2 * i + 1], b2 = hi[2 * i + 1];
            lo[2 * i] = a * t.x - b * t.y;
            hi[2 * i] = b * t.x + a * t.y;
            lo[2 * i + 1] = a2 * t.z - b2 * t.w;
            hi[2 * i + 1] = b2 * t.z + a2 * t.w;
        } else {
            float* v = i < 2 ? lo + 4 * i : hi + 4 * (i - 2);
            const float a = v[0], b = v[1], a2 = v[2], b2 = v[3];
            v[0] = a * t.x - b * t.y;
            v[1] = b * t.x + a * t.y;
            v[2] = a2 * t.z - b2 * t.w;
            v[3] = b2 * t.z + a2 * t.w;
        }
    }
}
__device__ __forceinline__ void load_eight(const float* g, float* v) {
    const float4 a = reinterpret_cast<const float4*>(g)[0], b = reinterpret_cast<const float4*>(g)[1];
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}

// Whether a call's rows can be worked off in units; `width`: lanes of a head.
inline bool in_units(const HeadRowsParams& p, bool vec) {
    return vec && p.head_dim % 16 == 0 && (!p.halves || p.n_pairs % 8 == 0);
}
inline int lanes_of_head(const HeadRowsParams& p) { return p.head_dim <= 64 ? 4 : (p.head_dim <= 128 ? 8 : 16); }

// Element form (rows without 16-byte alignment, other head_dim): a warp holds a head, unit u of it is pair u for
// u < n_pairs and one unrotated element behind; up to 255 units, eight to a lane.
constexpr int kUnits = 8;
__device__ __forceinline__ int unit_first(int u, const HeadRowsParams& p) {
    return u >= p.n_pairs ? p.n_pairs + u : (p.halves ? u : 2 * u);
}
__device__ __forceinline__ int unit_second(int u, const HeadRowsParams& p) { return p.halves ? u + p.n_pairs : 2 * u + 1; }

}  // namespace
}  // namespace regenvc
