// Pieces shared by the kernels on the heads of queries and keys: the table of a token group's angles, the gains, and the
// pieces of a head.
//
// A lane holds sixteen elements of a head, as two pieces of eight: eight of the first and the matching eight of the second
// half (in half pairs: of the rotated part, and of the part that is not rotated alike).  Either way it holds both elements of
// its pairs, and neighbouring lanes read neighbouring 16-byte words (sixteen neighbours to a lane touched every sector twice,
// at twice the time).  A group of 4, 8 or 16 lanes (the next power of two) holds a head; its sums are a few shuffles.
// What these kernels run out of first is issue slots, so a lane's eight pairs are four twos of pairs, first elements in one
// 64-bit register and second elements in another, and all arithmetic is on two of them at once.
#pragma once
#include "head_rows.cuh"
#include "row_io.cuh"

namespace regenvc {
namespace {

constexpr int kHeadThreads = 256;

enum { kPlain = 0, kAdjacentUnits = 1, kHalfUnits = 2 };

// Units of eight pairs of a table: the rotated ones, and for adjacent pairs, to the end of the head, (1, 0).  (Those pairs do
// not turn, see turn(); the angles fill the words that whole units are read in.)
template <int ORDER>
__device__ __forceinline__ int table_units(const HeadRowsParams& p) {
    return ORDER == kAdjacentUnits ? p.head_dim / 16 : p.n_pairs / 8;
}
// Where in a token's table (in floats) the cosine of pair j lies; its sine lies two behind.  Two pairs make a 16-byte word
// (cos, cos, sin, sin), word i (of four) of unit u is at i * units + u: neighbouring lanes read neighbouring words.
template <int ORDER>
__device__ __forceinline__ int place(const HeadRowsParams& p, int j) {
    const int units = table_units<ORDER>(p);
    if (ORDER == kHalfUnits) return ((j >> 1 & 3) * units + (j >> 3)) * 4 + (j & 1);
    const int half = j >= 4 * units;
    j -= half * 4 * units;
    return ((2 * half + (j >> 1 & 1)) * units + (j >> 2)) * 4 + (j & 1);
}
// Angles in whole turns, position * frequency / (2 pi) in 64 bits, its fraction taken there too; sine and cosine of the
// fraction in 32 bits.
template <int ORDER>
__device__ __forceinline__ void fill_table(const HeadRowsParams& p, float2* table, int pitch, int token0, int tokens, bool back) {
    // a thread has one pair throughout (its axis, frequency and place), and every so many tokens
    const int entries = ORDER == kAdjacentUnits ? p.head_dim / 2 : p.n_pairs;
    const int at_a_time = blockDim.x / entries, first = threadIdx.x / entries, j = threadIdx.x - first * entries;
    if (first >= at_a_time) return;
    float* to = reinterpret_cast<float*>(table) + (ORDER == kPlain ? 2 * j : place<ORDER>(p, j));
    const int sine = ORDER == kPlain ? 1 : 2;
    if (j >= p.n_pairs) {
        for (int t = first; t < tokens; t += at_a_time) to[2 * t * pitch] = 1.0f, to[2 * t * pitch + sine] = 0.0f;
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
        to[2 * t * pitch] = k;
        to[2 * t * pitch + sine] = back ? -s : s;
    }
}
__host__ __device__ inline int table_pitch(const HeadRowsParams& p) {
    return ((p.n_axes ? p.head_dim / 2 : 0) + 3) & ~3;
}
// Where the gains of an operand lie (in floats, head_dim of them): word i (of four) of unit u at i * units + u, as above, in
// the order of Unit.  offset: of an element in its head.
template <bool HALVES>
__device__ __forceinline__ int gain_place(const HeadRowsParams& p, int offset) {
    const int units = p.head_dim / 16;
    int u, second, e;                                       // e: of the eight of a piece
    if (HALVES) {
        const int turned = 2 * p.n_pairs, behind = offset >= turned, half = behind ? p.head_dim / 2 - p.n_pairs : p.n_pairs;
        offset -= behind ? turned : 0;
        second = offset >= half;
        offset -= second ? half : 0;
        u = (behind ? p.n_pairs / 8 : 0) + offset / 8;
        e = offset & 7;
        return ((2 * second + (e >> 2)) * units + u) * 4 + (e & 3);
    }
    second = offset >= p.head_dim / 2;
    offset -= second ? p.head_dim / 2 : 0;
    u = offset / 8;
    e = offset & 7;
    return ((2 * second + (e >> 2)) * units + u) * 4 + ((e & 1) << 1 | (e >> 1 & 1));
}
// Gains of q and k [2][head_dim] (ones where there are none).
template <bool HALVES>
__device__ __forceinline__ void fill_gains(const HeadRowsParams& p, float* gains) {
    for (int i = threadIdx.x; i < 2 * p.head_dim; i += blockDim.x) {
        const int w = i >= p.head_dim, offset = i - w * p.head_dim;
        gains[w * p.head_dim + gain_place<HALVES>(p, offset)] = p.weight[w] ? p.weight[w][offset] : 1.0f;
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

// A unit's eight pairs: two i holds the pairs 2i and 2i + 1, first elements in a, second ones in b.
struct Unit {
    uint64_t a[4], b[4];
};
// Offset in its head of element `second` (0 or 1) of pair 2i + k.
template <bool HALVES>
__device__ __forceinline__ int offset_of(const Pieces& at, int i, int k, int second) {
    return HALVES ? (second ? at.hi : at.lo) + 2 * i + k : (i < 2 ? at.lo + 4 * i : at.hi + 4 * (i - 2)) + 2 * k + second;
}
template <bool HALVES, typename T>
__device__ __forceinline__ Unit widen(const Raw8<T>& lo, const Raw8<T>& hi) {
    float l[8], h[8];
    widen8(lo, l);
    widen8(hi, h);
    Unit v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float* f = i < 2 ? l + 4 * i : h + 4 * (i - 2);
        v.a[i] = HALVES ? pack2(l[2 * i], l[2 * i + 1]) : pack2(f[0], f[2]);
        v.b[i] = HALVES ? pack2(h[2 * i], h[2 * i + 1]) : pack2(f[1], f[3]);
    }
    return v;
}
template <bool HALVES>
__device__ __forceinline__ void spread(const Unit& v, float* l, float* h) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float* f = i < 2 ? l + 4 * i : h + 4 * (i - 2);
        if (HALVES) unpack2(v.a[i], l[2 * i], l[2 * i + 1]), unpack2(v.b[i], h[2 * i], h[2 * i + 1]);
        else unpack2(v.a[i], f[0], f[2]), unpack2(v.b[i], f[1], f[3]);
    }
}
// The gains of a unit; words: those of its operand from the unit's word on.
template <bool HALVES>
__device__ __forceinline__ Unit load_gains(const ulonglong2* words, int units) {
    Unit v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const ulonglong2 g = words[i * units];
        if (HALVES) {
            uint64_t* to = i < 2 ? v.a + 2 * i : v.b + 2 * (i - 2);
            to[0] = g.x, to[1] = g.y;
        } else {
            v.a[i] = g.x, v.b[i] = g.y;
        }
    }
    return v;
}
// (a, b) -> (a cos - b sin, b cos + a sin)
struct Angles {
    uint64_t cos[4], sin[4];
};
__device__ __forceinline__ Angles load_angles(const ulonglong2* words, int units) {   // words: the token's, from the unit's on
    Angles v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const ulonglong2 t = words[i * units];
        v.cos[i] = t.x, v.sin[i] = t.y;
    }
    return v;
}
__device__ __forceinline__ void turn(Unit& v, const Angles& by) {
    const uint64_t minus = pack2(-1.0f, -1.0f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint64_t a = v.a[i], b = v.b[i];
        v.a[i] = fma2(a, by.cos[i], mul2(mul2(b, minus), by.sin[i]));
        v.b[i] = fma2(b, by.cos[i], mul2(a, by.sin[i]));
    }
}
// The same for adjacent pairs of which the head's last do not turn: they keep their values (a 1 - b 0 is not a number where b is
// infinite).  pairs: of a head that turn, less those before the unit's first piece; second: pairs from there to its second piece.
__device__ __forceinline__ void turn_some(Unit& v, const Angles& by, int pairs, int second) {
    Unit y = v;
    turn(y, by);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int left = pairs - (i < 2 ? 2 * i : second + 2 * (i - 2));   // of this two: none, one or both
        float a0, a1, b0, b1, c0, c1, d0, d1;
        unpack2(v.a[i], a0, a1), unpack2(v.b[i], b0, b1);
        unpack2(y.a[i], c0, c1), unpack2(y.b[i], d0, d1);
        v.a[i] = pack2(left > 0 ? c0 : a0, left > 1 ? c1 : a1);
        v.b[i] = pack2(left > 0 ? d0 : b0, left > 1 ? d1 : b1);
    }
}
__device__ __forceinline__ float sum2(uint64_t v) {
    float a, b;
    unpack2(v, a, b);
    return a + b;
}

// Whether a call's rows can be worked off in units: aligned, whole units, strides of less than 2 GB (farther vectors take the
// element form, with 64-bit strides).  Fills the views.
inline bool in_units(HeadRowsParams& p, bool vec, int size) {
    if (!vec || p.head_dim % 16 || (p.halves && p.n_pairs % 8)) return false;
    bool fits = true;
    auto bytes = [&](long long stride, int extent) {   // (of one vector no stride is taken)
        if (extent <= 1) return 0;
        fits = fits && stride * size >= 0 && stride * size <= 0x7FFFFFFFll;
        return (int)(stride * size);
    };
    for (int w = 0; w < 3; ++w) {
        HeadRowsView& v = p.view[w];
        v = {};
        if (!p.heads[w]) continue;
        v.from = (const char*)p.in[w];
        v.to = (char*)p.out[w];
        v.from_token = bytes(p.in_token[w], p.n_tokens);
        v.from_head = bytes(p.in_head[w], p.heads[w]);
        v.to_token = p.paged && w ? 0 : bytes(p.out_token[w], p.n_tokens);   // (a cache's slots have offsets of their own)
        v.to_head = bytes(p.out_head[w], p.heads[w]);
        if (w == 2 || !p.grad[w]) continue;
        v.dy = (const char*)p.grad[w];
        v.dy_token = bytes(p.grad_token[w], p.n_tokens);
        v.dy_head = bytes(p.grad_head[w], p.heads[w]);
    }
    return fits;
}
// Adjacent pairs of which some do not turn (half pairs have units of their own for what does not).
inline bool turns_some(const HeadRowsParams& p) { return !p.halves && p.n_axes > 0 && 2 * p.n_pairs < p.head_dim; }
inline int lanes_of_head(const HeadRowsParams& p) { return p.head_dim <= 64 ? 4 : (p.head_dim <= 128 ? 8 : 16); }

// Tokens per thread block: a power of two, so that a token has a whole number of the block's groups and these walk over its
// heads.  More of them leave less of the last round empty and form angles with more of the block at a time; up to `rounds`
// rounds, and only while `blocks` blocks are left.
constexpr int kHeadTokens = 16;
inline int tokens_of_block(int n_tokens, int all, int groups, int rounds, long long blocks) {
    int tokens = 1;
    while (2 * tokens <= kHeadTokens && 2 * tokens <= groups && ((long long)all * 2 * tokens + groups - 1) / groups <= rounds &&
           (n_tokens + 2 * tokens - 1) / (2 * tokens) >= blocks)
        tokens *= 2;
    return tokens;
}

// Element form (rows without 16-byte alignment, other head_dim): a warp holds a head, unit u of it is pair u for
// u < n_pairs and one unrotated element behind; up to 255 units, eight to a lane.
constexpr int kUnits = 8;
__device__ __forceinline__ int unit_first(int u, const HeadRowsParams& p) {
    return u >= p.n_pairs ? p.n_pairs + u : (p.halves ? u : 2 * u);
}
__device__ __forceinline__ int unit_second(int u, const HeadRowsParams& p) { return p.halves ? u + p.n_pairs : 2 * u + 1; }

}  // namespace
}  // namespace regenvc
