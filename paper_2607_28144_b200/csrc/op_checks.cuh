// Checks of arguments shared by the entry points beside the attention (host code): alignment, overlap of strided operands,
// vectors that do not share memory, the ladder of a rotation's frequencies.
#pragma once
#include <algorithm>
#include <cmath>

#include "../../include/regenvc_attn.h"
#include "common.cuh"

namespace regenvc {

inline bool type_ok(int t) { return t == REGENVC_BF16 || t == REGENVC_F16 || t == REGENVC_F32; }
inline size_t type_size(int t) { return t == REGENVC_F32 ? 4 : 2; }
inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// Bytes from an operand's first to its last element, for overlap tests.
struct Span {
    const void* p;
    size_t bytes;
};
inline Span rows_span(const void* p, long long rows, long long stride, long long width, size_t size) {
    return Span{p, p ? ((size_t)(rows - 1) * (size_t)stride + (size_t)width) * size : 0};
}
inline bool meet(const Span& a, const Span& b) {
    if (!a.p || !b.p || !a.bytes || !b.bytes) return false;
    const uintptr_t a0 = (uintptr_t)a.p, b0 = (uintptr_t)b.p;
    return a0 < b0 + b.bytes && b0 < a0 + a.bytes;
}
// An element's index times its size stays far inside 64 bits.
constexpr long long kMaxStride = 1ll << 31;

inline int launch_done(cudaError_t e, const char* what, int launches) {
    for (int i = 0; i < launches; ++i) count_launch();
    return e == cudaSuccess ? REGENVC_OK : record_cuda_failure(e, what);
}

// Strides of [tokens][heads][head_dim] vectors (0: packed): vectors of different (token, head) pairs do not share memory,
// that is, one of the two strides clears the other's extent.
inline bool head_strides(long long token_in, long long head_in, long long tokens, int heads, int head_dim, long long* token,
                         long long* head) {
    *head = head_in ? head_in : head_dim;
    *token = token_in ? token_in : (long long)heads * head_dim;
    if (*head < head_dim || *head > kMaxStride || *token < head_dim || *token > kMaxStride) return false;
    return *token >= (heads - 1) * *head + head_dim || *head >= (tokens - 1) * *token + head_dim;
}

// Axes of which each one's stride clears all that lies on those with shorter strides, from `extent` elements on: no two of
// their places share memory, and their bytes are counted in 64 bits.  Sorts them; `extent` becomes that of all together.
struct Axis {
    long long stride, count;
};
inline bool nested(Axis* axes, int n, long long* extent) {
    std::sort(axes, axes + n, [](const Axis& a, const Axis& b) { return a.stride < b.stride; });
    for (int i = 0; i < n; ++i) {
        if (axes[i].count == 1) continue;
        if (axes[i].stride < *extent || axes[i].count - 1 > (1ll << 58) / axes[i].stride) return false;
        *extent += (axes[i].count - 1) * axes[i].stride;
    }
    return true;
}

// An operand of [tokens][heads][head_dim] vectors, and whether the vectors of two that cover the same stretch of memory are
// different ones all the same, as in views of one fused tensor: the pair of them is one more axis among tokens and heads, or the
// one's heads lie behind the other's inside one token's stride.
struct HeadView {
    const void* p;
    long long token, head;
    int tokens, heads;
    Span span;
};
inline Span heads_span(const void* p, long long tokens, int heads, long long token, long long head, int head_dim, size_t size) {
    return Span{p, p ? ((size_t)(tokens - 1) * token + (size_t)(heads - 1) * head + head_dim) * size : 0};
}
inline bool views_apart(const HeadView& a, const HeadView& b, int head_dim, size_t size) {
    if (!meet(a.span, b.span)) return true;
    if (a.tokens > 1 && a.token != b.token) return false;
    const HeadView &low = (const char*)a.p < (const char*)b.p ? a : b, &high = &low == &a ? b : a;
    const long long gap = (long long)((const char*)high.p - (const char*)low.p) / (long long)size;
    const HeadView& more = low.heads > high.heads ? low : high;
    Axis axes[3] = {{low.token, low.tokens}, {more.head, more.heads}, {gap, 2}};
    long long extent = head_dim;
    if ((low.head == high.head || low.heads == 1 || high.heads == 1) && nested(axes, 3, &extent)) return true;
    return gap >= (low.heads - 1) * low.head + head_dim && gap + (high.heads - 1) * high.head + head_dim <= low.token;
}

// Frequencies as turns per unit of position: powers of one ratio per ladder, multiplied up in extended precision (64
// factors add up to 2^-58) and rounded to 64 bits.
inline void rope_turns(const int* widths, int n_axes, int n_pairs, bool whole_ladder, float theta, double* turns) {
    const long double turn = 1.0L / 6.283185307179586476925286766559L;
    int j = 0;
    for (int a = 0; a < n_axes; ++a) {
        const int pairs = widths[a] / 2;
        if (a == 0 || !whole_ladder) {
            const int steps = whole_ladder ? n_pairs : pairs;
            turns[j] = (double)turn;
            const long double ratio = std::pow((long double)theta, -1.0L / steps);
            long double f = turn;
            for (int i = 1; i < steps; ++i) turns[j + i] = (double)(f *= ratio);
        }
        j += pairs;
    }
}

}  // namespace regenvc
