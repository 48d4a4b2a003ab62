// Entry points of the operators of attention over cached windows: queries and keys normalised and rotated, appending to a
// paged cache, attention over it.  Arguments are checked before any CUDA call; nothing is allocated.
#include "head_rows.cuh"
#include "op_checks.cuh"
#include "paged_attn.cuh"

namespace {

using namespace regenvc;

constexpr long long kMaxPageStride = 1ll << 38;

// The rotation's part of a description, the same in both of those that have one.
template <typename Desc>
int rotation(const Desc* d, const void* positions, HeadRowsParams* p) {
    if (d->n_tokens < 1 || d->n_tokens > (1 << 30) || d->n_q_heads < 0 || d->n_q_heads > 65535 || d->n_k_heads < 0 ||
        d->n_k_heads > 65535 || d->head_dim < 1 || d->head_dim > 2 * kRopeMaxPairs || d->n_axes < 0 || d->n_axes > kRopeMaxAxes)
        return REGENVC_ERR_BAD_SHAPE;
    if ((d->n_axes > 0) != (positions != nullptr)) return REGENVC_ERR_NULL_POINTER;
    if (d->head_dim % 2 != 0 || !type_ok(d->type)) return REGENVC_ERR_UNSUPPORTED;
    if (!(d->eps >= 0.0f) || !std::isfinite(d->eps)) return REGENVC_ERR_UNSUPPORTED;
    if ((d->halves | d->whole_ladder | d->pos_float) & ~1) return REGENVC_ERR_UNSUPPORTED;
    p->n_tokens = d->n_tokens;
    p->head_dim = d->head_dim;
    p->eps = d->eps;
    p->n_axes = d->n_axes;
    if (d->n_axes == 0) return REGENVC_OK;
    if (!(d->rope_theta > 0.0f) || !std::isfinite(d->rope_theta)) return REGENVC_ERR_UNSUPPORTED;
    long long rotated = 0;
    for (int a = 0; a < d->n_axes; ++a) {
        if (d->widths[a] < 2 || d->widths[a] % 2 != 0 || d->widths[a] > d->head_dim) return REGENVC_ERR_BAD_SHAPE;
        rotated += d->widths[a];
        if (rotated > d->head_dim) return REGENVC_ERR_BAD_SHAPE;
        p->axis_end[a] = (int)(rotated / 2);
    }
    p->n_pairs = (int)(rotated / 2);
    p->positions = positions;
    p->pos_stride = d->pos_stride ? d->pos_stride : d->n_tokens;
    if (p->pos_stride < d->n_tokens || p->pos_stride > kMaxStride) return REGENVC_ERR_BAD_SHAPE;
    if (!aligned(positions, 4)) return REGENVC_ERR_MISALIGNED;
    p->pos_float = d->pos_float;
    p->halves = d->halves;
    return REGENVC_OK;
}
template <typename Desc>
void ladder(const Desc* d, HeadRowsParams* p) {
    if (d->n_axes) rope_turns(d->widths, d->n_axes, p->n_pairs, d->whole_ladder != 0, d->rope_theta, p->turns);
}
template <typename Desc>
Span positions_span(const Desc* d, const HeadRowsParams& p) {
    return Span{p.positions, p.positions ? ((size_t)(d->n_axes - 1) * p.pos_stride + d->n_tokens) * 4 : 0};
}

// One operand of [tokens][heads][head_dim] vectors; clears *vec where its rows do not allow 16-byte accesses.
int view_of(const void* ptr, long long token, long long head, int n_tokens, int heads, int head_dim, size_t size, HeadView* v, bool* vec) {
    *v = HeadView{ptr, 0, 0, n_tokens, heads, Span{nullptr, 0}};
    if (!ptr) return REGENVC_OK;
    if (!head_strides(token, head, n_tokens, heads, head_dim, &v->token, &v->head)) return REGENVC_ERR_BAD_SHAPE;
    if (!aligned(ptr, size)) return REGENVC_ERR_MISALIGNED;
    if (!aligned(ptr, 16) || v->token % 8 != 0 || v->head % 8 != 0) *vec = false;
    v->span = heads_span(ptr, n_tokens, heads, v->token, v->head, head_dim, size);
    return REGENVC_OK;
}
bool same_view(const HeadView& a, const HeadView& b) { return a.p == b.p && a.token == b.token && a.head == b.head; }

// A result is one of the operands that it may replace (in place), or clear of every operand's vectors.
bool clear_of(const HeadView& out, const HeadView* ins, int n, const HeadView* in_place, int head_dim, size_t size) {
    if (!out.p) return true;
    const bool replaces = in_place && in_place->p && same_view(out, *in_place);
    for (int i = 0; i < n; ++i) {
        if (!ins[i].p || (in_place && &ins[i] == in_place && replaces)) continue;
        if (!meet(out.span, ins[i].span)) continue;
        if (!replaces || !views_apart(out, ins[i], head_dim, size)) return false;
    }
    return true;
}

// A cache [pages][slots][heads][head_dim] in any order of its strides: vectors do not share memory.  The stride of an axis with
// one entry is never used and taken as a short one.
struct CacheView {
    long long page, slot, head, in_page;   // in_page: elements from a page's first to one past its last
    Span span;
};
int cache_of(const void* ptr, long long page, long long slot, long long head, int n_pages, int page_size, int heads, int head_dim,
             size_t size, CacheView* c) {
    c->head = head ? head : head_dim;
    c->slot = slot ? slot : (long long)heads * head_dim;
    c->page = page ? page : (long long)page_size * heads * head_dim;
    const long long unused = (head_dim + 7) / 8 * 8;
    if (heads == 1) c->head = unused;
    if (page_size == 1) c->slot = unused;
    if (n_pages == 1) c->page = unused;
    if (c->head < head_dim || c->head > kMaxStride || c->slot < head_dim || c->slot > kMaxStride || c->page < head_dim ||
        c->page > kMaxPageStride)
        return REGENVC_ERR_BAD_SHAPE;
    c->in_page = (heads - 1) * c->head + (page_size - 1) * c->slot + head_dim;
    Axis axes[3] = {{c->head, heads}, {c->slot, page_size}, {c->page, n_pages}};
    long long extent = head_dim;
    if (!nested(axes, 3, &extent)) return REGENVC_ERR_BAD_SHAPE;
    c->span = Span{ptr, (size_t)extent * size};
    return REGENVC_OK;
}

// The lists that say which tokens are whose and where they lie.
int lists_ok(int n_sequences, int page_size, int n_pages, int pages_per_sequence, long long* table_stride, const void* starts,
             const void* lengths, const void* table, Span* spans) {
    if (!starts || !lengths || !table) return REGENVC_ERR_NULL_POINTER;
    if (n_sequences < 1 || n_sequences > kPagedMaxSequences || page_size < 1 || page_size > (1 << 20) || n_pages < 1 ||
        n_pages > (1 << 30) || pages_per_sequence < 1 || pages_per_sequence > (1 << 30))
        return REGENVC_ERR_BAD_SHAPE;
    if (*table_stride == 0) *table_stride = pages_per_sequence;
    if (*table_stride < pages_per_sequence || *table_stride > kMaxStride) return REGENVC_ERR_BAD_SHAPE;
    if (!aligned(starts, 4) || !aligned(lengths, 4) || !aligned(table, 4)) return REGENVC_ERR_MISALIGNED;
    spans[0] = Span{starts, ((size_t)n_sequences + 1) * 4};
    spans[1] = Span{lengths, (size_t)n_sequences * 4};
    spans[2] = rows_span(table, n_sequences, *table_stride, pages_per_sequence, 4);
    return REGENVC_OK;
}

}  // namespace

extern "C" {

int regenvc_qk_norm_rope_forward(const regenvc_qk_norm_rope_desc* d, const void* q, const void* k, const void* q_weight,
                                 const void* k_weight, const void* positions, void* q_out, void* k_out, void* stream) {
    if (!d) return REGENVC_ERR_NULL_POINTER;
    HeadRowsParams p{};
    int rc = rotation(d, positions, &p);
    if (rc != REGENVC_OK) return rc;
    if ((!q) != (d->n_q_heads == 0) || (!q_out) != (!q) || (!k) != (d->n_k_heads == 0) || (!k_out) != (!k) || (!q && !k) ||
        (q_weight && !q) || (k_weight && !k))
        return REGENVC_ERR_NULL_POINTER;
    const size_t size = type_size(d->type);
    bool vec = true;
    HeadView in[2], out[2];
    rc = view_of(q, d->q_token_stride, d->q_head_stride, d->n_tokens, d->n_q_heads, d->head_dim, size, &in[0], &vec);
    if (rc == REGENVC_OK) rc = view_of(k, d->k_token_stride, d->k_head_stride, d->n_tokens, d->n_k_heads, d->head_dim, size, &in[1], &vec);
    if (rc == REGENVC_OK)
        rc = view_of(q_out, d->q_out_token_stride, d->q_out_head_stride, d->n_tokens, d->n_q_heads, d->head_dim, size, &out[0], &vec);
    if (rc == REGENVC_OK)
        rc = view_of(k_out, d->k_out_token_stride, d->k_out_head_stride, d->n_tokens, d->n_k_heads, d->head_dim, size, &out[1], &vec);
    if (rc != REGENVC_OK) return rc;
    if (!aligned(q_weight, 4) || !aligned(k_weight, 4)) return REGENVC_ERR_MISALIGNED;
    const Span small[3] = {positions_span(d, p), rows_span(q_weight, 1, 0, d->head_dim, 4), rows_span(k_weight, 1, 0, d->head_dim, 4)};
    for (int w = 0; w < 2; ++w) {
        if (!clear_of(out[w], in, 2, &in[w], d->head_dim, size)) return REGENVC_ERR_ALIASING;
        for (const Span& s : small)
            if (meet(out[w].span, s)) return REGENVC_ERR_ALIASING;
        p.in[w] = in[w].p;
        p.out[w] = const_cast<void*>(out[w].p);
        p.in_token[w] = in[w].token;
        p.in_head[w] = in[w].head;
        p.out_token[w] = out[w].token;
        p.out_head[w] = out[w].head;
    }
    if (out[0].p && out[1].p && !views_apart(out[0], out[1], d->head_dim, size)) return REGENVC_ERR_ALIASING;
    p.heads[0] = d->n_q_heads;
    p.heads[1] = d->n_k_heads;
    p.norm = 1;
    p.weight[0] = reinterpret_cast<const float*>(q_weight);
    p.weight[1] = reinterpret_cast<const float*>(k_weight);
    ladder(d, &p);
    int sm_count = 0;
    rc = op_device(&sm_count, &p.status);
    if (rc != REGENVC_OK) return rc;
    const cudaError_t e = launch_head_rows(p, d->type, vec, sm_count, (cudaStream_t)stream);
    return launch_done(e, "launch of the norm and rotation of the heads", e == cudaSuccess ? 1 : 0);
}

size_t regenvc_qk_norm_rope_workspace_bytes(int head_dim) {
    return head_dim >= 2 && head_dim <= 2 * kRopeMaxPairs && head_dim % 2 == 0 ? head_grad_workspace_bytes(head_dim) : 0;
}

int regenvc_qk_norm_rope_backward(const regenvc_qk_norm_rope_desc* d, const void* dq_out, const void* dk_out, const void* q,
                                  const void* k, const void* q_weight, const void* k_weight, const void* positions, void* dq,
                                  void* dk, void* dq_weight, void* dk_weight, void* workspace, size_t workspace_bytes,
                                  void* stream) {
    if (!d) return REGENVC_ERR_NULL_POINTER;
    HeadRowsParams p{};
    int rc = rotation(d, positions, &p);
    if (rc != REGENVC_OK) return rc;
    if ((!q) != (d->n_q_heads == 0) || (!dq_out) != (!q) || (!dq) != (!q) || (!k) != (d->n_k_heads == 0) || (!dk_out) != (!k) ||
        (!dk) != (!k) || (!q && !k) || (q_weight && !q) || (k_weight && !k) || (dq_weight && !q_weight) || (dk_weight && !k_weight))
        return REGENVC_ERR_NULL_POINTER;
    const bool sums = dq_weight || dk_weight;
    if (sums && !workspace) return REGENVC_ERR_NULL_POINTER;
    const size_t size = type_size(d->type), need = head_grad_workspace_bytes(d->head_dim);
    bool vec = true;
    HeadView ins[4], out[2];   // q, k, the results' gradients
    const long long token[6] = {d->q_token_stride, d->k_token_stride, d->q_out_token_stride, d->k_out_token_stride, d->dq_token_stride, d->dk_token_stride};
    const long long head[6] = {d->q_head_stride, d->k_head_stride, d->q_out_head_stride, d->k_out_head_stride, d->dq_head_stride, d->dk_head_stride};
    const void* ptr[6] = {q, k, dq_out, dk_out, dq, dk};
    for (int i = 0; i < 6; ++i) {
        rc = view_of(ptr[i], token[i], head[i], d->n_tokens, i & 1 ? d->n_k_heads : d->n_q_heads, d->head_dim, size, i < 4 ? &ins[i] : &out[i - 4], &vec);
        if (rc != REGENVC_OK) return rc;
    }
    const void* vectors[4] = {q_weight, k_weight, dq_weight, dk_weight};
    Span small[5] = {positions_span(d, p)};
    for (int i = 0; i < 4; ++i) {
        if (!aligned(vectors[i], 4)) return REGENVC_ERR_MISALIGNED;
        small[1 + i] = rows_span(vectors[i], 1, 0, d->head_dim, 4);
    }
    if (sums && (workspace_bytes < need || !aligned(workspace, 16))) return REGENVC_ERR_WORKSPACE;
    const Span ws{sums ? workspace : nullptr, sums ? need : 0};
    for (int w = 0; w < 2; ++w) {
        // in place over the result's gradient
        if (!clear_of(out[w], ins, 4, &ins[2 + w], d->head_dim, size)) return REGENVC_ERR_ALIASING;
        for (const Span& s : small)
            if (meet(out[w].span, s)) return REGENVC_ERR_ALIASING;
        if (meet(out[w].span, ws)) return REGENVC_ERR_ALIASING;
    }
    if (out[0].p && out[1].p && !views_apart(out[0], out[1], d->head_dim, size)) return REGENVC_ERR_ALIASING;
    // the gains' gradients and the workspace are written too
    for (int i = 3; i < 5; ++i) {
        for (const HeadView& v : ins)
            if (meet(small[i], v.span)) return REGENVC_ERR_ALIASING;
        for (int j = 0; j < 5; ++j)
            if (j != i && meet(small[i], small[j])) return REGENVC_ERR_ALIASING;
    }
    for (const HeadView& v : ins)
        if (meet(ws, v.span)) return REGENVC_ERR_ALIASING;
    for (const Span& s : small)
        if (meet(ws, s)) return REGENVC_ERR_ALIASING;
    for (int w = 0; w < 2; ++w) {
        p.in[w] = ins[w].p;
        p.in_token[w] = ins[w].token;
        p.in_head[w] = ins[w].head;
        p.grad[w] = ins[2 + w].p;
        p.grad_token[w] = ins[2 + w].token;
        p.grad_head[w] = ins[2 + w].head;
        p.out[w] = const_cast<void*>(out[w].p);
        p.out_token[w] = out[w].token;
        p.out_head[w] = out[w].head;
    }
    p.heads[0] = d->n_q_heads;
    p.heads[1] = d->n_k_heads;
    p.norm = 1;
    p.weight[0] = reinterpret_cast<const float*>(q_weight);
    p.weight[1] = reinterpret_cast<const float*>(k_weight);
    p.dweight[0] = reinterpret_cast<float*>(dq_weight);
    p.dweight[1] = reinterpret_cast<float*>(dk_weight);
    p.partial = sums ? reinterpret_cast<float*>(workspace) : nullptr;
    ladder(d, &p);
    int sm_count = 0, launches = 0;
    rc = op_device(&sm_count, &p.status);
    if (rc != REGENVC_OK) return rc;
    const cudaError_t e = launch_head_rows_grad(p, d->type, vec, sm_count, &launches, (cudaStream_t)stream);
    return launch_done(e, "launch of the gradients of the heads' norm and rotation", launches);
}

int regenvc_paged_append(const regenvc_paged_append_desc* d, const void* q, const void* k, const void* v, const void* q_weight,
                         const void* k_weight, const void* positions, const void* row_starts, const void* lengths,
                         const void* block_table, void* q_out, void* k_cache, void* v_cache, void* stream) {
    if (!d) return REGENVC_ERR_NULL_POINTER;
    HeadRowsParams p{};
    int rc = rotation(d, positions, &p);
    if (rc != REGENVC_OK) return rc;
    if (!k || !v || !k_cache || !v_cache || (!q) != (d->n_q_heads == 0) || (!q_out) != (!q)) return REGENVC_ERR_NULL_POINTER;
    if (d->n_k_heads < 1) return REGENVC_ERR_BAD_SHAPE;
    if (d->norm != REGENVC_NORM_NONE && d->norm != REGENVC_NORM_RMS) return REGENVC_ERR_UNSUPPORTED;
    if ((q_weight && (!q || d->norm == REGENVC_NORM_NONE)) || (k_weight && d->norm == REGENVC_NORM_NONE)) return REGENVC_ERR_NULL_POINTER;
    Span lists[6];
    long long table_stride = d->table_stride;
    rc = lists_ok(d->n_sequences, d->page_size, d->n_pages, d->pages_per_sequence, &table_stride, row_starts, lengths, block_table, lists);
    if (rc != REGENVC_OK) return rc;
    const size_t size = type_size(d->type);
    bool vec = true;
    HeadView in[3], out;
    const long long token[3] = {d->q_token_stride, d->k_token_stride, d->v_token_stride};
    const long long head[3] = {d->q_head_stride, d->k_head_stride, d->v_head_stride};
    const void* ptr[3] = {q, k, v};
    for (int i = 0; i < 3; ++i) {
        rc = view_of(ptr[i], token[i], head[i], d->n_tokens, i ? d->n_k_heads : d->n_q_heads, d->head_dim, size, &in[i], &vec);
        if (rc != REGENVC_OK) return rc;
    }
    rc = view_of(q_out, d->q_out_token_stride, d->q_out_head_stride, d->n_tokens, d->n_q_heads, d->head_dim, size, &out, &vec);
    if (rc != REGENVC_OK) return rc;
    CacheView cache[2];
    void* cache_ptr[2] = {k_cache, v_cache};
    rc = cache_of(k_cache, d->k_page_stride, d->k_slot_stride, d->k_cache_head_stride, d->n_pages, d->page_size, d->n_k_heads, d->head_dim, size, &cache[0]);
    if (rc == REGENVC_OK)
        rc = cache_of(v_cache, d->v_page_stride, d->v_slot_stride, d->v_cache_head_stride, d->n_pages, d->page_size, d->n_k_heads, d->head_dim, size, &cache[1]);
    if (rc != REGENVC_OK) return rc;
    if (!aligned(q_weight, 4) || !aligned(k_weight, 4)) return REGENVC_ERR_MISALIGNED;
    lists[3] = positions_span(d, p);
    lists[4] = rows_span(q_weight, 1, 0, d->head_dim, 4);
    lists[5] = rows_span(k_weight, 1, 0, d->head_dim, 4);
    if (!clear_of(out, in, 3, &in[0], d->head_dim, size)) return REGENVC_ERR_ALIASING;
    for (const Span& s : lists)
        if (meet(out.span, s)) return REGENVC_ERR_ALIASING;
    for (int w = 0; w < 2; ++w) {
        if (!aligned(cache_ptr[w], size)) return REGENVC_ERR_MISALIGNED;
        if (!aligned(cache_ptr[w], 16) || cache[w].page % 8 != 0 || cache[w].slot % 8 != 0 || cache[w].head % 8 != 0) vec = false;
        for (const HeadView& i : in)
            if (meet(cache[w].span, i.span)) return REGENVC_ERR_ALIASING;
        for (const Span& s : lists)
            if (meet(cache[w].span, s)) return REGENVC_ERR_ALIASING;
        if (meet(cache[w].span, out.span)) return REGENVC_ERR_ALIASING;
    }
    if (meet(cache[0].span, cache[1].span)) {
        // One tensor with keys beside values: a pair of them is one more axis, in any place among the others; or a page's or a
        // slot's keys lie in front of its values, in orders of their own.
        const bool k_first = (const char*)k_cache < (const char*)v_cache;
        const CacheView &low = k_first ? cache[0] : cache[1], &high = k_first ? cache[1] : cache[0];
        const long long gap = ((const char*)high.span.p - (const char*)low.span.p) / (long long)size;
        Axis axes[4] = {{low.head, d->n_k_heads}, {low.slot, d->page_size}, {low.page, d->n_pages}, {gap, 2}};
        long long extent = d->head_dim;
        const bool alike = low.head == high.head && low.slot == high.slot && low.page == high.page && nested(axes, 4, &extent);
        const bool by_page = low.page == high.page && gap >= low.in_page && gap + high.in_page <= low.page;
        const int heads_behind = d->n_k_heads - 1;
        axes[0] = {low.slot, d->page_size}, axes[1] = {low.page, d->n_pages};
        extent = gap + heads_behind * high.head + d->head_dim;
        const bool by_slot = low.slot == high.slot && low.page == high.page && gap >= heads_behind * low.head + d->head_dim && nested(axes, 2, &extent);
        if (!alike && !by_page && !by_slot) return REGENVC_ERR_ALIASING;
    }
    for (int i = 0; i < 3; ++i) {
        p.in[i] = in[i].p;
        p.in_token[i] = in[i].token;
        p.in_head[i] = in[i].head;
    }
    p.out[0] = q_out;
    p.out_token[0] = out.token;
    p.out_head[0] = out.head;
    for (int w = 0; w < 2; ++w) {
        p.out[1 + w] = cache_ptr[w];
        p.out_token[1 + w] = cache[w].slot;
        p.out_head[1 + w] = cache[w].head;
        p.page_stride[w] = cache[w].page;
    }
    p.heads[0] = d->n_q_heads;
    p.heads[1] = p.heads[2] = d->n_k_heads;
    p.norm = d->norm == REGENVC_NORM_RMS;
    p.weight[0] = reinterpret_cast<const float*>(q_weight);
    p.weight[1] = reinterpret_cast<const float*>(k_weight);
    p.paged = 1;
    p.row_starts = reinterpret_cast<const int*>(row_starts);
    p.lengths = reinterpret_cast<const int*>(lengths);
    p.table = reinterpret_cast<const int*>(block_table);
    p.table_stride = table_stride;
    p.n_sequences = d->n_sequences;
    p.page_size = d->page_size;
    p.n_pages = d->n_pages;
    p.most_tokens = (int)std::min((long long)d->pages_per_sequence * d->page_size, kMaxCachedTokens);
    ladder(d, &p);
    int sm_count = 0;
    rc = op_device(&sm_count, &p.status);
    if (rc != REGENVC_OK) return rc;
    const cudaError_t e = launch_head_rows(p, d->type, vec, sm_count, (cudaStream_t)stream);
    return launch_done(e, "launch of the append to a paged cache", e == cudaSuccess ? 1 : 0);
}

size_t regenvc_paged_attn_workspace_bytes(int n_q_heads, int n_k_heads, int head_dim) {
    if (n_q_heads < 1 || n_k_heads < 1 || n_q_heads % n_k_heads != 0 || (head_dim != 64 && head_dim != 128)) return 0;
    return paged_attn_workspace_bytes(head_dim);
}

int regenvc_paged_attn_forward(const regenvc_paged_attn_desc* d, const void* q, const void* k_cache, const void* v_cache,
                               const void* row_starts, const void* lengths, const void* block_table, void* out, void* lse,
                               void* workspace, size_t workspace_bytes, void* stream) {
    if (!d || !q || !k_cache || !v_cache || !out || !workspace) return REGENVC_ERR_NULL_POINTER;
    if (d->n_tokens < 1 || d->n_tokens > (1 << 30) || d->n_q_heads < 1 || d->n_q_heads > 65535 || d->n_k_heads < 1 ||
        d->n_q_heads % d->n_k_heads != 0 || (long long)d->n_tokens * d->n_q_heads >= (1ll << 31) - kPagedRows || d->group < 0 ||
        d->window < 0 || (d->window > 0 && d->group == 0))
        return REGENVC_ERR_BAD_SHAPE;
    if ((d->head_dim != 64 && d->head_dim != 128) || (d->type != REGENVC_BF16 && d->type != REGENVC_F16)) return REGENVC_ERR_UNSUPPORTED;
    const double scale = d->scale > 0.0f ? (double)d->scale : 1.0 / std::sqrt((double)d->head_dim);
    const float scale_log2 = (float)(scale * 1.4426950408889634);
    if (!(d->scale >= 0.0f) || !std::isfinite(scale_log2)) return REGENVC_ERR_UNSUPPORTED;
    Span lists[3];
    long long table_stride = d->table_stride;
    int rc = lists_ok(d->n_sequences, d->page_size, d->n_pages, d->pages_per_sequence, &table_stride, row_starts, lengths, block_table, lists);
    if (rc != REGENVC_OK) return rc;
    if (d->page_size % 8 != 0) return REGENVC_ERR_UNSUPPORTED;
    bool vec = true;
    HeadView in, res;
    rc = view_of(q, d->q_token_stride, d->q_head_stride, d->n_tokens, d->n_q_heads, d->head_dim, 2, &in, &vec);
    if (rc == REGENVC_OK) rc = view_of(out, d->out_token_stride, d->out_head_stride, d->n_tokens, d->n_q_heads, d->head_dim, 2, &res, &vec);
    if (rc != REGENVC_OK) return rc;
    CacheView cache[2];
    rc = cache_of(k_cache, d->k_page_stride, d->k_slot_stride, d->k_head_stride, d->n_pages, d->page_size, d->n_k_heads, d->head_dim, 2, &cache[0]);
    if (rc == REGENVC_OK)
        rc = cache_of(v_cache, d->v_page_stride, d->v_slot_stride, d->v_head_stride, d->n_pages, d->page_size, d->n_k_heads, d->head_dim, 2, &cache[1]);
    if (rc != REGENVC_OK) return rc;
    for (const CacheView& c : cache)
        if (!aligned(c.span.p, 16) || c.page % 8 != 0 || c.slot % 8 != 0 || c.head % 8 != 0) vec = false;
    if (!vec || !aligned(lse, 4)) return REGENVC_ERR_MISALIGNED;
    const size_t need = paged_attn_workspace_bytes(d->head_dim);
    if (workspace_bytes < need || !aligned(workspace, 16)) return REGENVC_ERR_WORKSPACE;
    const Span ws{workspace, need}, ls{lse, lse ? (size_t)d->n_tokens * d->n_q_heads * 4 : 0};
    const Span reads[6] = {in.span, cache[0].span, cache[1].span, lists[0], lists[1], lists[2]};
    for (const Span& s : reads)
        if (meet(res.span, s) || meet(ls, s) || meet(ws, s)) return REGENVC_ERR_ALIASING;
    if (meet(res.span, ls) || meet(res.span, ws) || meet(ls, ws)) return REGENVC_ERR_ALIASING;

    PagedAttnParams p{};
    p.q = q;
    p.out = out;
    p.lse = reinterpret_cast<float*>(lse);
    p.q_token = in.token;
    p.q_head = in.head;
    p.out_token = res.token;
    p.out_head = res.head;
    p.row_starts = reinterpret_cast<const int*>(row_starts);
    p.lengths = reinterpret_cast<const int*>(lengths);
    p.table = reinterpret_cast<const int*>(block_table);
    p.table_stride = table_stride;
    p.n_tokens = d->n_tokens;
    p.n_sequences = d->n_sequences;
    p.n_q_heads = d->n_q_heads;
    p.n_k_heads = d->n_k_heads;
    p.share = d->n_q_heads / d->n_k_heads;
    p.page_size = d->page_size;
    p.n_pages = d->n_pages;
    p.pages_per_sequence = d->pages_per_sequence;
    p.group = d->group;
    p.window = d->window;
    p.scale_log2 = scale_log2;
    // A tile of 128 keys comes in boxes of as many rows as divide a page; one that lies within a page in one box.
    p.box_rows = 128;
    while (d->page_size % p.box_rows != 0) p.box_rows /= 2;
    p.one_page_box = p.box_rows < 128 && d->page_size >= 128;
    char* w = reinterpret_cast<char*>(workspace);
    p.part_o = reinterpret_cast<float4*>(w);
    w += (size_t)kPagedMaxGrid * 2 * kPagedRows * d->head_dim * sizeof(float);
    p.part_ml = reinterpret_cast<float2*>(w);
    w += (size_t)kPagedMaxGrid * 2 * kPagedRows * sizeof(float2);
    p.pieces = reinterpret_cast<PagedPiece*>(w);
    int sm_count = 0;
    rc = op_device(&sm_count, &p.status);
    if (rc != REGENVC_OK) return rc;
    // Whole items in rounds where several tiles of rows share a head's keys and there can be an item for every thread block; calls
    // of few rows per sequence have nothing to share (a batch of 9 chunks and single tokens: 216 us with one round, 233 without).
    // A sequence's last item may hold one row, so these are as many items as the rows can make (planning for rounds where there
    // are too few for one takes longer: 132 items over 4096 keys 95 us, 101 when planned so).
    const long long rows = (long long)d->n_tokens * p.share, most_items = (rows + (kPagedRows - 1ll) * d->n_sequences) / kPagedRows * d->n_k_heads;
    p.rounds = rows >= 64ll * d->n_sequences && most_items >= paged_attn_grid(sm_count);
    PagedMaps maps;
    const CUtensorMapDataType type = d->type == REGENVC_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    CUtensorMap* small[2] = {&maps.k, &maps.v};
    CUtensorMap* large[2] = {&maps.k_page, &maps.v_page};
    for (int i = 0; i < 2; ++i) {
        const uint64_t extent[4] = {(uint64_t)d->head_dim, (uint64_t)d->page_size, (uint64_t)d->n_k_heads, (uint64_t)d->n_pages};
        const uint64_t stride[3] = {(uint64_t)cache[i].slot * 2, (uint64_t)cache[i].head * 2, (uint64_t)cache[i].page * 2};
        const uint32_t box[4] = {64, (uint32_t)p.box_rows, 1, 1}, page_box[4] = {64, 128, 1, 1};
        void* base = const_cast<void*>(cache[i].span.p);
        rc = encode_map_4d(small[i], type, base, extent, stride, box, CU_TENSOR_MAP_SWIZZLE_128B);
        if (rc == REGENVC_OK && p.one_page_box) rc = encode_map_4d(large[i], type, base, extent, stride, page_box, CU_TENSOR_MAP_SWIZZLE_128B);
        if (rc != REGENVC_OK) return rc;
        if (!p.one_page_box) *large[i] = *small[i];
    }
    int launches = 0;
    const cudaError_t e = launch_paged_attn(maps, p, d->head_dim, d->type == REGENVC_F16, sm_count, &launches, (cudaStream_t)stream);
    return launch_done(e, "launch of the attention over a paged cache", launches);
}

}  // extern "C"
