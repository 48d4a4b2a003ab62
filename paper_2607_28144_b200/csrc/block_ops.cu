// Entry points of the operators around a block's attention: norms fused with gate and residual scale, rotation by
// explicit positions, microscaled 4-bit matrices.  Arguments are checked before any CUDA call; nothing is allocated.
#include "block_norm.cuh"
#include "mxfp4.cuh"
#include "op_checks.cuh"
#include "rope_axes.cuh"

namespace {

using namespace regenvc;

// ------------------------------------------------------------------------------------------------ block norm
struct NormArgs {
    BlockNormParams p;
    long long mods;
    bool vec;
};

int norm_common(const regenvc_block_norm_desc* d, NormArgs* a) {
    if (!d) return REGENVC_ERR_NULL_POINTER;
    if (d->n_tokens < 1 || d->n_tokens > (1 << 30) || d->channels < 1 || d->channels > kNormMaxChannels ||
        d->tokens_per_mod < 1)
        return REGENVC_ERR_BAD_SHAPE;
    if (!type_ok(d->x_type) || !type_ok(d->io_type) || (d->x_type != REGENVC_F32 && d->x_type != d->io_type))
        return REGENVC_ERR_UNSUPPORTED;
    if (d->norm < 0 || d->norm > 2 || d->post_norm < 0 || d->post_norm > 2) return REGENVC_ERR_UNSUPPORTED;
    if (!(d->eps >= 0.0f) || !std::isfinite(d->eps) || !(d->post_eps >= 0.0f) || !std::isfinite(d->post_eps) ||
        !std::isfinite(d->residual_scale))
        return REGENVC_ERR_UNSUPPORTED;
    BlockNormParams& p = a->p;
    p = BlockNormParams{};
    p.n_tokens = d->n_tokens;
    p.channels = d->channels;
    p.tokens_per_mod = d->tokens_per_mod < d->n_tokens ? d->tokens_per_mod : d->n_tokens;
    a->mods = ((long long)p.n_tokens + p.tokens_per_mod - 1) / p.tokens_per_mod;
    p.norm = d->norm;
    p.post_norm = d->post_norm;
    p.eps = d->eps;
    p.post_eps = d->post_eps;
    p.residual_scale = d->residual_scale;
    const long long given[8] = {d->mod_stride, d->x_stride, d->y_stride, d->x_out_stride, d->h_stride, d->dx_out_stride,
                                d->dx_stride, d->dy_stride};
    long long* use[8] = {&p.mod_stride, &p.x_stride, &p.y_stride, &p.x_out_stride, &p.h_stride, &p.dx_out_stride,
                         &p.dx_stride, &p.dy_stride};
    a->vec = p.channels % 8 == 0;
    for (int i = 0; i < 8; ++i) {
        if (given[i] != 0 && (given[i] < p.channels || given[i] > kMaxStride)) return REGENVC_ERR_BAD_SHAPE;
        *use[i] = given[i] != 0 ? given[i] : p.channels;
        if (*use[i] % 8 != 0) a->vec = false;
    }
    return REGENVC_OK;
}

// Alignment and overlap: outs[i] may coincide with in_place[i] exactly (same address and stride checked by the caller).
int norm_memory(NormArgs* a, const Span* ins, const size_t* in_size, int n_in, const Span* outs, const size_t* out_size,
                int n_out, const int* in_place) {
    for (int i = 0; i < n_in; ++i) {
        if (!aligned(ins[i].p, in_size[i])) return REGENVC_ERR_MISALIGNED;
        if (!aligned(ins[i].p, 16)) a->vec = false;
    }
    for (int i = 0; i < n_out; ++i) {
        if (!aligned(outs[i].p, out_size[i])) return REGENVC_ERR_MISALIGNED;
        if (!aligned(outs[i].p, 16)) a->vec = false;
    }
    for (int i = 0; i < n_out; ++i) {
        for (int j = 0; j < n_in; ++j)
            if (j != in_place[i] && meet(outs[i], ins[j])) return REGENVC_ERR_ALIASING;
        for (int j = 0; j < i; ++j)
            if (meet(outs[i], outs[j])) return REGENVC_ERR_ALIASING;
    }
    return REGENVC_OK;
}

// ------------------------------------------------------------------------------------------------ 4-bit matrices
bool mx_shape_ok(int rows, int cols) {
    if (rows < 1 || cols < 1 || rows > (1 << 30) || cols > (1 << 24)) return false;
    return MxLayout(rows, cols).scale_tiles() < (1ll << 30);   // tile numbers are 32-bit coordinates
}

int mx_convert(const void* values, int type, int rows, int cols, long long row_stride, const void* packed, bool quantize,
               cudaStream_t stream) {
    if (!values || !packed) return REGENVC_ERR_NULL_POINTER;
    if (!mx_shape_ok(rows, cols) || (row_stride != 0 && (row_stride < cols || row_stride > kMaxStride)))
        return REGENVC_ERR_BAD_SHAPE;
    if (!type_ok(type)) return REGENVC_ERR_UNSUPPORTED;
    if (!aligned(values, type_size(type)) || !aligned(packed, 256)) return REGENVC_ERR_MISALIGNED;
    MxConvertParams p{};
    p.rows = rows;
    p.cols = cols;
    p.row_stride = row_stride ? row_stride : cols;
    const Span v = rows_span(values, rows, p.row_stride, cols, type_size(type));
    const Span k{packed, (size_t)MxLayout(rows, cols).bytes};
    if (meet(v, k)) return REGENVC_ERR_ALIASING;
    const size_t step = (size_t)p.row_stride * type_size(type);
    p.vec = aligned(values, 32) && step % 32 == 0 ? 2 : (aligned(values, 16) && step % 16 == 0 ? 1 : 0);
    p.src = quantize ? values : packed;
    p.dst = const_cast<void*>(quantize ? packed : values);
    int sm_count = 0, *status = nullptr;
    const int rc = op_device(&sm_count, &status);
    if (rc != REGENVC_OK) return rc;
    const cudaError_t e = quantize ? launch_mxfp4_quantize(p, type, sm_count, stream) : launch_mxfp4_dequantize(p, type, sm_count, stream);
    return launch_done(e, quantize ? "launch of the 4-bit quantisation" : "launch of the 4-bit expansion", e == cudaSuccess ? 1 : 0);
}

int mx_project_checks(const void* w, const void* bias, const void* y, int y_type, int n, int features, int cols) {
    if (!w || !y) return REGENVC_ERR_NULL_POINTER;
    if (!mx_shape_ok(n, cols) || !mx_shape_ok(features, cols)) return REGENVC_ERR_BAD_SHAPE;
    if (((long long)n + 127) / 128 * (((long long)features + 63) / 64) >= (1ll << 31)) return REGENVC_ERR_BAD_SHAPE;
    if (features % 8 != 0 || (y_type != REGENVC_BF16 && y_type != REGENVC_F16)) return REGENVC_ERR_UNSUPPORTED;
    if (!aligned(w, 256) || !aligned(y, 16) || !aligned(bias, 4)) return REGENVC_ERR_MISALIGNED;
    const Span ys{y, (size_t)n * features * 2}, ws{w, (size_t)MxLayout(features, cols).bytes}, bs{bias, (size_t)features * 4};
    if (meet(ys, ws) || meet(ys, bs)) return REGENVC_ERR_ALIASING;
    return REGENVC_OK;
}

int mx_project(const void* x, const void* w, const void* bias, void* y, int y_type, int n, int features, int cols,
               bool early, int sm_count, int* status, cudaStream_t stream) {
    const MxLayout lx(n, cols), lw(features, cols);
    const MxProjectPlan plan = plan_mxfp4_project(n, features, cols, sm_count);
    CUtensorMap mx, mxs, mw, mws, my;
    char* xb = reinterpret_cast<char*>(const_cast<void*>(x));
    char* wb = reinterpret_cast<char*>(const_cast<void*>(w));
    const CUtensorMapDataType u8 = CU_TENSOR_MAP_DATA_TYPE_UINT8, u32 = CU_TENSOR_MAP_DATA_TYPE_UINT32;
    const CUtensorMapSwizzle sw = CU_TENSOR_MAP_SWIZZLE_128B, plain = CU_TENSOR_MAP_SWIZZLE_NONE;
    const uint64_t rb = (uint64_t)lx.cols_pad / 2;
    int rc = encode_map(&mx, u8, xb, rb, (uint64_t)n, rb, 128, 128, sw);
    if (rc == REGENVC_OK) rc = encode_map(&mw, u8, wb, rb, (uint64_t)features, rb, 128, (uint32_t)plan.w_box_rows, sw);
    // scales: rows of one 512-byte tile; a load takes the two tiles of 256 columns
    if (rc == REGENVC_OK) rc = encode_map(&mxs, u32, xb + lx.scale_at, 128, (uint64_t)lx.scale_tiles(), 512, 128, 2, plain);
    if (rc == REGENVC_OK) rc = encode_map(&mws, u32, wb + lw.scale_at, 128, (uint64_t)lw.scale_tiles(), 512, 128, 2, plain);
    if (rc == REGENVC_OK)
        rc = encode_map(&my, y_type == REGENVC_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, y,
                        (uint64_t)features, (uint64_t)n, (uint64_t)features * 2, 64, 128, sw);
    if (rc != REGENVC_OK) return rc;
    MxProjectParams p{};
    p.bias = reinterpret_cast<const float*>(bias);
    p.n_tokens = n;
    p.features = features;
    p.k_blocks = (int)(lx.cols_pad / 128);
    p.y_f16 = y_type == REGENVC_F16;
    p.status = status;
    const cudaError_t e = launch_mxfp4_project(plan, mx, mxs, mw, mws, my, p, early, sm_count, stream);
    return launch_done(e, "launch of the 4-bit product", e == cudaSuccess ? 1 : 0);
}

// Few tokens: one launch, from x itself (type) or from its packed form (x_stride < 0).
int mx_rows(const void* x, int type, long long x_stride, const void* w, const void* bias, void* y, int y_type, int n,
            int features, int cols, int sm_count, cudaStream_t stream) {
    const MxLayout lx(n, cols), lw(features, cols);
    const bool packed = x_stride < 0;
    MxRowsParams p{};
    p.x = x;
    p.x_stride = x_stride ? x_stride : cols;
    p.w = reinterpret_cast<const uint8_t*>(w);
    p.bias = reinterpret_cast<const float*>(bias);
    p.y = y;
    p.cols_pad = lx.cols_pad;
    p.x_scale_at = lx.scale_at;
    p.w_scale_at = lw.scale_at;
    p.n_tokens = n;
    p.features = features;
    p.cols = cols;
    p.vec = !packed && aligned(x, 16) && p.x_stride % 8 == 0;
    p.y_f16 = y_type == REGENVC_F16;
    const cudaError_t e = launch_mxfp4_rows(p, type, packed, sm_count, stream);
    return launch_done(e, "launch of the 4-bit product of a few rows", e == cudaSuccess ? 1 : 0);
}

}  // namespace

extern "C" {

int regenvc_block_norm_forward(const regenvc_block_norm_desc* desc, const void* x, const void* y, const void* gate,
                               const void* post_weight, const void* weight, const void* bias, const void* scale,
                               const void* shift, void* x_out, void* h, void* stream) {
    NormArgs a;
    int rc = norm_common(desc, &a);
    if (rc != REGENVC_OK) return rc;
    BlockNormParams& p = a.p;
    if (!x || (!h) != (p.norm == REGENVC_NORM_NONE) || (!x_out && !h)) return REGENVC_ERR_NULL_POINTER;
    if (!y && (x_out || gate || post_weight || p.post_norm != REGENVC_NORM_NONE)) return REGENVC_ERR_NULL_POINTER;
    const size_t xs = type_size(desc->x_type), is = type_size(desc->io_type);
    const long long n = p.n_tokens, c = p.channels;
    const Span ins[8] = {rows_span(x, n, p.x_stride, c, xs), rows_span(y, n, p.y_stride, c, is),
                         rows_span(gate, a.mods, p.mod_stride, c, 4), rows_span(scale, a.mods, p.mod_stride, c, 4),
                         rows_span(shift, a.mods, p.mod_stride, c, 4), rows_span(post_weight, 1, c, c, 4),
                         rows_span(weight, 1, c, c, 4), rows_span(bias, 1, c, c, 4)};
    const size_t in_size[8] = {xs, is, 4, 4, 4, 4, 4, 4};
    const Span outs[2] = {rows_span(x_out, n, p.x_out_stride, c, xs), rows_span(h, n, p.h_stride, c, is)};
    const size_t out_size[2] = {xs, is};
    const int in_place[2] = {x_out == x && p.x_out_stride == p.x_stride ? 0 : -1, -1};
    rc = norm_memory(&a, ins, in_size, 8, outs, out_size, 2, in_place);
    if (rc != REGENVC_OK) return rc;
    p.x = x;
    p.y = y;
    p.gate = reinterpret_cast<const float*>(gate);
    p.post_weight = reinterpret_cast<const float*>(post_weight);
    p.weight = reinterpret_cast<const float*>(weight);
    p.bias = reinterpret_cast<const float*>(bias);
    p.scale = reinterpret_cast<const float*>(scale);
    p.shift = reinterpret_cast<const float*>(shift);
    p.x_out = x_out;
    p.h = h;
    int sm_count = 0, *status = nullptr;
    rc = op_device(&sm_count, &status);
    if (rc != REGENVC_OK) return rc;
    const cudaError_t e = launch_block_norm_forward(p, desc->x_type, desc->io_type, a.vec, sm_count, (cudaStream_t)stream);
    return launch_done(e, "launch of the block norm", e == cudaSuccess ? 1 : 0);
}

size_t regenvc_block_norm_workspace_bytes(int n_tokens, int channels) {
    if (n_tokens < 1 || channels < 1 || channels > kNormMaxChannels) return 0;
    return block_norm_workspace_bytes(n_tokens, channels);
}

int regenvc_block_norm_backward(const regenvc_block_norm_desc* desc, const void* x_out, const void* y, const void* gate,
                                const void* post_weight, const void* weight, const void* bias, const void* scale,
                                const void* dh, const void* dx_out, void* dx, void* dy, void* dgate, void* dpost_weight,
                                void* dweight, void* dbias, void* dscale, void* dshift, void* workspace,
                                size_t workspace_bytes, void* stream) {
    NormArgs a;
    int rc = norm_common(desc, &a);
    if (rc != REGENVC_OK) return rc;
    BlockNormParams& p = a.p;
    if ((!dh) != (p.norm == REGENVC_NORM_NONE) || (dh && !x_out) || !workspace) return REGENVC_ERR_NULL_POINTER;
    if (!dh && (dweight || dbias || dscale || dshift)) return REGENVC_ERR_NULL_POINTER;
    if (!dh && !dx_out) return REGENVC_ERR_NULL_POINTER;
    if (!y && (dy || gate || dgate || post_weight || dpost_weight || p.post_norm != REGENVC_NORM_NONE)) return REGENVC_ERR_NULL_POINTER;
    if ((dgate && !gate) || (dpost_weight && !post_weight) || (dweight && !weight) || (dscale && !scale))
        return REGENVC_ERR_NULL_POINTER;
    if (!dx && !dy && !dgate && !dpost_weight && !dweight && !dbias && !dscale && !dshift) return REGENVC_ERR_NULL_POINTER;
    if (workspace_bytes < block_norm_workspace_bytes(p.n_tokens, p.channels) || !aligned(workspace, 16)) return REGENVC_ERR_WORKSPACE;
    if (!y) p.residual_scale = 1.0f;
    const size_t xs = type_size(desc->x_type), is = type_size(desc->io_type);
    const long long n = p.n_tokens, c = p.channels;
    const Span ins[9] = {rows_span(dx_out, n, p.dx_out_stride, c, xs), rows_span(dh ? x_out : nullptr, n, p.x_out_stride, c, xs),
                         rows_span(y, n, p.y_stride, c, is), rows_span(dh, n, p.h_stride, c, is),
                         rows_span(gate, a.mods, p.mod_stride, c, 4), rows_span(scale, a.mods, p.mod_stride, c, 4),
                         rows_span(post_weight, 1, c, c, 4), rows_span(weight, 1, c, c, 4), rows_span(bias, 1, c, c, 4)};
    const size_t in_size[9] = {xs, xs, is, is, 4, 4, 4, 4, 4};
    const Span outs[9] = {rows_span(dx, n, p.dx_stride, c, xs), rows_span(dy, n, p.dy_stride, c, is),
                          rows_span(dgate, a.mods, c, c, 4), rows_span(dscale, a.mods, c, c, 4), rows_span(dshift, a.mods, c, c, 4),
                          rows_span(dpost_weight, 1, c, c, 4), rows_span(dweight, 1, c, c, 4), rows_span(dbias, 1, c, c, 4),
                          Span{workspace, block_norm_workspace_bytes(n, c)}};
    const size_t out_size[9] = {xs, is, 4, 4, 4, 4, 4, 4, 16};
    int in_place[9] = {-1, -1, -1, -1, -1, -1, -1, -1, -1};
    if (dx && dx == dx_out && p.dx_stride == p.dx_out_stride) in_place[0] = 0;
    rc = norm_memory(&a, ins, in_size, 9, outs, out_size, 9, in_place);
    if (rc != REGENVC_OK) return rc;
    p.x = x_out;
    p.x_stride = p.x_out_stride;   // the kernel's x is the saved x'
    p.y = y;
    p.gate = reinterpret_cast<const float*>(gate);
    p.post_weight = reinterpret_cast<const float*>(post_weight);
    p.weight = reinterpret_cast<const float*>(weight);
    p.bias = reinterpret_cast<const float*>(bias);
    p.scale = reinterpret_cast<const float*>(scale);
    p.dh = dh;
    p.dx_out = dx_out;
    p.dx = dx;
    p.dy = dy;
    p.dgate = reinterpret_cast<float*>(dgate);
    p.dpost_weight = reinterpret_cast<float*>(dpost_weight);
    p.dweight = reinterpret_cast<float*>(dweight);
    p.dbias = reinterpret_cast<float*>(dbias);
    p.dscale = reinterpret_cast<float*>(dscale);
    p.dshift = reinterpret_cast<float*>(dshift);
    p.partials = reinterpret_cast<float*>(workspace);
    int sm_count = 0, *status = nullptr, launches = 0;
    rc = op_device(&sm_count, &status);
    if (rc != REGENVC_OK) return rc;
    const cudaError_t e = launch_block_norm_backward(p, desc->x_type, desc->io_type, a.vec, sm_count, &launches, (cudaStream_t)stream);
    return launch_done(e, "launch of the block norm's gradients", launches);
}

int regenvc_rope_axes(const regenvc_rope_axes_desc* d, const void* q, const void* k, const void* positions, void* q_out,
                      void* k_out, void* stream) {
    if (!d || !q || !q_out || !positions) return REGENVC_ERR_NULL_POINTER;
    if (d->n_k_heads < 0 || d->n_tokens < 1 || d->n_tokens > (1 << 30) || d->n_q_heads < 1 || d->n_q_heads > 65535 ||
        d->n_k_heads > 65535 || d->head_dim < 2 || d->head_dim > 2 * kRopeMaxPairs || d->n_axes < 1 || d->n_axes > kRopeMaxAxes)
        return REGENVC_ERR_BAD_SHAPE;
    if ((!k || !k_out) != (d->n_k_heads == 0) || (!k) != (!k_out)) return REGENVC_ERR_NULL_POINTER;
    if (d->head_dim % 2 != 0 || !type_ok(d->type)) return REGENVC_ERR_UNSUPPORTED;
    if (!(d->rope_theta > 0.0f) || !std::isfinite(d->rope_theta)) return REGENVC_ERR_UNSUPPORTED;
    if ((d->halves | d->whole_ladder | d->pos_float | d->inverse) & ~1) return REGENVC_ERR_UNSUPPORTED;
    RopeAxesParams p{};
    long long rotated = 0;
    for (int a = 0; a < d->n_axes; ++a) {
        if (d->widths[a] < 2 || d->widths[a] % 2 != 0 || d->widths[a] > d->head_dim) return REGENVC_ERR_BAD_SHAPE;
        rotated += d->widths[a];
        if (rotated > d->head_dim) return REGENVC_ERR_BAD_SHAPE;
        p.axis_end[a] = (int)(rotated / 2);
    }
    p.n_pairs = (int)(rotated / 2);
    p.n_tokens = d->n_tokens;
    p.head_dim = d->head_dim;
    p.n_axes = d->n_axes;
    p.heads[0] = d->n_q_heads;
    p.heads[1] = d->n_k_heads;
    p.positions = positions;
    p.pos_stride = d->pos_stride ? d->pos_stride : d->n_tokens;
    if (p.pos_stride < d->n_tokens || p.pos_stride > kMaxStride) return REGENVC_ERR_BAD_SHAPE;
    p.pos_float = d->pos_float;
    p.inverse = d->inverse;
    p.halves = d->halves;
    const size_t size = type_size(d->type);
    const void* ptr[4] = {q, k, q_out, k_out};
    const long long token[4] = {d->q_token_stride, d->k_token_stride, d->q_out_token_stride, d->k_out_token_stride};
    const long long head[4] = {d->q_head_stride, d->k_head_stride, d->q_out_head_stride, d->k_out_head_stride};
    long long ts[4], hs[4];
    Span span[4] = {};
    bool vec = true;
    for (int i = 0; i < 4; ++i) {
        const int heads = p.heads[i & 1];
        hs[i] = head[i] ? head[i] : d->head_dim;
        ts[i] = token[i] ? token[i] : (long long)heads * d->head_dim;
        if (!ptr[i]) continue;
        // elements of different (token, head) pairs do not share memory: one of the two strides clears the other's extent
        if (hs[i] < d->head_dim || hs[i] > kMaxStride || ts[i] < d->head_dim || ts[i] > kMaxStride) return REGENVC_ERR_BAD_SHAPE;
        const bool tokens_outside = ts[i] >= (heads - 1) * hs[i] + d->head_dim;
        const bool heads_outside = hs[i] >= (long long)(d->n_tokens - 1) * ts[i] + d->head_dim;
        if (!tokens_outside && !heads_outside) return REGENVC_ERR_BAD_SHAPE;
        if (!aligned(ptr[i], size)) return REGENVC_ERR_MISALIGNED;
        if (!aligned(ptr[i], 16) || hs[i] % 8 != 0 || ts[i] % 8 != 0) vec = false;
        span[i] = Span{ptr[i], ((size_t)(d->n_tokens - 1) * ts[i] + (size_t)(heads - 1) * hs[i] + d->head_dim) * size};
    }
    if (!aligned(positions, 4)) return REGENVC_ERR_MISALIGNED;
    const Span pos{positions, ((size_t)(d->n_axes - 1) * p.pos_stride + d->n_tokens) * 4};
    // Views of one fused tensor interleave: q and k (both read, or both written) may cover the same stretch of memory.
    // A result is either its operand itself or clear of both operands' memory -- except that when q and k are both
    // rotated in place, q's stretch may interleave with k's.
    bool same[2];
    for (int w = 0; w < 2; ++w) {
        same[w] = ptr[w] && ptr[w] == ptr[w + 2] && ts[w] == ts[w + 2] && hs[w] == hs[w + 2];
        if (meet(span[w + 2], pos)) return REGENVC_ERR_ALIASING;
        if (!same[w] && meet(span[w + 2], span[w])) return REGENVC_ERR_ALIASING;
        p.in[w] = ptr[w];
        p.out[w] = const_cast<void*>(ptr[w + 2]);
        p.in_token[w] = ts[w];
        p.in_head[w] = hs[w];
        p.out_token[w] = ts[w + 2];
        p.out_head[w] = hs[w + 2];
    }
    if (k) {
        // the (token, head) vectors of the two tensors must be different ones: true if they lie a whole number of
        // vectors apart inside one token's stride
        auto apart = [&](int i, int j) {
            if (!meet(span[i], span[j])) return true;
            if (ts[i] != ts[j] || hs[i] != hs[j]) return false;
            const char *a = (const char*)ptr[i], *b = (const char*)ptr[j];
            const long long gap = (long long)(a < b ? b - a : a - b) / (long long)size;
            const int low = a < b ? i : j, high = a < b ? j : i;
            const long long low_end = (long long)(p.heads[low & 1] - 1) * hs[i] + d->head_dim;
            const long long high_end = gap + (long long)(p.heads[high & 1] - 1) * hs[i] + d->head_dim;
            return gap >= low_end && high_end <= ts[i];
        };
        if (!apart(2, 3)) return REGENVC_ERR_ALIASING;
        if (!(same[0] && apart(2, 1)) && meet(span[2], span[1])) return REGENVC_ERR_ALIASING;
        if (!(same[1] && apart(3, 0)) && meet(span[3], span[0])) return REGENVC_ERR_ALIASING;
    }
    rope_turns(d->widths, d->n_axes, p.n_pairs, d->whole_ladder != 0, d->rope_theta, p.turns);
    int sm_count = 0, *status = nullptr;
    const int rc = op_device(&sm_count, &status);
    if (rc != REGENVC_OK) return rc;
    const cudaError_t e = launch_rope_axes(p, d->type, vec, sm_count, (cudaStream_t)stream);
    return launch_done(e, "launch of the rotation", e == cudaSuccess ? 1 : 0);
}

size_t regenvc_mxfp4_bytes(int rows, int cols) {
    return mx_shape_ok(rows, cols) ? (size_t)MxLayout(rows, cols).bytes : 0;
}

int regenvc_mxfp4_quantize(const void* src, int type, int rows, int cols, long long row_stride, void* packed, void* stream) {
    return mx_convert(src, type, rows, cols, row_stride, packed, true, (cudaStream_t)stream);
}

int regenvc_mxfp4_dequantize(const void* packed, void* dst, int type, int rows, int cols, long long row_stride,
                             void* stream) {
    return mx_convert(dst, type, rows, cols, row_stride, packed, false, (cudaStream_t)stream);
}

int regenvc_mxfp4_project(const void* x_packed, const void* w_packed, const void* bias, void* y, int y_type, int n_tokens,
                          int out_features, int in_features, void* stream) {
    if (!x_packed) return REGENVC_ERR_NULL_POINTER;
    int rc = mx_project_checks(w_packed, bias, y, y_type, n_tokens, out_features, in_features);
    if (rc != REGENVC_OK) return rc;
    if (!aligned(x_packed, 256)) return REGENVC_ERR_MISALIGNED;
    if (meet(Span{y, (size_t)n_tokens * out_features * 2}, Span{x_packed, (size_t)MxLayout(n_tokens, in_features).bytes}))
        return REGENVC_ERR_ALIASING;
    int sm_count = 0, *status = nullptr;
    rc = op_device(&sm_count, &status);
    if (rc != REGENVC_OK) return rc;
    if (mxfp4_rows_fits(n_tokens, out_features, MxLayout(n_tokens, in_features).cols_pad))
        return mx_rows(x_packed, REGENVC_BF16, -1, w_packed, bias, y, y_type, n_tokens, out_features, in_features, sm_count,
                       (cudaStream_t)stream);
    return mx_project(x_packed, w_packed, bias, y, y_type, n_tokens, out_features, in_features, false, sm_count, status,
                      (cudaStream_t)stream);
}

size_t regenvc_mxfp4_linear_scratch_bytes(int n_tokens, int out_features, int in_features) {
    if (!mx_shape_ok(n_tokens, in_features) || !mx_shape_ok(out_features, in_features)) return 0;
    const MxLayout l(n_tokens, in_features);
    return mxfp4_rows_fits(n_tokens, out_features, l.cols_pad) ? 0 : (size_t)l.bytes;
}

int regenvc_mxfp4_linear(const void* x, int x_type, long long x_stride, const void* w_packed, const void* bias, void* y,
                         int y_type, int n_tokens, int out_features, int in_features, void* scratch, void* stream) {
    if (!x) return REGENVC_ERR_NULL_POINTER;
    int rc = mx_project_checks(w_packed, bias, y, y_type, n_tokens, out_features, in_features);
    if (rc != REGENVC_OK) return rc;
    if (!type_ok(x_type)) return REGENVC_ERR_UNSUPPORTED;
    if (x_stride != 0 && (x_stride < in_features || x_stride > kMaxStride)) return REGENVC_ERR_BAD_SHAPE;
    const bool few = mxfp4_rows_fits(n_tokens, out_features, MxLayout(n_tokens, in_features).cols_pad);
    if (!few && !scratch) return REGENVC_ERR_NULL_POINTER;
    if (!aligned(x, type_size(x_type)) || (!few && !aligned(scratch, 256))) return REGENVC_ERR_MISALIGNED;
    const Span xs = rows_span(x, n_tokens, x_stride ? x_stride : in_features, in_features, type_size(x_type));
    const Span ss{few ? nullptr : scratch, (size_t)MxLayout(n_tokens, in_features).bytes};
    const Span ys{y, (size_t)n_tokens * out_features * 2}, ws{w_packed, (size_t)MxLayout(out_features, in_features).bytes};
    if (meet(ys, xs) || meet(ys, ss) || meet(ss, xs) || meet(ss, ws) || meet(ss, Span{bias, (size_t)out_features * 4}))
        return REGENVC_ERR_ALIASING;
    int sm_count = 0, *status = nullptr;
    rc = op_device(&sm_count, &status);
    if (rc != REGENVC_OK) return rc;
    if (few)
        return mx_rows(x, x_type, x_stride, w_packed, bias, y, y_type, n_tokens, out_features, in_features, sm_count,
                       (cudaStream_t)stream);
    rc = mx_convert(x, x_type, n_tokens, in_features, x_stride, scratch, true, (cudaStream_t)stream);
    if (rc != REGENVC_OK) return rc;
    return mx_project(scratch, w_packed, bias, y, y_type, n_tokens, out_features, in_features, true, sm_count, status,
                      (cudaStream_t)stream);
}

}  // extern "C"
