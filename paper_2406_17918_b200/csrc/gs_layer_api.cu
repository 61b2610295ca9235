// The C ABI of the operators around an attention layer: argument checks and launches.
#include <algorithm>
#include <memory>
#include <new>

#include "gs_train_args.h"

using namespace gs;

namespace {

// Rows [rows][dim] in memory; data NULL: no such operand.
struct RowSpan {
    const void* data;
    int64_t ld;
};

// Whether two of them have elements in common.  Rows of one pitch may lie beside one another; of two pitches they are taken to meet
// where their ranges do.
bool rows_meet(RowSpan a, RowSpan b, int64_t rows, int64_t dim, size_t size) {
    if (!a.data || !b.data) return false;
    if (rows == 1) a.ld = b.ld = dim;
    const uint64_t begin_a = (uint64_t)a.data, begin_b = (uint64_t)b.data, width = (uint64_t)dim * size, last = (uint64_t)rows - 1;
    if (begin_a + last * (uint64_t)a.ld * size + width <= begin_b || begin_b + last * (uint64_t)b.ld * size + width <= begin_a) return false;
    if (a.ld != b.ld) return true;
    const uint64_t pitch = (uint64_t)a.ld * size, off = (begin_a < begin_b ? begin_b - begin_a : begin_a - begin_b) % pitch;
    return off < width || pitch - off < width;
}

gs_status check_norm(const RmsNorm& p, bool backward) {
    if (!known(p.dtype) || (p.weight && !known(p.weight_dtype))) return set_error(GS_ERR_ARG, "unknown dtype");
    if (p.n.bound < 0) return set_error(GS_ERR_ARG, "rows is negative");
    if (p.dim < 1 || p.dim > NORM_MAX_DIM) return set_error(GS_ERR_ARG, "dim %d outside [1, %d]", p.dim, NORM_MAX_DIM);
    if (!(p.eps >= 0.f)) return set_error(GS_ERR_ARG, "eps is negative or NaN");
    const size_t size = size_of(p.dtype);
    if (p.n.bound > 0) {
        if (!p.x || (backward && (!p.dout || !p.out))) return set_error(GS_ERR_ARG, "NULL argument");
        if (p.x_ld < p.dim || (p.residual && p.residual_ld < p.dim) || (p.hidden && p.hidden_ld < p.dim) || (p.out && p.out_ld < p.dim) || (p.dout && p.dout_ld < p.dim))
            return set_error(GS_ERR_ARG, "a row pitch is smaller than dim");
    }
    if (!aligned_to(p.x, size) || !aligned_to(p.residual, size) || !aligned_to(p.hidden, size) || !aligned_to(p.out, size) || !aligned_to(p.dout, size) ||
        (p.weight && !aligned_to(p.weight, size_of(p.weight_dtype))) || (p.dweight && !aligned_to(p.dweight, size_of(p.weight_dtype))) || !aligned_to(p.n.d_n, 4))
        return set_error(GS_ERR_ALIGN, "misaligned argument");
    if (p.n.bound > 0) {
        // a row is written by the threads that have read it: a result may be an operand's array, but lie across none
        const RowSpan results[] = {{p.hidden, p.hidden_ld}, {p.out, p.out_ld}}, operands[] = {{p.x, p.x_ld}, {p.residual, p.residual_ld}, {p.dout, p.dout_ld}};
        if (rows_meet(results[0], results[1], p.n.bound, p.dim, size)) return set_error(GS_ERR_ARG, "hidden and out overlap");
        for (const RowSpan& r : results)
            for (const RowSpan& o : operands)
                if (rows_meet(r, o, p.n.bound, p.dim, size) && (r.data != o.data || (p.n.bound > 1 && r.ld != o.ld)))
                    return set_error(GS_ERR_ARG, "a result overlaps an operand without being its array");
    }
    return GS_OK;
}

gs_status check_coded(const char* name, const gs_coded* c, CodedView* out) {
    if (!c) return set_error(GS_ERR_ARG, "%s is NULL", name);
    if (c->rows < 0 || c->rows >= ((int64_t)1 << 31)) return set_error(GS_ERR_ARG, "%s: rows outside [0, 2^31)", name);
    if (c->heads < 1 || c->heads > (1 << 16) || c->head_dim < 1 || c->head_dim > (1 << 16)) return set_error(GS_ERR_ARG, "%s: heads or head_dim outside [1, 2^16]", name);
    if (c->block < 1 || c->block > 64 || (c->block & (c->block - 1))) return set_error(GS_ERR_ARG, "%s: block %d is not a power of two from 1 to 64", name, c->block);
    const int32_t pitch = (c->head_dim + 15) / 16 * 16;
    if ((int64_t)c->heads * pitch >= ((int64_t)1 << 30)) return set_error(GS_ERR_ARG, "%s: a row has 2^30 bytes or more", name);
    if (c->rows > 0 && (!c->d_codes || !c->d_scales)) return set_error(GS_ERR_ARG, "%s has no arrays", name);
    if (c->row_stride % 16 || (c->rows > 1 && c->row_stride < (int64_t)c->heads * pitch)) return set_error(GS_ERR_ARG, "%s: row_stride is no multiple of 16, or too small", name);
    if (c->rows > c->block && c->scale_stride < c->heads) return set_error(GS_ERR_ARG, "%s: scale_stride is too small", name);
    if (c->row_stride < 0 || c->row_stride >= ((int64_t)1 << 32) || c->scale_stride < 0 || c->scale_stride >= ((int64_t)1 << 32))
        return set_error(GS_ERR_ARG, "%s: a stride is negative, or 4 GB or more", name);
    if (!aligned_to(c->d_codes, 16)) return set_error(GS_ERR_ALIGN, "%s: the codes are not 16-byte aligned", name);
    int shift = 0;
    while ((1 << shift) < c->block) ++shift;
    *out = CodedView{(uint8_t*)c->d_codes, c->d_scales, c->rows, c->row_stride, c->scale_stride, c->heads, c->head_dim, pitch, shift};
    return GS_OK;
}

gs_status check_list(const int32_t* ids, int64_t first, const int32_t* count, int32_t bound, int64_t rows) {
    if (bound < 0) return set_error(GS_ERR_ARG, "count_bound is negative");
    if (!ids && (first < 0 || first + bound > rows)) return set_error(GS_ERR_ARG, "the range of rows is not inside the store");
    if (!aligned_to(ids, 4) || !aligned_to(count, 4)) return set_error(GS_ERR_ALIGN, "misaligned argument");
    return GS_OK;
}

struct Range {
    uintptr_t begin, end;
    int32_t i;
};

gs_status grads(const gs_grad* g, int32_t n, bool clip, float max_norm, float* norm, void* ws, size_t ws_bytes, cudaStream_t s) {
    if (n < 0 || n > (1 << 16)) return set_error(GS_ERR_ARG, "n outside [0, 65536]");
    if ((n > 0 && !g) || (!clip && !norm)) return set_error(GS_ERR_ARG, "NULL argument");
    if (clip && !(max_norm >= 0.f)) return set_error(GS_ERR_ARG, "max_norm is negative or NaN");
    if (!aligned_to(norm, 4)) return set_error(GS_ERR_ALIGN, "d_norm is misaligned");
    const std::unique_ptr<GradTensor[]> list(new (std::nothrow) GradTensor[n + 1]);
    const std::unique_ptr<Range[]> outs(new (std::nothrow) Range[n + 1]);
    if (!list || !outs) return set_error(GS_ERR_ARG, "no host memory for %d gradients", n);
    int32_t kept = 0;
    int64_t total = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (!known(g[i].dtype)) return set_error(GS_ERR_ARG, "gradient %d: unknown dtype", i);
        if (g[i].elems < 0 || g[i].elems > ((int64_t)1 << 42)) return set_error(GS_ERR_ARG, "gradient %d: elems out of range", i);
        if (g[i].elems == 0) continue;
        if (!g[i].d_grad || (clip && !g[i].d_out)) return set_error(GS_ERR_ARG, "gradient %d is NULL", i);
        if (g[i].d_rows_or_null && (g[i].row_elems < 1 || g[i].row_elems > g[i].elems)) return set_error(GS_ERR_ARG, "gradient %d: row_elems out of range", i);
        const size_t size = size_of(g[i].dtype);
        if (!aligned_to(g[i].d_grad, size) || (clip && !aligned_to(g[i].d_out, size)) || !aligned_to(g[i].d_rows_or_null, 4)) return set_error(GS_ERR_ALIGN, "gradient %d is misaligned", i);
        total += g[i].elems;
        list[kept] = GradTensor{g[i].d_grad, clip ? g[i].d_out : nullptr, g[i].d_rows_or_null, g[i].elems, g[i].row_elems, g[i].dtype, 0};
        outs[kept] = Range{(uintptr_t)g[i].d_out, (uintptr_t)g[i].d_out + (uintptr_t)g[i].elems * size, kept};
        ++kept;
    }
    if (total > ((int64_t)1 << 42)) return set_error(GS_ERR_ARG, "the gradients have too many elements");
    if (clip) {
        // every number is written by one thread and read by none but that one
        std::sort(outs.get(), outs.get() + kept, [](const Range& a, const Range& b) { return a.begin < b.begin; });
        for (int32_t i = 1; i < kept; ++i)
            if (outs[i].begin < outs[i - 1].end) return set_error(GS_ERR_ARG, "the results of two gradients overlap (is one listed twice?)");
        for (int32_t i = 0; i < kept; ++i) {
            const uintptr_t begin = (uintptr_t)list[i].grad, end = begin + (uintptr_t)list[i].elems * size_of(list[i].dtype);
            const Range* o = std::lower_bound(outs.get(), outs.get() + kept, begin, [](const Range& a, uintptr_t b) { return a.end <= b; });
            for (; o < outs.get() + kept && o->begin < end; ++o)
                if (o->i != i || o->begin != begin) return set_error(GS_ERR_ARG, "a result overlaps another gradient, or its own without being it");
        }
    }
    GS_TRY(check_workspace(ws, ws_bytes, grad_workspace(n)));
    GS_TRAIN_CUDA(launch_grad_norm(list.get(), kept, clip, max_norm, norm, ws, s));
    return GS_OK;
}

}  // namespace

extern "C" {

gs_status gs_rms_norm_workspace_bytes(int32_t rows, int32_t dim, size_t* bytes) {
    if (!bytes) return set_error(GS_ERR_ARG, "bytes is NULL");
    if (rows < 0 || dim < 1 || dim > NORM_MAX_DIM) return set_error(GS_ERR_ARG, "rows negative or dim outside [1, %d]", NORM_MAX_DIM);
    *bytes = norm_workspace(rows, dim);
    return GS_OK;
}

gs_status gs_rms_norm_forward(const void* d_x, int64_t x_ld, const void* d_residual_or_null, int64_t residual_ld, gs_dtype dtype,
                              const void* d_weight_or_null, gs_dtype weight_dtype, const int32_t* d_count_or_null, int32_t rows,
                              int32_t dim, float eps, void* d_hidden_or_null, int64_t hidden_ld, void* d_out, int64_t out_ld, void* stream) {
    RmsNorm p{};
    p.x = d_x; p.x_ld = x_ld; p.residual = d_residual_or_null; p.residual_ld = residual_ld; p.dtype = dtype;
    p.weight = d_weight_or_null; p.weight_dtype = weight_dtype; p.n = Count{d_count_or_null, rows}; p.dim = dim; p.eps = eps;
    p.hidden = d_hidden_or_null; p.hidden_ld = hidden_ld; p.out = d_out; p.out_ld = out_ld;
    GS_TRY(check_norm(p, false));
    if (rows == 0) return GS_OK;
    if (!d_out) return set_error(GS_ERR_ARG, "NULL argument");
    GS_TRAIN_CUDA(launch_norm_forward(p, false, (cudaStream_t)stream));
    return GS_OK;
}

gs_status gs_rms_norm_coded(const void* d_x, int64_t x_ld, const void* d_residual_or_null, int64_t residual_ld, gs_dtype dtype,
                            const void* d_weight_or_null, gs_dtype weight_dtype, const int32_t* d_count_or_null, int32_t rows,
                            int32_t dim, float eps, void* d_hidden_or_null, int64_t hidden_ld, const gs_coded* out, void* stream) {
    RmsNorm p{};
    p.x = d_x; p.x_ld = x_ld; p.residual = d_residual_or_null; p.residual_ld = residual_ld; p.dtype = dtype;
    p.weight = d_weight_or_null; p.weight_dtype = weight_dtype; p.n = Count{d_count_or_null, rows}; p.dim = dim; p.eps = eps;
    p.hidden = d_hidden_or_null; p.hidden_ld = hidden_ld;
    GS_TRY(check_norm(p, false));
    GS_TRY(check_coded("out", out, &p.coded));
    if (out->block != 1) return set_error(GS_ERR_ARG, "out has one scale for several rows");
    if ((int64_t)out->heads * out->head_dim != dim) return set_error(GS_ERR_ARG, "out holds %d * %d columns, x has %d", out->heads, out->head_dim, dim);
    if (out->rows < rows) return set_error(GS_ERR_ARG, "out has fewer rows than x");
    if (rows == 0) return GS_OK;
    GS_TRAIN_CUDA(launch_norm_forward(p, true, (cudaStream_t)stream));
    return GS_OK;
}

gs_status gs_rms_norm_backward(const void* d_hidden, int64_t hidden_ld, const void* d_dout, int64_t dout_ld,
                               const void* d_dhidden_or_null, int64_t dhidden_ld, gs_dtype dtype, const void* d_weight_or_null,
                               gs_dtype weight_dtype, const int32_t* d_count_or_null, int32_t rows, int32_t dim, float eps, void* d_dx,
                               int64_t dx_ld, void* d_dweight_or_null, void* d_workspace, size_t workspace_bytes, void* stream) {
    RmsNorm p{};
    p.x = d_hidden; p.x_ld = hidden_ld; p.dout = d_dout; p.dout_ld = dout_ld; p.residual = d_dhidden_or_null; p.residual_ld = dhidden_ld; p.dtype = dtype;
    p.weight = d_weight_or_null; p.weight_dtype = weight_dtype; p.n = Count{d_count_or_null, rows}; p.dim = dim; p.eps = eps;
    p.out = d_dx; p.out_ld = dx_ld; p.dweight = d_dweight_or_null;
    GS_TRY(check_norm(p, true));
    if (p.dweight && !known(weight_dtype)) return set_error(GS_ERR_ARG, "unknown dtype");
    if (rows == 0) {
        if (p.dweight) GS_TRAIN_CUDA(cudaMemsetAsync(p.dweight, 0, (size_t)dim * size_of(weight_dtype), (cudaStream_t)stream));
        return GS_OK;
    }
    GS_TRY(check_workspace(d_workspace, workspace_bytes, norm_workspace(rows, dim)));
    GS_TRAIN_CUDA(launch_norm_backward(p, d_workspace, (cudaStream_t)stream));
    return GS_OK;
}

gs_status gs_coded_write(const gs_coded* to, gs_dtype dtype, const gs_heads* rows, const int32_t* d_ids_or_null, int64_t first,
                         const int32_t* d_count_or_null, int32_t count_bound, int32_t* d_claims, void* stream) {
    CodedWrite p{};
    GS_TRY(check_coded("to", to, &p.to));
    if (!known(dtype)) return set_error(GS_ERR_ARG, "unknown dtype %d", (int)dtype);
    GS_TRY(check_list(d_ids_or_null, first, d_count_or_null, count_bound, to->rows));
    GS_TRY(check_heads("rows", rows, count_bound, to->heads, to->head_dim, dtype, &p.in));
    if (rows->row_stride * (int64_t)size_of(dtype) >= ((int64_t)1 << 32)) return set_error(GS_ERR_ARG, "the row pitch of rows is 4 GB or more");
    if (d_ids_or_null && !d_claims && to->rows > 0) return set_error(GS_ERR_ARG, "d_claims is NULL");
    if (!aligned_to(d_claims, 4)) return set_error(GS_ERR_ALIGN, "d_claims is misaligned");
    if (count_bound == 0 || to->rows == 0) return GS_OK;
    p.dtype = dtype; p.ids = d_ids_or_null; p.first = first; p.n = Count{d_count_or_null, count_bound}; p.claims = d_claims;
    GS_TRAIN_CUDA(launch_coded_write(p, (cudaStream_t)stream));
    return GS_OK;
}

gs_status gs_coded_read(const gs_coded* from, const int32_t* d_ids_or_null, int64_t first, const int32_t* d_count_or_null,
                        int32_t count_bound, gs_dtype dtype, const gs_heads* out, void* stream) {
    CodedRead p{};
    GS_TRY(check_coded("from", from, &p.from));
    if (!known(dtype)) return set_error(GS_ERR_ARG, "unknown dtype %d", (int)dtype);
    GS_TRY(check_list(d_ids_or_null, first, d_count_or_null, count_bound, from->rows));
    GS_TRY(check_heads("out", out, count_bound, from->heads, from->head_dim, dtype, &p.out));
    if (count_bound == 0) return GS_OK;
    p.dtype = dtype; p.ids = d_ids_or_null; p.first = first; p.n = Count{d_count_or_null, count_bound};
    GS_TRAIN_CUDA(launch_coded_read(p, (cudaStream_t)stream));
    return GS_OK;
}

gs_status gs_coded_attention_workspace_bytes(int32_t max_edges, int32_t q_heads, int32_t head_dim, size_t* bytes) {
    if (!bytes) return set_error(GS_ERR_ARG, "bytes is NULL");
    if (max_edges < 0 || max_edges >= (1 << 30)) return set_error(GS_ERR_ARG, "max_edges outside [0, 2^30)");
    if (q_heads < 1 || q_heads > 128 || head_dim < 1 || head_dim > 256) return set_error(GS_ERR_ARG, "q_heads outside [1, 128] or head_dim outside [1, 256]");
    *bytes = coded_attention_workspace(max_edges, q_heads, head_dim);
    return GS_OK;
}

gs_status gs_coded_attention_forward(const gs_block* block, const int32_t* d_rows_or_null, int32_t max_row, gs_dtype dtype,
                                     int32_t q_heads, int32_t head_dim, float scale, const gs_heads* q, const gs_coded* k,
                                     const gs_coded* v, const gs_heads* out, float* d_lse, void* d_workspace, size_t workspace_bytes,
                                     void* stream) {
    CodedAttention a{};
    GS_TRY(check_block(block));
    if (!known(dtype)) return set_error(GS_ERR_ARG, "unknown dtype %d", (int)dtype);
    if (max_row < 0) return set_error(GS_ERR_ARG, "max_row is negative");
    if (head_dim < 1 || head_dim > 256) return set_error(GS_ERR_ARG, "head_dim %d outside [1, 256]", head_dim);
    GS_TRY(check_coded("k", k, &a.k));
    GS_TRY(check_coded("v", v, &a.v));
    if (k->rows != v->rows || k->heads != v->heads || k->block != v->block || k->head_dim != head_dim || v->head_dim != head_dim)
        return set_error(GS_ERR_ARG, "k and v differ in rows, heads, block or head_dim");
    if (q_heads < 1 || q_heads > 128 || q_heads % k->heads) return set_error(GS_ERR_ARG, "q_heads %d, kv heads %d: 1 to 128, the second a divisor of the first", q_heads, k->heads);
    if (!d_rows_or_null && block->max_src > k->rows) return set_error(GS_ERR_ARG, "the block has more sources than k has rows");
    GS_TRY(check_heads("q", q, block->max_dst, q_heads, head_dim, dtype, &a.q));
    GS_TRY(check_heads("out", out, block->max_dst, q_heads, head_dim, dtype, &a.out));
    if (!aligned_to(d_rows_or_null, 4) || !aligned_to(d_lse, 4)) return set_error(GS_ERR_ALIGN, "misaligned argument");
    if (block->max_dst == 0) return GS_OK;
    if (!d_lse) return set_error(GS_ERR_ARG, "d_lse is NULL");
    a.indptr = block->d_indptr; a.indices = block->d_indices; a.row_of = d_rows_or_null;
    a.dst = Count{block->d_num_dst, block->max_dst}; a.src = Count{block->d_num_src, block->max_src};
    a.edge_bound = block->max_edges; a.max_row = max_row; a.dtype = dtype;
    a.q_heads = q_heads; a.kv_heads = k->heads; a.head_dim = head_dim; a.scale = scale; a.lse = d_lse;
    GS_TRY(check_workspace(d_workspace, workspace_bytes, coded_attention_workspace(block->max_edges, q_heads, head_dim)));
    GS_TRAIN_CUDA(launch_coded_attention(a, d_workspace, (cudaStream_t)stream));
    return GS_OK;
}

gs_status gs_grad_workspace_bytes(int32_t n, size_t* bytes) {
    if (!bytes) return set_error(GS_ERR_ARG, "bytes is NULL");
    if (n < 0 || n > (1 << 16)) return set_error(GS_ERR_ARG, "n outside [0, 65536]");
    *bytes = grad_workspace(n);
    return GS_OK;
}

gs_status gs_grad_norm(const gs_grad* list, int32_t n, float* d_norm, void* d_workspace, size_t workspace_bytes, void* stream) {
    return grads(list, n, false, 0.f, d_norm, d_workspace, workspace_bytes, (cudaStream_t)stream);
}

gs_status gs_grad_clip(const gs_grad* list, int32_t n, float max_norm, float* d_norm_or_null, void* d_workspace, size_t workspace_bytes,
                       void* stream) {
    return grads(list, n, true, max_norm, d_norm_or_null, d_workspace, workspace_bytes, (cudaStream_t)stream);
}

}  // extern "C"
