// The C ABI of the training operators: argument checks and launches.
#include "gs_train.h"
#include "gs_xent.h"

using namespace gs;

namespace {

bool aligned_to(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
bool known(gs_dtype t) { return t == GS_F32 || t == GS_BF16; }
constexpr int64_t XENT_MAX_VOCAB = ((int64_t)1 << 31) - 257;   // row numbers of whole tiles stay below 2^31
size_t size_of(gs_dtype t) { return t == GS_BF16 ? 2 : 4; }

gs_status cuda_error(cudaError_t e, const char* what) { return set_error(GS_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e)); }

#define GS_TRAIN_CUDA(call)                                     \
    do {                                                        \
        const cudaError_t e__ = (call);                         \
        if (e__ != cudaSuccess) return cuda_error(e__, #call);  \
    } while (0)

gs_status check_workspace(const void* ws, size_t have, size_t need) {
    if (!ws) return set_error(GS_ERR_ARG, "workspace is NULL");
    if (!aligned_to(ws, 256)) return set_error(GS_ERR_ALIGN, "workspace is not 256-byte aligned");
    if (have < need) return set_error(GS_ERR_WORKSPACE, "workspace holds %zu bytes, %zu are needed", have, need);
    return GS_OK;
}

gs_status check_table(int64_t rows, int32_t dim) {
    if (rows < 1 || rows >= ((int64_t)1 << 31)) return set_error(GS_ERR_ARG, "table_rows outside [1, 2^31)");
    if (dim < 1 || dim > (1 << 20)) return set_error(GS_ERR_ARG, "dim %d outside [1, 2^20]", dim);
    return GS_OK;
}

gs_status embedding_grad(EmbedGrad g, bool sparse, void* ws, size_t ws_bytes, cudaStream_t s) {
    if (!known(g.dout_dtype) || !known(g.grad_dtype)) return set_error(GS_ERR_ARG, "unknown dtype");
    if (g.n.bound < 0 || g.n.bound >= (1 << 30)) return set_error(GS_ERR_ARG, "count_bound outside [0, 2^30)");
    const gs_status st = check_table(g.table_rows, g.dim);
    if (st != GS_OK) return st;
    if ((!g.grad && (!sparse || g.n.bound > 0)) || (sparse && (!g.d_num_rows || (!g.rows && g.n.bound > 0)))) return set_error(GS_ERR_ARG, "NULL argument");
    if (g.grad_ld < g.dim || g.dout_ld < g.dim) return set_error(GS_ERR_ARG, "a row pitch is smaller than dim");
    if (g.dout_ld * (int64_t)size_of(g.dout_dtype) >= ((int64_t)1 << 32)) return set_error(GS_ERR_ARG, "the row pitch of dout is 4 GB or more");
    if (!aligned_to(g.grad, size_of(g.grad_dtype)) || !aligned_to(g.dout, size_of(g.dout_dtype)) || !aligned_to(g.ids, 4) ||
        !aligned_to(g.rows, 4) || !aligned_to(g.d_num_rows, 4) || !aligned_to(g.n.d_n, 4))
        return set_error(GS_ERR_ALIGN, "misaligned argument");
    if (g.n.bound == 0) {
        if (sparse) GS_TRAIN_CUDA(cudaMemsetAsync(g.d_num_rows, 0, 4, s));
        else GS_TRAIN_CUDA(cudaMemset2DAsync(g.grad, (size_t)g.grad_ld * size_of(g.grad_dtype), 0, (size_t)g.dim * size_of(g.grad_dtype), (size_t)g.table_rows, s));
        return GS_OK;
    }
    if (!g.dout || !g.ids) return set_error(GS_ERR_ARG, "NULL argument");
    const gs_status w = check_workspace(ws, ws_bytes, embedding_workspace(g.n.bound, g.table_rows, g.dim));
    if (w != GS_OK) return w;
    GS_TRAIN_CUDA(launch_embedding_grad(g, ws, s));
    return GS_OK;
}

gs_status check_block(const gs_block* b) {
    if (!b) return set_error(GS_ERR_ARG, "block is NULL");
    if (b->max_dst < 0 || b->max_src < 0 || b->max_edges < 0 || b->max_edges >= (1 << 30)) return set_error(GS_ERR_ARG, "a size of the block is out of range");
    if (!b->d_indptr || (b->max_edges > 0 && !b->d_indices)) return set_error(GS_ERR_ARG, "the block has no arrays");
    const int given = (b->d_num_dst != nullptr) + (b->d_num_src != nullptr) + (b->d_num_edges != nullptr);
    if (given != 0 && given != 3) return set_error(GS_ERR_ARG, "the block's device counts are given all together or not at all");
    if (!aligned_to(b->d_indptr, 4) || !aligned_to(b->d_indices, 4) || !aligned_to(b->d_num_dst, 4) || !aligned_to(b->d_num_src, 4) || !aligned_to(b->d_num_edges, 4))
        return set_error(GS_ERR_ALIGN, "misaligned block array");
    return GS_OK;
}

gs_status check_heads(const char* name, const gs_heads* h, int64_t rows, int32_t heads, int32_t dim, gs_dtype t, HeadView* out) {
    if (!h || (!h->d_data && rows > 0)) return set_error(GS_ERR_ARG, "%s is NULL", name);
    if ((heads > 1 && h->head_stride < dim) || (rows > 1 && h->row_stride < dim)) return set_error(GS_ERR_ARG, "%s: a stride is smaller than head_dim", name);
    if (!aligned_to(h->d_data, size_of(t))) return set_error(GS_ERR_ALIGN, "%s is misaligned", name);
    *out = HeadView{h->d_data, h->row_stride, h->head_stride};
    return GS_OK;
}

#define GS_TRY(call)                          \
    do {                                      \
        const gs_status s__ = (call);         \
        if (s__ != GS_OK) return s__;         \
    } while (0)

gs_status check_attention(const gs_block* b, int32_t max_row, gs_dtype t, int32_t q_heads, int32_t kv_heads, int32_t dim, BlockAttention* a) {
    GS_TRY(check_block(b));
    if (!known(t)) return set_error(GS_ERR_ARG, "unknown dtype %d", (int)t);
    if (max_row < 0) return set_error(GS_ERR_ARG, "max_row is negative");
    if (dim < 1 || dim > 256) return set_error(GS_ERR_ARG, "head_dim %d outside [1, 256]", dim);
    if (q_heads < 1 || q_heads > 128 || kv_heads < 1 || q_heads % kv_heads) return set_error(GS_ERR_ARG, "q_heads %d, kv_heads %d: 1 to 128, the second a divisor of the first", q_heads, kv_heads);
    a->indptr = b->d_indptr;
    a->indices = b->d_indices;
    a->dst = Count{b->d_num_dst, b->max_dst};
    a->src = Count{b->d_num_src, b->max_src};
    a->edge_bound = b->max_edges;
    a->max_row = max_row;
    a->dtype = t;
    a->q_heads = q_heads;
    a->kv_heads = kv_heads;
    a->head_dim = dim;
    return GS_OK;
}

gs_status check_xent(const Xent& a, const void* ws, size_t ws_bytes) {
    if (!known(a.dtype)) return set_error(GS_ERR_ARG, "unknown dtype %d", (int)a.dtype);
    if (a.rows < 0 || a.rows > XENT_MAX_VOCAB) return set_error(GS_ERR_ARG, "rows outside [0, 2^31 - 256)");
    if (a.vocab < 1 || a.vocab > XENT_MAX_VOCAB) return set_error(GS_ERR_ARG, "vocab outside [1, 2^31 - 256)");
    if (a.dim < 1 || a.dim > 4096) return set_error(GS_ERR_ARG, "dim %d outside [1, 4096]", a.dim);
    if (!a.table || (a.rows > 0 && (!a.hidden || !a.labels))) return set_error(GS_ERR_ARG, "NULL argument");
    if (a.hidden_ld < a.dim || a.table_ld < a.dim) return set_error(GS_ERR_ARG, "a row pitch is smaller than dim");
    if (!aligned_to(a.hidden, size_of(a.dtype)) || !aligned_to(a.table, size_of(a.dtype)) || !aligned_to(a.labels, 4))
        return set_error(GS_ERR_ALIGN, "misaligned argument");
    if (a.rows == 0) return GS_OK;
    return check_workspace(ws, ws_bytes, xent_workspace(a));
}

}  // namespace

extern "C" {

gs_status gs_embedding_lookup(const void* d_table, gs_dtype table_dtype, int64_t table_rows, int32_t dim, int64_t table_ld,
                              const int32_t* d_ids, const int32_t* d_count_or_null, int32_t count_bound, float scale,
                              void* d_out, gs_dtype out_dtype, int64_t out_ld, void* stream) {
    if (!known(table_dtype) || !known(out_dtype)) return set_error(GS_ERR_ARG, "unknown dtype");
    const gs_status st = check_table(table_rows, dim);
    if (st != GS_OK) return st;
    if (count_bound < 0) return set_error(GS_ERR_ARG, "count_bound is negative");
    if (count_bound == 0) return GS_OK;
    if (!d_table || !d_ids || !d_out) return set_error(GS_ERR_ARG, "NULL argument");
    if (table_ld < dim || out_ld < dim) return set_error(GS_ERR_ARG, "a row pitch is smaller than dim");
    if (!aligned_to(d_table, size_of(table_dtype)) || !aligned_to(d_out, size_of(out_dtype)) || !aligned_to(d_ids, 4) || !aligned_to(d_count_or_null, 4))
        return set_error(GS_ERR_ALIGN, "misaligned argument");
    EmbedLookup p{d_table, d_out, d_ids, Count{d_count_or_null, count_bound}, table_rows, table_ld, out_ld, dim, table_dtype, out_dtype, scale};
    GS_TRAIN_CUDA(launch_embedding_lookup(p, (cudaStream_t)stream));
    return GS_OK;
}

gs_status gs_embedding_workspace_bytes(int32_t count_bound, int64_t table_rows, int32_t dim, size_t* bytes) {
    if (!bytes) return set_error(GS_ERR_ARG, "bytes is NULL");
    if (count_bound < 0 || count_bound >= (1 << 30)) return set_error(GS_ERR_ARG, "count_bound outside [0, 2^30)");
    const gs_status st = check_table(table_rows, dim);
    if (st != GS_OK) return st;
    *bytes = embedding_workspace(count_bound, table_rows, dim);
    return GS_OK;
}

gs_status gs_embedding_backward(const void* d_dout, gs_dtype dout_dtype, int64_t dout_ld, const int32_t* d_ids,
                                const int32_t* d_count_or_null, int32_t count_bound, int64_t table_rows, int32_t dim,
                                float scale, void* d_dtable, gs_dtype dtable_dtype, int64_t dtable_ld, void* d_workspace,
                                size_t workspace_bytes, void* stream) {
    EmbedGrad g{d_dout, d_dtable, d_ids, Count{d_count_or_null, count_bound}, table_rows, dout_ld, dtable_ld, dim,
                dout_dtype, dtable_dtype, scale, nullptr, nullptr};
    return embedding_grad(g, false, d_workspace, workspace_bytes, (cudaStream_t)stream);
}

gs_status gs_embedding_backward_sparse(const void* d_dout, gs_dtype dout_dtype, int64_t dout_ld, const int32_t* d_ids,
                                       const int32_t* d_count_or_null, int32_t count_bound, int64_t table_rows, int32_t dim,
                                       float scale, int32_t* d_rows, int32_t* d_num_rows, void* d_grad, gs_dtype grad_dtype,
                                       int64_t grad_ld, void* d_workspace, size_t workspace_bytes, void* stream) {
    EmbedGrad g{d_dout, d_grad, d_ids, Count{d_count_or_null, count_bound}, table_rows, dout_ld, grad_ld, dim,
                dout_dtype, grad_dtype, scale, d_rows, d_num_rows};
    return embedding_grad(g, true, d_workspace, workspace_bytes, (cudaStream_t)stream);
}

gs_status gs_block_attention_workspace_bytes(int32_t max_dst, int32_t max_edges, int32_t q_heads, int32_t head_dim, size_t* bytes) {
    if (!bytes) return set_error(GS_ERR_ARG, "bytes is NULL");
    if (max_dst < 0 || max_edges < 0 || max_edges >= (1 << 30)) return set_error(GS_ERR_ARG, "a size of the block is out of range");
    if (q_heads < 1 || q_heads > 128 || head_dim < 1 || head_dim > 256) return set_error(GS_ERR_ARG, "q_heads outside [1, 128] or head_dim outside [1, 256]");
    *bytes = attention_workspace(max_dst, max_edges, q_heads, head_dim);
    return GS_OK;
}

gs_status gs_block_attention_forward(const gs_block* block, int32_t max_row, gs_dtype dtype, int32_t q_heads, int32_t kv_heads,
                                     int32_t head_dim, float scale, const gs_heads* q, const gs_heads* k, const gs_heads* v,
                                     const gs_heads* out, float* d_lse, void* d_workspace, size_t workspace_bytes, void* stream) {
    BlockAttention a{};
    GS_TRY(check_attention(block, max_row, dtype, q_heads, kv_heads, head_dim, &a));
    a.scale = scale;
    GS_TRY(check_heads("q", q, block->max_dst, q_heads, head_dim, dtype, &a.q));
    GS_TRY(check_heads("k", k, block->max_src, kv_heads, head_dim, dtype, &a.k));
    GS_TRY(check_heads("v", v, block->max_src, kv_heads, head_dim, dtype, &a.v));
    GS_TRY(check_heads("out", out, block->max_dst, q_heads, head_dim, dtype, &a.out));
    if (block->max_dst == 0) return GS_OK;
    if (!d_lse) return set_error(GS_ERR_ARG, "d_lse is NULL");
    if (!aligned_to(d_lse, 4)) return set_error(GS_ERR_ALIGN, "d_lse is misaligned");
    a.lse = d_lse;
    GS_TRY(check_workspace(d_workspace, workspace_bytes, attention_workspace(block->max_dst, block->max_edges, q_heads, head_dim)));
    GS_TRAIN_CUDA(launch_attention_forward(a, d_workspace, (cudaStream_t)stream));
    return GS_OK;
}

gs_status gs_block_reverse(const gs_block* block, int32_t* d_rev_indptr, int32_t* d_rev_dst, int32_t* d_rev_edge, void* d_workspace,
                           size_t workspace_bytes, void* stream) {
    GS_TRY(check_block(block));
    if (!d_rev_indptr || ((!d_rev_dst || !d_rev_edge) && block->max_edges > 0)) return set_error(GS_ERR_ARG, "NULL argument");
    if (!aligned_to(d_rev_indptr, 4) || !aligned_to(d_rev_dst, 4) || !aligned_to(d_rev_edge, 4)) return set_error(GS_ERR_ALIGN, "misaligned argument");
    if (block->max_src == ((int32_t)0x7FFFFFFF)) return set_error(GS_ERR_ARG, "a size of the block is out of range");
    GS_TRY(check_workspace(d_workspace, workspace_bytes, reverse_workspace(block->max_edges)));
    // without a device count the edges end where the last row does
    const int32_t* d_edges = block->d_num_edges ? block->d_num_edges : block->d_indptr + block->max_dst;
    GS_TRAIN_CUDA(launch_block_reverse(block->d_indptr, block->d_indices, Count{block->d_num_dst, block->max_dst},
                                       Count{block->d_num_src, block->max_src}, Count{d_edges, block->max_edges}, d_rev_indptr, d_rev_dst, d_rev_edge,
                                       d_workspace, (cudaStream_t)stream));
    return GS_OK;
}

gs_status gs_block_attention_backward(const gs_block* block, int32_t max_row, const int32_t* d_rev_indptr, const int32_t* d_rev_dst,
                                      const int32_t* d_rev_edge, gs_dtype dtype, int32_t q_heads, int32_t kv_heads, int32_t head_dim, float scale,
                                      const gs_heads* q, const gs_heads* k, const gs_heads* v, const gs_heads* out,
                                      const float* d_lse, const gs_heads* dout, const gs_heads* dq, const gs_heads* dk,
                                      const gs_heads* dv, void* d_workspace, size_t workspace_bytes, void* stream) {
    BlockAttention a{};
    GS_TRY(check_attention(block, max_row, dtype, q_heads, kv_heads, head_dim, &a));
    a.scale = scale;
    GS_TRY(check_heads("q", q, block->max_dst, q_heads, head_dim, dtype, &a.q));
    GS_TRY(check_heads("k", k, block->max_src, kv_heads, head_dim, dtype, &a.k));
    GS_TRY(check_heads("v", v, block->max_src, kv_heads, head_dim, dtype, &a.v));
    GS_TRY(check_heads("out", out, block->max_dst, q_heads, head_dim, dtype, &a.out));
    GS_TRY(check_heads("dout", dout, block->max_dst, q_heads, head_dim, dtype, &a.dout));
    GS_TRY(check_heads("dq", dq, block->max_dst, q_heads, head_dim, dtype, &a.dq));
    GS_TRY(check_heads("dk", dk, block->max_src, kv_heads, head_dim, dtype, &a.dk));
    GS_TRY(check_heads("dv", dv, block->max_src, kv_heads, head_dim, dtype, &a.dv));
    if (!d_rev_indptr || ((!d_rev_dst || !d_rev_edge) && block->max_edges > 0) || (!d_lse && block->max_dst > 0)) return set_error(GS_ERR_ARG, "NULL argument");
    if (!aligned_to(d_rev_indptr, 4) || !aligned_to(d_rev_dst, 4) || !aligned_to(d_rev_edge, 4) || !aligned_to(d_lse, 4)) return set_error(GS_ERR_ALIGN, "misaligned argument");
    a.lse = const_cast<float*>(d_lse);
    GS_TRY(check_workspace(d_workspace, workspace_bytes, attention_workspace(block->max_dst, block->max_edges, q_heads, head_dim)));
    GS_TRAIN_CUDA(launch_attention_backward(a, d_rev_indptr, d_rev_dst, d_rev_edge, d_workspace, (cudaStream_t)stream));
    return GS_OK;
}

gs_status gs_xent_workspace_bytes(int32_t rows, int64_t vocab, int32_t dim, gs_dtype dtype, size_t* bytes) {
    if (!bytes) return set_error(GS_ERR_ARG, "bytes is NULL");
    if (!known(dtype) || rows < 0 || vocab < 1 || vocab > XENT_MAX_VOCAB || dim < 1 || dim > 4096) return set_error(GS_ERR_ARG, "a size or the dtype is out of range");
    Xent a{};
    a.rows = rows;
    a.vocab = vocab;
    a.dim = dim;
    a.dtype = dtype;
    *bytes = xent_workspace(a);
    return GS_OK;
}

gs_status gs_xent_forward(const void* d_hidden, int64_t hidden_ld, const void* d_table, int64_t table_ld, gs_dtype dtype,
                          int32_t rows, int64_t vocab, int32_t dim, float scale, const int32_t* d_labels, float* d_loss,
                          float* d_lse, void* d_workspace, size_t workspace_bytes, void* stream) {
    Xent a{};
    a.hidden = d_hidden; a.hidden_ld = hidden_ld; a.table = d_table; a.table_ld = table_ld; a.dtype = dtype;
    a.rows = rows; a.vocab = vocab; a.dim = dim; a.scale = scale; a.labels = d_labels; a.loss = d_loss; a.lse_out = d_lse;
    GS_TRY(check_xent(a, d_workspace, workspace_bytes));
    if (rows == 0) return GS_OK;
    if (!d_loss || !d_lse) return set_error(GS_ERR_ARG, "NULL argument");
    if (!aligned_to(d_loss, 4) || !aligned_to(d_lse, 4)) return set_error(GS_ERR_ALIGN, "misaligned argument");
    GS_TRAIN_CUDA(launch_xent_forward(a, d_workspace, (cudaStream_t)stream));
    return GS_OK;
}

gs_status gs_xent_backward(const void* d_hidden, int64_t hidden_ld, const void* d_table, int64_t table_ld, gs_dtype dtype,
                           int32_t rows, int64_t vocab, int32_t dim, float scale, const int32_t* d_labels, const float* d_lse,
                           const float* d_dloss, void* d_dhidden, int64_t dhidden_ld, void* d_dtable, int64_t dtable_ld,
                           gs_dtype grad_dtype, void* d_workspace, size_t workspace_bytes, void* stream) {
    Xent a{};
    a.hidden = d_hidden; a.hidden_ld = hidden_ld; a.table = d_table; a.table_ld = table_ld; a.dtype = dtype;
    a.rows = rows; a.vocab = vocab; a.dim = dim; a.scale = scale; a.labels = d_labels; a.lse = d_lse; a.dloss = d_dloss;
    a.dhidden = d_dhidden; a.dhidden_ld = dhidden_ld; a.dtable = d_dtable; a.dtable_ld = dtable_ld; a.grad_dtype = grad_dtype;
    GS_TRY(check_xent(a, d_workspace, workspace_bytes));
    if (!known(grad_dtype)) return set_error(GS_ERR_ARG, "unknown dtype %d", (int)grad_dtype);
    if (!d_dtable || (rows > 0 && (!d_dhidden || !d_lse || !d_dloss))) return set_error(GS_ERR_ARG, "NULL argument");
    if (dhidden_ld < dim || dtable_ld < dim) return set_error(GS_ERR_ARG, "a row pitch is smaller than dim");
    if (!aligned_to(d_dhidden, size_of(grad_dtype)) || !aligned_to(d_dtable, size_of(grad_dtype)) || !aligned_to(d_lse, 4) || !aligned_to(d_dloss, 4))
        return set_error(GS_ERR_ALIGN, "misaligned argument");
    if (rows == 0) {
        GS_TRAIN_CUDA(cudaMemset2DAsync(d_dtable, (size_t)dtable_ld * size_of(grad_dtype), 0, (size_t)dim * size_of(grad_dtype), (size_t)vocab, (cudaStream_t)stream));
        return GS_OK;
    }
    GS_TRAIN_CUDA(launch_xent_backward(a, d_workspace, (cudaStream_t)stream));
    return GS_OK;
}

gs_status gs_train_status(void* stream) {
    int xent = 0;
    GS_TRAIN_CUDA(xent_gave_up((cudaStream_t)stream, &xent));
    if (xent) return set_error(GS_ERR_CUDA, "a softmax kernel gave up waiting for a copy or a product");
    return GS_OK;
}

}  // extern "C"
