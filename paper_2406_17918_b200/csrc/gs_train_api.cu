// The C ABI of the training operators: argument checks and launches.
#include "gs_train.h"

using namespace gs;

namespace {

bool aligned_to(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
bool known(gs_dtype t) { return t == GS_F32 || t == GS_BF16; }
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

gs_status gs_train_status(void* stream) {
    int sort = 0;
    GS_TRAIN_CUDA(train_gave_up((cudaStream_t)stream, &sort));
    if (sort) return set_error(GS_ERR_CUDA, "a sort gave up waiting for an earlier tile");
    return GS_OK;
}

}  // extern "C"
