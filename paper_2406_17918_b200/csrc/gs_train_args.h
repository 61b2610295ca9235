// Argument checks that the training operators' entry points share.
#pragma once
#include "gs_train.h"

namespace gs {

inline bool aligned_to(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
inline bool known(gs_dtype t) { return t == GS_F32 || t == GS_BF16; }
inline size_t size_of(gs_dtype t) { return t == GS_BF16 ? 2 : 4; }

inline gs_status cuda_error(cudaError_t e, const char* what) { return set_error(GS_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e)); }

#define GS_TRAIN_CUDA(call)                                     \
    do {                                                        \
        const cudaError_t e__ = (call);                         \
        if (e__ != cudaSuccess) return cuda_error(e__, #call);  \
    } while (0)

inline gs_status check_workspace(const void* ws, size_t have, size_t need) {
    if (!ws) return set_error(GS_ERR_ARG, "workspace is NULL");
    if (!aligned_to(ws, 256)) return set_error(GS_ERR_ALIGN, "workspace is not 256-byte aligned");
    if (have < need) return set_error(GS_ERR_WORKSPACE, "workspace holds %zu bytes, %zu are needed", have, need);
    return GS_OK;
}

#define GS_TRY(call)                          \
    do {                                      \
        const gs_status s__ = (call);         \
        if (s__ != GS_OK) return s__;         \
    } while (0)

inline gs_status check_block(const gs_block* b) {
    if (!b) return set_error(GS_ERR_ARG, "block is NULL");
    if (b->max_dst < 0 || b->max_src < 0 || b->max_edges < 0 || b->max_edges >= (1 << 30)) return set_error(GS_ERR_ARG, "a size of the block is out of range");
    if (!b->d_indptr || (b->max_edges > 0 && !b->d_indices)) return set_error(GS_ERR_ARG, "the block has no arrays");
    const int given = (b->d_num_dst != nullptr) + (b->d_num_src != nullptr) + (b->d_num_edges != nullptr);
    if (given != 0 && given != 3) return set_error(GS_ERR_ARG, "the block's device counts are given all together or not at all");
    if (!aligned_to(b->d_indptr, 4) || !aligned_to(b->d_indices, 4) || !aligned_to(b->d_num_dst, 4) || !aligned_to(b->d_num_src, 4) || !aligned_to(b->d_num_edges, 4))
        return set_error(GS_ERR_ALIGN, "misaligned block array");
    return GS_OK;
}

inline gs_status check_heads(const char* name, const gs_heads* h, int64_t rows, int32_t heads, int32_t dim, gs_dtype t, HeadView* out) {
    if (!h || (!h->d_data && rows > 0)) return set_error(GS_ERR_ARG, "%s is NULL", name);
    if ((heads > 1 && h->head_stride < dim) || (rows > 1 && h->row_stride < dim)) return set_error(GS_ERR_ARG, "%s: a stride is smaller than head_dim", name);
    if (!aligned_to(h->d_data, size_of(t))) return set_error(GS_ERR_ALIGN, "%s is misaligned", name);
    *out = HeadView{h->d_data, h->row_stride, h->head_stride};
    return GS_OK;
}

}  // namespace gs
