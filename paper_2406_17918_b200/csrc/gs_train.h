// Host-side descriptors of the training operators: embedding rows, attention over blocks, softmax over a table's rows.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <atomic>

#include "gs_internal.h"

namespace gs {

// Length of a list whose size only the device may know: *d_n if d_n is set, never more than `bound`.
struct Count {
    const int32_t* d_n;
    int32_t bound;
};

// Rows of a list by their offsets; NULL: none, the list as a whole.
struct Rows {
    const int32_t* offsets;
    Count n;
};

// Kernels of a call are set up while their predecessor drains; each begins with chain_wait().
template <typename... KArgs, typename... Args>
inline cudaError_t launch_train(void (*kernel)(KArgs...), int64_t grid, int block, size_t smem, cudaStream_t s, Args... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)limit_grid(grid));
    cfg.blockDim = dim3((unsigned)block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    count_launches(1);
    return cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);
}

// Allows `kernel` that much dynamic shared memory, once per device.
template <typename F> inline cudaError_t allow_smem(F* kernel, int bytes, std::atomic<uint64_t>& done) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = dev >= 0 && dev < 64 ? (uint64_t)1 << dev : 0;
    if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

// Resident blocks of a kernel on one SM, looked up once per device.
template <typename F> inline int resident_blocks(F* kernel, int threads, size_t smem, std::atomic<uint64_t>& known) {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 1;
    const uint64_t key = ((uint64_t)(dev + 1) << 48) | ((uint64_t)threads << 32) | (smem << 8), have = known.load(std::memory_order_relaxed);
    if ((have & ~0xFFull) == key) return (int)(have & 0xFF);
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, smem) != cudaSuccess || n < 1) n = 1;
    known.store(key | (uint64_t)n, std::memory_order_relaxed);
    return n;
}

// Memory to be cleared: 16-byte pieces (none: nothing) and fewer than 16 bytes behind them.
struct Fill {
    uint4* p;
    int64_t pieces;
    int tail;
};

// ---- stable sort of (key, payload) pairs by key: ascending keys, equal keys in input order ----
size_t key_sort_bytes(int64_t n_bound);
// Keys outside [0, key_limit), and those at positions outside the rows of `within`, take the value key_limit and end behind all
// others.  payload NULL: the position.
// `zero_words` int32 words at `zero` (or none) and `fill` are cleared on the way.
cudaError_t launch_key_sort(const int32_t* keys, const int32_t* payload, Count n, Rows within, int64_t key_limit, void* workspace,
                            uint32_t* out_keys, int32_t* out_payload, int32_t* zero, int zero_words, Fill fill, cudaStream_t s);
// starts[r] = number of sorted keys < r, r = 0 .. rows (rows from the device if rows.d_n is set).
cudaError_t launch_row_starts(const uint32_t* keys, Count n, Count rows, int32_t* starts, cudaStream_t s);

// ---- embedding rows ----
struct EmbedLookup {
    const void* table;
    void* out;
    const int32_t* ids;
    Count n;
    int64_t table_rows, table_ld, out_ld;
    int32_t dim;
    gs_dtype table_dtype, out_dtype;
    float scale;
};
cudaError_t launch_embedding_lookup(const EmbedLookup& p, cudaStream_t s);

struct EmbedGrad {
    const void* dout;
    void* grad;              // dense: [table_rows][grad_ld]; sparse: [n bound][grad_ld]
    const int32_t* ids;
    Count n;
    int64_t table_rows, dout_ld, grad_ld;
    int32_t dim;
    gs_dtype dout_dtype, grad_dtype;
    float scale;
    int32_t* rows;           // sparse only: ids of the rows, ascending, -1 behind them
    int32_t* d_num_rows;     // sparse only
};
size_t embedding_workspace(int64_t n_bound, int64_t table_rows, int32_t dim);
cudaError_t launch_embedding_grad(const EmbedGrad& p, void* workspace, cudaStream_t s);

// ---- attention over a block ----
struct HeadView {           // [rows][heads][head_dim], strides in elements, the last one 1
    void* data;
    int64_t row_stride, head_stride;
};
struct BlockAttention {
    const int32_t* indptr;
    const int32_t* indices;
    Count dst, src;
    int32_t edge_bound, max_row;
    gs_dtype dtype;
    int32_t q_heads, kv_heads, head_dim;
    float scale;
    HeadView q, k, v, out, dout, dq, dk, dv;
    float* lse;             // [dst][q_heads]
};
size_t attention_workspace(int64_t dst, int64_t edges, int32_t q_heads, int32_t head_dim);
size_t reverse_workspace(int64_t edges);
cudaError_t launch_attention_forward(const BlockAttention& a, void* workspace, cudaStream_t s);
cudaError_t launch_attention_backward(const BlockAttention& a, const int32_t* rev_indptr, const int32_t* rev_dst, const int32_t* rev_edge,
                                      void* workspace, cudaStream_t s);
cudaError_t launch_block_reverse(const int32_t* indptr, const int32_t* indices, Count dst, Count src, Count edges, int32_t* rev_indptr,
                                 int32_t* rev_dst, int32_t* rev_edge, void* workspace, cudaStream_t s);

// ---- softmax cross entropy against every row of a table ----
struct Xent {
    const void* hidden;
    const void* table;
    int64_t hidden_ld, table_ld, vocab;
    gs_dtype dtype;
    int32_t rows, dim;
    float scale;
    const int32_t* labels;
    float* loss;            // forward
    float* lse_out;
    const float* lse;       // backward
    const float* dloss;
    void* dhidden;
    void* dtable;
    int64_t dhidden_ld, dtable_ld;
    gs_dtype grad_dtype;
#ifdef __CUDACC__
    __device__ void store(void* to, int64_t at, float x) const {
        if (grad_dtype == GS_BF16) static_cast<__nv_bfloat16*>(to)[at] = __float2bfloat16_rn(x);
        else static_cast<float*>(to)[at] = x;
    }
    __device__ void store_dhidden(int64_t r, int c, float x) const { store(dhidden, r * dhidden_ld + c, x); }
    __device__ void store_dtable(int64_t r, int c, float x) const { store(dtable, r * dtable_ld + c, x); }
#endif
};
size_t xent_workspace(const Xent& a);      // sizes and dtype only
cudaError_t launch_xent_forward(const Xent& a, void* workspace, cudaStream_t s);
cudaError_t launch_xent_backward(const Xent& a, void* workspace, cudaStream_t s);

// ---- rows in 8 bits ----
struct CodedView {
    uint8_t* codes;         // [rows][row_stride], head h at h * pitch
    uint8_t* scales;        // [blocks][scale_stride]
    int64_t rows, row_stride, scale_stride;
    int32_t heads, head_dim, pitch, shift;    // blocks of 1 << shift rows
};
struct CodedWrite {
    CodedView to;
    HeadView in;
    gs_dtype dtype;
    const int32_t* ids;     // NULL: the rows from `first` on
    int64_t first;
    Count n;
    int32_t* claims;
    int tl, head_tiles;
};
cudaError_t launch_coded_write(const CodedWrite& p, cudaStream_t s);
struct CodedRead {
    CodedView from;
    HeadView out;
    gs_dtype dtype;
    const int32_t* ids;
    int64_t first;
    Count n;
    int tl;
};
cudaError_t launch_coded_read(const CodedRead& p, cudaStream_t s);

// ---- attention over such rows ----
struct CodedAttention {
    const int32_t* indptr;
    const int32_t* indices;
    const int32_t* row_of;  // NULL: a source is its row
    Count dst, src;
    int32_t edge_bound, max_row;
    gs_dtype dtype;
    int32_t q_heads, kv_heads, head_dim;
    float scale;
    HeadView q, out;
    CodedView k, v;
    float* lse;
};
size_t coded_attention_workspace(int64_t edges, int32_t q_heads, int32_t head_dim);
cudaError_t launch_coded_attention(const CodedAttention& a, void* workspace, cudaStream_t s);

// ---- root-mean-square norm ----
struct RmsNorm {
    const void* x;          // backward: what was normalised
    const void* residual;   // backward: the gradient that comes along the residual path
    const void* dout;       // backward
    const void* weight;
    void* hidden;
    void* out;              // backward: dx
    void* dweight;
    int64_t x_ld, residual_ld, dout_ld, hidden_ld, out_ld;
    gs_dtype dtype, weight_dtype;
    Count n;
    int32_t dim;
    float eps;
    CodedView coded;        // output in 8 bits
    int tl, period, phase;
    float inv_dim;
};
constexpr int NORM_MAX_DIM = 8192;      // 512 threads of 16 elements
size_t norm_workspace(int64_t rows, int32_t dim);
cudaError_t launch_norm_forward(const RmsNorm& p, bool coded, cudaStream_t s);
cudaError_t launch_norm_backward(const RmsNorm& p, void* workspace, cudaStream_t s);

// ---- the norm over many gradients ----
struct GradTensor {
    const void* grad;
    void* out;              // clipping: where the scaled gradient goes (grad itself: in place)
    const int32_t* d_rows;  // NULL: all of it; else the rows of row_elems that count
    int64_t elems;
    int64_t row_elems;
    gs_dtype dtype;
    int32_t first_tile;
};
size_t grad_workspace(int32_t tensors);
// norm: the global norm, on the device.  clip: `out` of every tensor gets the scaled gradient.
cudaError_t launch_grad_norm(const GradTensor* tensors, int32_t n, bool clip, float max_norm, float* norm, void* workspace, cudaStream_t s);

}  // namespace gs
