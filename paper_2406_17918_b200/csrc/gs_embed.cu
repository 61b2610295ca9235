// Embedding rows: out[p] = scale * table[ids[p]], and the gradient of the table.
//
// The gradient of row r is scale * (sum of the rows dout[p] with ids[p] = r): the positions are sorted by id (stable,
// gs_sort.cu), the rows of a run are added in ascending position in 32 bits and rounded once.  No atomics on
// floats: the result does not depend on the schedule.  Runs of up to ES_CHUNK entries are summed by the group of
// lanes that writes the row; a longer run (a hub) is cut into chunks whose sums go to the workspace and are added in order.
#include "gs_device.cuh"
#include "gs_train.cuh"
#include "gs_train.h"

namespace gs {

constexpr int EL_THREADS = 256;
constexpr int EL_ROWS = 4;      // rows in flight per thread of the lookup

__device__ __forceinline__ int list_length(const Count& c) {
    if (!c.d_n) return c.bound;
    const int n = __ldcg(c.d_n);      // may be the work of the kernel before
    return n < 0 ? 0 : (n > c.bound ? c.bound : n);
}

template <typename Tin, typename Tout, int VE>
__global__ void __launch_bounds__(EL_THREADS) k_embed_lookup(EmbedLookup P) {
    const int n = list_length(P.n);
    const int units = P.dim / VE;
    const int tpr = units < EL_THREADS ? units : EL_THREADS;
    const int rows_per_iter = EL_THREADS / tpr;
    const int r_in = threadIdx.x / tpr;
    const int u0 = threadIdx.x - r_in * tpr;
    if (r_in >= rows_per_iter) return;
    const Tin* table = (const Tin*)P.table;
    Tout* out = (Tout*)P.out;
    const int64_t step = (int64_t)gridDim.x * rows_per_iter;
    for (int64_t row = (int64_t)blockIdx.x * rows_per_iter + r_in; row < n; row += step * EL_ROWS) {
        int32_t id[EL_ROWS];
#pragma unroll
        for (int j = 0; j < EL_ROWS; ++j) {
            const int64_t rj = row + j * step;
            id[j] = rj < n ? __ldg(P.ids + rj) : -1;
        }
        for (int u = u0; u < units; u += tpr) {
            Raw<Tin, VE> v[EL_ROWS];
#pragma unroll
            for (int j = 0; j < EL_ROWS; ++j)
                v[j] = (uint32_t)id[j] < (uint32_t)P.table_rows ? load_raw_stream<Tin, VE>(table + (int64_t)id[j] * P.table_ld + (int64_t)u * VE)
                                                                 : zero_raw<Tin, VE>();
#pragma unroll
            for (int j = 0; j < EL_ROWS; ++j) {
                const int64_t rj = row + j * step;
                if (rj >= n) continue;
                float x[VE];
                unpack<Tin, VE>(v[j], x);
                const bool in = (uint32_t)id[j] < (uint32_t)P.table_rows;
#pragma unroll
                for (int i = 0; i < VE; ++i) x[i] = in ? x[i] * P.scale : 0.f;     // a row outside the table is zero whatever the scale
                store_vec<Tout, VE>(out + rj * P.out_ld + (int64_t)u * VE, x);
            }
        }
    }
}

// The widest unit, in elements of an input type of `in` bytes, that divides the row and keeps both sides aligned.
static int unit_elems(const void* src, int64_t src_ld, int in, const void* dst, int64_t dst_ld, int out, int dim) {
    for (int ve = 16 / in; ve > 1; ve /= 2) {
        const int wout = ve * out > 16 ? 16 : ve * out;
        if (dim % ve == 0 && ((uintptr_t)src | (uint64_t)(src_ld * in)) % (ve * in) == 0 && ((uintptr_t)dst | (uint64_t)(dst_ld * out)) % wout == 0)
            return ve;
    }
    return 1;
}

static int bytes_of(gs_dtype t) { return t == GS_BF16 ? 2 : 4; }

template <typename Tin, typename Tout, int VE> static void lookup_t(const EmbedLookup& p, cudaStream_t s) {
    const int units = p.dim / VE, tpr = units < EL_THREADS ? units : EL_THREADS, rpi = EL_THREADS / tpr;
    int64_t blocks = ((int64_t)p.n.bound + (int64_t)rpi * EL_ROWS - 1) / ((int64_t)rpi * EL_ROWS);
    if (blocks > sm_count() * 64) blocks = sm_count() * 64;
    k_embed_lookup<Tin, Tout, VE><<<(int)limit_grid(blocks), EL_THREADS, 0, s>>>(p);
}

template <typename Tin, typename Tout> static void lookup_tt(const EmbedLookup& p, int ve, cudaStream_t s) {
    if constexpr (sizeof(Tin) == 2) {
        if (ve == 8) return lookup_t<Tin, Tout, 8>(p, s);
    }
    if (ve == 4) return lookup_t<Tin, Tout, 4>(p, s);
    if (ve == 2) return lookup_t<Tin, Tout, 2>(p, s);
    lookup_t<Tin, Tout, 1>(p, s);
}

cudaError_t launch_embedding_lookup(const EmbedLookup& p, cudaStream_t s) {
    if (p.n.bound <= 0) return cudaSuccess;
    const int in = bytes_of(p.table_dtype), out = bytes_of(p.out_dtype);
    const int ve = unit_elems(p.table, p.table_ld, in, p.out, p.out_ld, out, p.dim);
    if (in == 4 && out == 4) lookup_tt<float, float>(p, ve, s);
    else if (in == 4) lookup_tt<float, bf16>(p, ve, s);
    else if (out == 4) lookup_tt<bf16, float>(p, ve, s);
    else lookup_tt<bf16, bf16>(p, ve, s);
    count_launches(1);
    return cudaGetLastError();
}

// ---------------------------------------------------------------- gradient
constexpr int ES_CHUNK = 256;       // entries of one run summed by one group of lanes
constexpr int ES_UNROLL = 4;        // rows in flight per lane
constexpr int ES_ROWS = 4;          // rows a group of lanes takes at a time
constexpr int ES_THREADS = 256;
constexpr int HEAD_TILE = 1024;

struct RunSum {
    EmbedGrad g;
    const int32_t* order;           // positions in the order of their ids
    const int32_t* starts;          // row r's entries are order[starts[r] .. starts[r + 1])
    Count rows;                     // dense: the table's rows; sparse: the runs (device) of at most n
    int tl;                         // lanes per row (power of two)
    int32_t* words;                 // [0] chunks, [1] long rows
    int2* items;                    // chunk -> (row, chunk of the row)
    int4* longs;                    // long row -> (row, first chunk, chunks, -)
    float* partial;                 // [chunks][dim]
};

// Sum of the entries [b, e) at columns c .. c + VE of dout, in ascending position.
template <typename Tin, int VE>
__device__ __forceinline__ void run_sum(const RunSum& P, int b, int e, int col, float (&acc)[VE]) {
    const Tin* dout = (const Tin*)P.g.dout + col;
#pragma unroll
    for (int i = 0; i < VE; ++i) acc[i] = 0.f;
    int k = b;
    for (; k + ES_UNROLL <= e; k += ES_UNROLL) {
        Raw<Tin, VE> v[ES_UNROLL];
#pragma unroll
        for (int j = 0; j < ES_UNROLL; ++j) v[j] = load_raw_stream<Tin, VE>(dout + (int64_t)__ldcg(P.order + k + j) * P.g.dout_ld);
#pragma unroll
        for (int j = 0; j < ES_UNROLL; ++j) {
            float x[VE];
            unpack<Tin, VE>(v[j], x);
#pragma unroll
            for (int i = 0; i < VE; ++i) acc[i] += x[i];
        }
    }
    for (; k < e; ++k) {
        float x[VE];
        unpack<Tin, VE>(load_raw_stream<Tin, VE>(dout + (int64_t)__ldcg(P.order + k) * P.g.dout_ld), x);
#pragma unroll
        for (int i = 0; i < VE; ++i) acc[i] += x[i];
    }
}

// Most rows have one entry or none, so a group of lanes takes ES_ROWS neighbouring rows at a time: their offsets, first
// positions and first rows are each in flight together.
template <typename Tin, typename Tout, int VE>
__global__ void __launch_bounds__(ES_THREADS) k_run_sum(RunSum P) {
    chain_wait();
    const int rows = list_length(P.rows), bound = P.rows.bound;
    const int units = P.g.dim / VE, t = threadIdx.x & (P.tl - 1);
    const int per_block = ES_THREADS / P.tl;
    const Tin* dout = (const Tin*)P.g.dout;
    Tout* grad = (Tout*)P.g.grad;
    for (int64_t r = ((int64_t)blockIdx.x * per_block + threadIdx.x / P.tl) * ES_ROWS; r < bound; r += (int64_t)gridDim.x * per_block * ES_ROWS) {
        int b[ES_ROWS + 1], first[ES_ROWS];
#pragma unroll
        for (int j = 0; j <= ES_ROWS; ++j) b[j] = __ldcg(P.starts + (r + j < rows ? r + j : rows));      // behind the last row: empty
#pragma unroll
        for (int j = 0; j < ES_ROWS; ++j) first[j] = b[j + 1] > b[j] ? __ldcg(P.order + b[j]) : -1;
        bool listed[ES_ROWS];
#pragma unroll
        for (int j = 0; j < ES_ROWS; ++j) {
            const int len = b[j + 1] - b[j];
            listed[j] = len > ES_CHUNK;
            if (listed[j] && t == 0) {
                const int nc = (len + ES_CHUNK - 1) / ES_CHUNK;
                const int at = atomicAdd(P.words, nc);
                P.longs[atomicAdd(P.words + 1, 1)] = make_int4((int)(r + j), at, nc, 0);
                for (int c = 0; c < nc; ++c) P.items[at + c] = make_int2((int)(r + j), c);
            }
        }
        for (int u = t; u < units; u += P.tl) {
            Raw<Tin, VE> v[ES_ROWS];
#pragma unroll
            for (int j = 0; j < ES_ROWS; ++j)
                v[j] = first[j] >= 0 && !listed[j] ? load_raw_stream<Tin, VE>(dout + (int64_t)first[j] * P.g.dout_ld + (int64_t)u * VE) : zero_raw<Tin, VE>();
#pragma unroll
            for (int j = 0; j < ES_ROWS; ++j) {
                if (r + j >= bound || listed[j]) continue;
                float acc[VE];
                unpack<Tin, VE>(v[j], acc);
                if (b[j + 1] - b[j] > 1) {
                    float more[VE];
                    run_sum<Tin, VE>(P, b[j] + 1, b[j + 1], u * VE, more);
#pragma unroll
                    for (int i = 0; i < VE; ++i) acc[i] += more[i];
                }
                if (first[j] >= 0) {
#pragma unroll
                    for (int i = 0; i < VE; ++i) acc[i] *= P.g.scale;
                }
                store_vec<Tout, VE>(grad + (r + j) * P.g.grad_ld + (int64_t)u * VE, acc);
            }
        }
    }
}

template <typename Tin, int VE>
__global__ void __launch_bounds__(ES_THREADS) k_run_chunks(RunSum P) {
    chain_wait();
    const int chunks = __ldcg(P.words);
    const int units = P.g.dim / VE, t = threadIdx.x & (P.tl - 1);
    const int per_block = ES_THREADS / P.tl;
    for (int64_t c = (int64_t)blockIdx.x * per_block + threadIdx.x / P.tl; c < chunks; c += (int64_t)gridDim.x * per_block) {
        const int2 it = P.items[c];
        const int b = __ldcg(P.starts + it.x) + it.y * ES_CHUNK;
        const int end = __ldcg(P.starts + it.x + 1), e = b + ES_CHUNK < end ? b + ES_CHUNK : end;
        for (int u = t; u < units; u += P.tl) {
            float acc[VE];
            run_sum<Tin, VE>(P, b, e, u * VE, acc);
#pragma unroll
            for (int i = 0; i < VE; ++i) P.partial[c * P.g.dim + u * VE + i] = acc[i];
        }
    }
}

// One block per (long row, 32 columns): each warp adds a contiguous share of the chunks, the shares are added in order.
template <typename Tout>
__global__ void __launch_bounds__(ES_THREADS) k_run_join(RunSum P) {
    constexpr int W = ES_THREADS / 32;
    __shared__ float share[W][32];
    chain_wait();
    const int longs = __ldcg(P.words + 1), lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const int ctiles = (P.g.dim + 31) / 32;
    Tout* grad = (Tout*)P.g.grad;
    for (int64_t i = blockIdx.x; i < (int64_t)longs * ctiles; i += gridDim.x) {
        const int4 l = P.longs[i / ctiles];
        const int col = (int)(i % ctiles) * 32 + lane;
        const int per = (l.z + W - 1) / W, c0 = wid * per, c1 = c0 + per < l.z ? c0 + per : l.z;
        float acc = 0.f;
        if (col < P.g.dim) {
            const float* p = P.partial + (int64_t)l.y * P.g.dim + col;
#pragma unroll 4
            for (int c = c0; c < c1; ++c) acc += __ldcg(p + (int64_t)c * P.g.dim);
        }
        share[wid][lane] = acc;
        __syncthreads();
        if (wid == 0 && col < P.g.dim) {
            for (int w = 1; w < W; ++w) acc += share[w][lane];
            grad[(int64_t)l.x * P.g.grad_ld + col] = from_f32<Tout>(acc * P.g.scale);
        }
        __syncthreads();
    }
}

// Heads of runs of equal ids per tile of the sorted list ...
__global__ void __launch_bounds__(HEAD_TILE) k_head_counts(const uint32_t* __restrict__ keys, Count nc, uint32_t limit,
                                                           int32_t* __restrict__ tile_heads) {
    chain_wait();
    const int n = list_length(nc);
    const int tiles = (nc.bound + HEAD_TILE - 1) / HEAD_TILE;
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t i = (int64_t)tile * HEAD_TILE + threadIdx.x;
        bool head = false;
        if (i < n) {
            const uint32_t k = __ldcg(keys + i);
            head = k < limit && (i == 0 || __ldcg(keys + i - 1) != k);
        }
        const int c = __syncthreads_count(head);
        if (threadIdx.x == 0) tile_heads[tile] = c;
    }
}

// ... and the list of runs: id and first entry of each; -1 behind the last one.
__global__ void __launch_bounds__(HEAD_TILE) k_head_list(const uint32_t* __restrict__ keys, Count nc, uint32_t limit,
                                                         const int32_t* __restrict__ tile_heads, int32_t* __restrict__ rows,
                                                         int32_t* __restrict__ starts, int32_t* __restrict__ d_num_rows) {
    __shared__ int warp_sums[33];
    chain_wait();
    const int n = list_length(nc);
    const int tiles = (nc.bound + HEAD_TILE - 1) / HEAD_TILE;
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        int mine = 0, all = 0;
        for (int t = threadIdx.x; t < tiles; t += HEAD_TILE) {
            const int c = __ldcg(tile_heads + t);
            all += c;
            if (t < tile) mine += c;
        }
        int before, runs, total;
        block_exclusive_scan<HEAD_TILE>(mine, warp_sums, &before);
        block_exclusive_scan<HEAD_TILE>(all, warp_sums, &runs);
        const int64_t i = (int64_t)tile * HEAD_TILE + threadIdx.x;
        bool head = false, valid = false;
        uint32_t k = 0;
        if (i < n) {
            k = __ldcg(keys + i);
            valid = k < limit;
            head = valid && (i == 0 || __ldcg(keys + i - 1) != k);
        }
        const int at = before + block_exclusive_scan<HEAD_TILE>(head ? 1 : 0, warp_sums, &total);
        if (head) {
            rows[at] = (int32_t)k;
            starts[at] = (int32_t)i;
        }
        // the end of the last run: where the valid entries end
        if (valid && (i + 1 == n || __ldcg(keys + i + 1) >= limit)) starts[runs] = (int32_t)i + 1;
        if (i >= runs && i < nc.bound) rows[i] = -1;
        if (tile == 0 && threadIdx.x == 0) {
            *d_num_rows = runs;
            if (runs == 0) starts[0] = 0;
        }
        __syncthreads();
    }
}

struct EmbedLayout {
    size_t sort, keys, order, starts, words, items, longs, partial, total;
    int64_t chunks, long_rows;
};

static EmbedLayout embed_layout(int64_t n, int64_t table_rows, int32_t dim) {
    EmbedLayout l{};
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t o = off; off = align_up(off + bytes, 256); return o; };
    l.sort = take(key_sort_bytes(n));
    l.keys = take((size_t)n * 4);
    l.order = take((size_t)n * 4);
    const int64_t rows = (table_rows > n ? table_rows : n) + 1;       // dense: per table row; sparse: per run
    l.starts = take((size_t)rows * 4);
    l.words = take(256 + ((size_t)n / HEAD_TILE + 1) * 4);
    l.long_rows = n / ES_CHUNK + 1;
    l.chunks = 2 * (n / ES_CHUNK) + 2;
    l.items = take((size_t)l.chunks * 8);
    l.longs = take((size_t)l.long_rows * 16);
    l.partial = take((size_t)l.chunks * dim * 4);
    l.total = off;
    return l;
}

size_t embedding_workspace(int64_t n, int64_t table_rows, int32_t dim) { return embed_layout(n, table_rows, dim).total; }

template <typename Tin, typename Tout, int VE> static cudaError_t run_sum_t(RunSum& P, cudaStream_t s) {
    const int units = P.g.dim / VE;
    P.tl = 1;
    while (P.tl < 32 && P.tl < units) P.tl *= 2;
    const int per_block = ES_THREADS / P.tl * ES_ROWS;
    int64_t blocks = ((int64_t)P.rows.bound + per_block - 1) / per_block;
    if (blocks > sm_count() * 256) blocks = sm_count() * 256;
    cudaError_t e = launch_train(k_run_sum<Tin, Tout, VE>, blocks, ES_THREADS, 0, s, P);
    if (P.g.n.bound <= ES_CHUNK || e != cudaSuccess) return e;           // no run can be longer than a chunk
    e = launch_train(k_run_chunks<Tin, VE>, sm_count() * 8, ES_THREADS, 0, s, P);
    if (e == cudaSuccess) e = launch_train(k_run_join<Tout>, sm_count() * 4, ES_THREADS, 0, s, P);
    return e;
}

template <typename Tin, typename Tout> static cudaError_t run_sum_tt(RunSum& P, int ve, cudaStream_t s) {
    if constexpr (sizeof(Tin) == 2) {
        if (ve == 8) return run_sum_t<Tin, Tout, 8>(P, s);
    }
    if (ve == 4) return run_sum_t<Tin, Tout, 4>(P, s);
    if (ve == 2) return run_sum_t<Tin, Tout, 2>(P, s);
    return run_sum_t<Tin, Tout, 1>(P, s);
}

cudaError_t launch_embedding_grad(const EmbedGrad& g, void* workspace, cudaStream_t s) {
    const EmbedLayout l = embed_layout(g.n.bound, g.table_rows, g.dim);
    char* ws = (char*)workspace;
    RunSum P{};
    P.g = g;
    P.words = (int32_t*)(ws + l.words);
    P.items = (int2*)(ws + l.items);
    P.longs = (int4*)(ws + l.longs);
    P.partial = (float*)(ws + l.partial);
    uint32_t* keys = (uint32_t*)(ws + l.keys);
    int32_t* order = (int32_t*)(ws + l.order);
    int32_t* starts = (int32_t*)(ws + l.starts);
    P.order = order;
    P.starts = starts;
    cudaError_t e = cudaMemsetAsync(P.words, 0, 8, s);
    if (e == cudaSuccess) e = launch_key_sort(g.ids, nullptr, g.n, g.table_rows, ws + l.sort, keys, order, s);
    if (e != cudaSuccess) return e;
    if (g.rows) {
        int32_t* heads = P.words + 64;
        const int64_t tiles = ((int64_t)g.n.bound + HEAD_TILE - 1) / HEAD_TILE;
        const int64_t grid = tiles < sm_count() * 2 ? tiles : sm_count() * 2;
        e = launch_train(k_head_counts, grid, HEAD_TILE, 0, s, keys, g.n, (uint32_t)g.table_rows, heads);
        if (e == cudaSuccess) e = launch_train(k_head_list, grid, HEAD_TILE, 0, s, keys, g.n, (uint32_t)g.table_rows, heads, g.rows, starts, g.d_num_rows);
        P.rows = Count{g.d_num_rows, g.n.bound};
    } else {
        P.rows = Count{nullptr, (int32_t)g.table_rows};
        e = launch_row_starts(keys, g.n, P.rows, starts, s);
    }
    if (e != cudaSuccess) return e;
    const int in = bytes_of(g.dout_dtype), out = bytes_of(g.grad_dtype);
    const int ve = unit_elems(g.dout, g.dout_ld, in, g.grad, g.grad_ld, out, g.dim);
    if (in == 4 && out == 4) return run_sum_tt<float, float>(P, ve, s);
    if (in == 4) return run_sum_tt<float, bf16>(P, ve, s);
    if (out == 4) return run_sum_tt<bf16, float>(P, ve, s);
    return run_sum_tt<bf16, bf16>(P, ve, s);
}

}  // namespace gs
