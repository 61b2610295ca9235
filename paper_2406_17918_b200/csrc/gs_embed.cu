// Embedding rows: out[p] = scale * table[ids[p]], and the gradient of the table.
//
// The gradient of row r is scale * (sum of the rows dout[p] with ids[p] = r): the positions are sorted by id (stable,
// gs_sort.cu; for 2.03 M ids below 2^26 about 100 of the 325 us), the rows of a run are added in ascending position in 32 bits and rounded once.  No atomics on
// floats: the result does not depend on the schedule.  Runs of up to ES_CHUNK entries are summed by the group of
// lanes that meets their head; a longer run (a hub) is cut into chunks whose sums go to the workspace and are added in order.
#include "gs_device.cuh"
#include "gs_train.cuh"
#include "gs_train.h"

namespace gs {

constexpr int EL_THREADS = 256;
constexpr int EL_FLIGHT = 4;    // loads in flight per thread of the lookup: over rows, or over the units of one row

__device__ __forceinline__ int list_length(const Count& c) {
    if (!c.d_n) return c.bound;
    const int n = __ldcg(c.d_n);      // may be the work of the kernel before
    return n < 0 ? 0 : (n > c.bound ? c.bound : n);
}

// out[p] = scale * table[ids[p]].  Bound by the rows' bytes; neighbouring threads take neighbouring units of a row, in the widest
// load that divides it.  A thread takes ROWS rows at a time, or, where rows are few and long, COLS units of one row:
// 2.03 M rows of 128 bf16 in 177 us (5.9 TB/s with the ids).
template <typename Tin, typename Tout, int VE, int ROWS, int COLS>
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
    for (int64_t row = (int64_t)blockIdx.x * rows_per_iter + r_in; row < n; row += step * ROWS) {
        int32_t id[ROWS];
#pragma unroll
        for (int j = 0; j < ROWS; ++j) {
            const int64_t rj = row + j * step;
            id[j] = rj < n ? __ldg(P.ids + rj) : -1;
        }
        for (int u = u0; u < units; u += tpr * COLS) {
            Raw<Tin, VE> v[ROWS * COLS];
#pragma unroll
            for (int j = 0; j < ROWS; ++j)
#pragma unroll
                for (int c = 0; c < COLS; ++c)
                    v[j * COLS + c] = (uint32_t)id[j] < (uint32_t)P.table_rows && u + c * tpr < units
                                          ? load_raw_stream<Tin, VE>(table + (int64_t)id[j] * P.table_ld + (int64_t)(u + c * tpr) * VE)
                                          : zero_raw<Tin, VE>();
#pragma unroll
            for (int j = 0; j < ROWS; ++j) {
                const int64_t rj = row + j * step;
                if (rj >= n) continue;
                const bool in = (uint32_t)id[j] < (uint32_t)P.table_rows;
#pragma unroll
                for (int c = 0; c < COLS; ++c) {
                    if (u + c * tpr >= units) continue;
                    float x[VE];
                    unpack<Tin, VE>(v[j * COLS + c], x);
#pragma unroll
                    for (int i = 0; i < VE; ++i) x[i] = in ? x[i] * P.scale : 0.f;     // a row outside the table is zero whatever the scale
                    store_vec<Tout, VE>(out + rj * P.out_ld + (int64_t)(u + c * tpr) * VE, x);
                }
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
    const int64_t groups = ((int64_t)p.n.bound + rpi - 1) / rpi;      // blocks' worth of rows
    int64_t blocks = (groups + EL_FLIGHT - 1) / EL_FLIGHT;
    // Rows longer than a block, and too few of them to fill the device four at a time:
    // 300 rows of 1,433 bf16 8 us this way, 18 four rows at a time, 1,100 rows 12 | 18, 4,700 rows 25 | 22.
    const bool few = units > EL_THREADS && blocks < sm_count() * 4;
    if (few) blocks = groups;
    if (blocks > sm_count() * 64) blocks = sm_count() * 64;
    if (few) k_embed_lookup<Tin, Tout, VE, 1, EL_FLIGHT><<<(int)limit_grid(blocks), EL_THREADS, 0, s>>>(p);
    else k_embed_lookup<Tin, Tout, VE, EL_FLIGHT, 1><<<(int)limit_grid(blocks), EL_THREADS, 0, s>>>(p);
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
constexpr int ES_CHUNK = 32;        // entries of one run summed by the group of lanes that meets its head
constexpr int ES_UNROLL = 8;        // rows in flight per lane
constexpr int ES_THREADS = 256;
constexpr int ES_TILE = ES_THREADS; // sorted entries per block of the sums

struct RunSum {
    EmbedGrad g;
    const uint32_t* keys;           // ids, ascending (table_rows stands for ids outside the table)
    const int32_t* order;           // their positions
    const int32_t* tile_runs;       // sparse: runs before each tile of the list
    int tl;                         // lanes per row (a power of two)
    int seg;                        // sorted entries per group, at most tl
    int32_t* words;                 // [0] chunks, [1] long runs
    int2* items;                    // chunk -> entries [x, y)
    int4* longs;                    // long run -> (row of the gradient, first chunk, chunks, -)
    float* partial;                 // [chunks][dim]
};

// First entry behind the run of `key` that entry e belongs to.
__device__ __forceinline__ int run_end(const uint32_t* keys, int e, int n, uint32_t key) {
    int lo = e, step = ES_CHUNK;                       // keys[lo] == key; double the step, then halve it
    while (lo + step < n && __ldcg(keys + lo + step) == key) {
        lo += step;
        step *= 2;
    }
    for (; step > 0; step >>= 1)
        while (lo + step < n && __ldcg(keys + lo + step) == key) lo += step;
    return lo + 1;
}

// A hub's run is listed for the chunk kernel.
__device__ __forceinline__ void list_run(const RunSum& P, int row, int b, int e) {
    const int nc = (e - b + ES_CHUNK - 1) / ES_CHUNK;
    const int at = atomicAdd(P.words, nc);
    P.longs[atomicAdd(P.words + 1, 1)] = make_int4(row, at, nc, 0);
    for (int c = 0; c < nc; ++c) P.items[at + c] = make_int2(b + c * ES_CHUNK, b + (c + 1) * ES_CHUNK < e ? b + (c + 1) * ES_CHUNK : e);
}

// Adds the entries [b, e) at columns col .. col + VE of dout in ascending position.
template <typename Tin, int VE>
__device__ __forceinline__ void add_entries(const RunSum& P, int b, int e, int64_t col, float (&acc)[VE]) {
    const Tin* dout = (const Tin*)P.g.dout + col;
    constexpr int U = ES_UNROLL;
    int k = b;
    for (; k + U <= e; k += U) {
        Raw<Tin, VE> v[U];
#pragma unroll
        for (int j = 0; j < U; ++j) v[j] = load_raw_stream<Tin, VE>(dout + (int64_t)__ldcg(P.order + k + j) * P.g.dout_ld);
#pragma unroll
        for (int j = 0; j < U; ++j) {
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

// The sorted entries, in equal pieces: a group of tl lanes takes `seg` neighbouring entries, whose rows are all in flight
// whatever runs they belong to, and owns the runs whose heads it meets (the last one beyond its own entries, if it
// continues).  Work by entries, not by rows: rows of the table are many and mostly empty, and the frequent ids lie together.
// Bound by the rows' bytes: 2.03 M rows of 128 bf16 in 185 us (0.87 of the copy rate with the rows written), 41 k rows of 128 f32
// in 13 us.  A block takes ES_THREADS / tl * seg entries: all of a tile of ES_THREADS when seg = tl, fewer of it where there are too
// few entries to fill the device that way.
template <typename Tin, typename Tout, int VE, bool SPARSE>
__global__ void __launch_bounds__(ES_THREADS, 4) k_run_sum(RunSum P) {
    __shared__ int warp_sums[33];
    __shared__ int s_key[ES_THREADS], s_pos[ES_THREADS], s_row[ES_THREADS];
    __shared__ unsigned char s_flag[ES_THREADS];            // 1: head, 2: of a listed run, 4: an entry with an id
    chain_wait();
    const int n = list_length(P.g.n), bound = P.g.n.bound;
    const uint32_t limit = (uint32_t)P.g.table_rows;
    const int tiles = (bound + ES_TILE - 1) / ES_TILE;
    const int tl = P.tl, t = threadIdx.x & (tl - 1), seg = P.seg, parts = tl / seg;      // blocks per tile
    const int units = P.g.dim / VE;
    const Tin* dout = (const Tin*)P.g.dout;
    for (int64_t bt = blockIdx.x; bt < (int64_t)tiles * parts; bt += gridDim.x) {
        const int tile = (int)(bt / parts), part = (int)(bt - (int64_t)tile * parts);
        const int before = SPARSE ? __ldcg(P.tile_runs + tile) : 0, runs = SPARSE ? __ldcg(P.g.d_num_rows) : 0;
        {
            const int64_t e64 = (int64_t)tile * ES_TILE + threadIdx.x;
            const int e = e64 < bound ? (int)e64 : bound;
            uint32_t key = limit;
            int pos = 0;
            bool head = false;
            if (e < n) {
                key = __ldcg(P.keys + e);
                pos = __ldcg(P.order + e);
                head = key < limit && (e == 0 || __ldcg(P.keys + e - 1) != key);
            }
            int row = (int)key;
            if (SPARSE) {
                int total;
                row = before + block_exclusive_scan<ES_THREADS>(head ? 1 : 0, warp_sums, &total);
                if (part == 0) {
                    if (head) P.g.rows[row] = (int32_t)key;
                    if (e >= runs && e < bound) P.g.rows[e] = -1;
                }
            }
            const bool listed = head && e + ES_CHUNK < n && __ldcg(P.keys + e + ES_CHUNK) == key;
            if (listed && part == 0) list_run(P, row, e, run_end(P.keys, e, n, key));
            __syncthreads();
            s_key[threadIdx.x] = (int)key;
            s_pos[threadIdx.x] = pos;
            s_row[threadIdx.x] = row;
            s_flag[threadIdx.x] = (head ? 1 : 0) | (listed ? 2 : 0) | (key < limit ? 4 : 0);
            __syncthreads();
        }
        // this group's entries of the tile: seg of them, the parts of a tile interleaved
        const int first = (part * (ES_THREADS / tl) + threadIdx.x / tl) * seg;
        for (int u = t; u < units; u += tl) {
            const int64_t col = (int64_t)u * VE;
            float acc[VE];
#pragma unroll
            for (int i = 0; i < VE; ++i) acc[i] = 0.f;
            int open = -1;                                             // entry of the head of the run being summed
            auto flush = [&]() {
#pragma unroll
                for (int i = 0; i < VE; ++i) acc[i] *= P.g.scale;
                store_vec<Tout, VE>((Tout*)P.g.grad + (int64_t)s_row[open] * P.g.grad_ld + col, acc);
                open = -1;
            };
            bool skip = true;                                          // entries of a run met before, or listed
            for (int j0 = 0; j0 < seg; j0 += ES_UNROLL) {
                Raw<Tin, VE> v[ES_UNROLL];
                bool mine = !skip;
#pragma unroll
                for (int j = 0; j < ES_UNROLL; ++j) {
                    const int l = first + j0 + j, flag = j0 + j < seg ? s_flag[l] : 0;
                    if (flag & 1) mine = !(flag & 2);
                    v[j] = mine && (flag & 4) ? load_raw_stream<Tin, VE>(dout + (int64_t)s_pos[l] * P.g.dout_ld + col) : zero_raw<Tin, VE>();
                }
#pragma unroll
                for (int j = 0; j < ES_UNROLL; ++j) {
                    const int l = first + j0 + j, flag = j0 + j < seg ? s_flag[l] : 4;
                    const bool starts = flag & 1;
                    if ((starts || !(flag & 4)) && open >= 0) flush();
                    float x[VE];
                    unpack<Tin, VE>(v[j], x);
#pragma unroll
                    for (int i = 0; i < VE; ++i) acc[i] = starts ? x[i] : acc[i] + x[i];
                    if (starts) {
                        skip = flag & 2;
                        open = skip ? -1 : l;
                    }
                }
            }
            if (open >= 0) {
                const int from = tile * ES_TILE + first + seg;         // behind the group's entries
                const uint32_t key = (uint32_t)s_key[open];
                int to = from;
                while (to < n && to - from < ES_CHUNK && __ldcg(P.keys + to) == key) ++to;
                if (to > from) add_entries<Tin, VE>(P, from, to, col, acc);
                flush();
            }
        }
        if (SPARSE) {                                                  // rows behind the last run
            const int64_t f0 = (int64_t)tile * ES_TILE, end = f0 + ES_TILE < bound ? f0 + ES_TILE : bound;
            const float zero[VE] = {};
            for (int64_t r = (f0 > runs ? f0 : runs) + part * (ES_THREADS / tl) + threadIdx.x / tl; r < end; r += (ES_THREADS / tl) * parts)
                for (int u = t; u < units; u += tl) store_vec<Tout, VE>((Tout*)P.g.grad + r * P.g.grad_ld + (int64_t)u * VE, zero);
        }
    }
}

// The listed runs, ES_CHUNK entries at a time: a group of lanes per chunk, sixteen rows in flight (14 us beside 2.03 M
// ids by a squared law, 9 us beside 41 k).
template <typename Tin, int VE>
__global__ void __launch_bounds__(ES_THREADS) k_run_chunks(RunSum P) {
    chain_wait();
    const int chunks = __ldcg(P.words);
    constexpr int CHUNK_UNROLL = 16;
    const int units = P.g.dim / VE, t = threadIdx.x & (P.tl - 1), base = threadIdx.x & 31 & ~(P.tl - 1);
    const uint32_t group = P.tl == 32 ? FULL : ((1u << P.tl) - 1u) << base;
    const int per_block = ES_THREADS / P.tl;
    for (int64_t c = (int64_t)blockIdx.x * per_block + threadIdx.x / P.tl; c < chunks; c += (int64_t)gridDim.x * per_block) {
        const int2 it = P.items[c];
        const Tin* dout = (const Tin*)P.g.dout;
        // positions by lane, tl at a time, then as many rows in flight as fit
        for (int u = t; u < units + t; u += P.tl) {                   // the same number of turns for all lanes of the group
            const int64_t col = (int64_t)u * VE;
            const bool on = u < units;
            float acc[VE];
#pragma unroll
            for (int i = 0; i < VE; ++i) acc[i] = 0.f;
            for (int b = it.x; b < it.y; b += P.tl) {
                const int pos = b + t < it.y ? __ldcg(P.order + b + t) : 0;
                for (int j0 = 0; j0 < P.tl && b + j0 < it.y; j0 += CHUNK_UNROLL) {
                    Raw<Tin, VE> v[CHUNK_UNROLL];
#pragma unroll
                    for (int j = 0; j < CHUNK_UNROLL; ++j) {
                        const int p = __shfl_sync(group, pos, base + ((j0 + j) & (P.tl - 1)));
                        v[j] = on && j0 + j < P.tl && b + j0 + j < it.y ? load_raw_stream<Tin, VE>(dout + (int64_t)p * P.g.dout_ld + col) : zero_raw<Tin, VE>();
                    }
#pragma unroll
                    for (int j = 0; j < CHUNK_UNROLL; ++j) {
                        float x[VE];
                        unpack<Tin, VE>(v[j], x);
#pragma unroll
                        for (int i = 0; i < VE; ++i) acc[i] += x[i];
                    }
                }
            }
            if (on) {
#pragma unroll
                for (int i = 0; i < VE; ++i) P.partial[c * P.g.dim + u * VE + i] = acc[i];
            }
        }
    }
}

// One block per (long row, 32 columns), 4 us: each warp adds a contiguous share of the chunks, the shares are added in order.
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
__global__ void __launch_bounds__(ES_THREADS) k_head_counts(const uint32_t* __restrict__ keys, Count nc, uint32_t limit,
                                                            int32_t* __restrict__ tile_runs) {
    chain_wait();
    const int n = list_length(nc), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int tiles = (nc.bound + ES_TILE - 1) / ES_TILE;
    // a warp per tile
    for (int tile = blockIdx.x * (ES_THREADS / 32) + warp; tile < tiles; tile += gridDim.x * (ES_THREADS / 32)) {
        int c = 0;
#pragma unroll
        for (int j = 0; j < ES_TILE; j += 32) {
            const int64_t i = (int64_t)tile * ES_TILE + j + lane;
            const uint32_t k = i < n ? __ldcg(keys + i) : limit;
            uint32_t prev = __shfl_up_sync(FULL, k, 1);
            if (lane == 0) prev = i > 0 && i < n ? __ldcg(keys + i - 1) : 0xFFFFFFFFu;
            c += __popc(__ballot_sync(FULL, k < limit && k != prev));
        }
        if (lane == 0) tile_runs[tile] = c;
    }
}

// ... and the runs before each tile, and in all.
__global__ void __launch_bounds__(1024) k_head_scan(int tiles, int32_t* __restrict__ tile_runs, int32_t* __restrict__ d_num_rows) {
    __shared__ int warp_sums[33];
    chain_wait();
    constexpr int PER = 8;
    int carry = 0;
    for (int base = 0; base < tiles; base += 1024 * PER) {
        int c[PER], sum = 0, total;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int i = base + (int)threadIdx.x * PER + j;
            c[j] = i < tiles ? __ldcg(tile_runs + i) : 0;
            sum += c[j];
        }
        int at = carry + block_exclusive_scan<1024>(sum, warp_sums, &total);
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int i = base + (int)threadIdx.x * PER + j;
            if (i < tiles) tile_runs[i] = at;
            at += c[j];
        }
        carry += total;
    }
    if (threadIdx.x == 0) *d_num_rows = carry;
}

struct EmbedLayout {
    size_t sort, keys, order, heads, words, items, longs, partial, total;
};

static EmbedLayout embed_layout(int64_t n, int32_t dim) {
    EmbedLayout l{};
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t o = off; off = align_up(off + bytes, 256); return o; };
    l.sort = take(key_sort_bytes(n));
    l.keys = take((size_t)n * 4);
    l.order = take((size_t)n * 4);
    l.heads = take(((size_t)n / ES_TILE + 1) * 4);
    l.words = take(256);
    const int64_t chunks = 2 * (n / ES_CHUNK) + 2;       // a listed run has more than ES_CHUNK entries
    l.items = take((size_t)chunks * 8);
    l.longs = take((size_t)(n / ES_CHUNK + 1) * 16);
    l.partial = take((size_t)chunks * dim * 4);
    l.total = off;
    return l;
}

size_t embedding_workspace(int64_t n, int64_t, int32_t dim) { return embed_layout(n, dim).total; }

template <typename Tin, typename Tout, int VE> static cudaError_t run_sum_t(RunSum& P, cudaStream_t s) {
    const int units = P.g.dim / VE;
    P.tl = 1;
    while (P.tl < 32 && P.tl < units) P.tl *= 2;
    int64_t tiles = ((int64_t)P.g.n.bound + ES_TILE - 1) / ES_TILE;
    P.seg = P.tl;
    while (P.seg > 4 && tiles < sm_count() * 4) {        // four blocks per SM, as long as a group keeps four entries
        P.seg /= 2;
        tiles *= 2;
    }
    cudaError_t e = P.g.rows ? launch_train(k_run_sum<Tin, Tout, VE, true>, tiles, ES_THREADS, 0, s, P)
                             : launch_train(k_run_sum<Tin, Tout, VE, false>, tiles, ES_THREADS, 0, s, P);
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
    const EmbedLayout l = embed_layout(g.n.bound, g.dim);
    char* ws = (char*)workspace;
    RunSum P{};
    P.g = g;
    P.words = (int32_t*)(ws + l.words);
    P.items = (int2*)(ws + l.items);
    P.longs = (int4*)(ws + l.longs);
    P.partial = (float*)(ws + l.partial);
    uint32_t* keys = (uint32_t*)(ws + l.keys);
    int32_t* order = (int32_t*)(ws + l.order);
    int32_t* heads = (int32_t*)(ws + l.heads);
    P.keys = keys;
    P.order = order;
    P.tile_runs = heads;
    const int in = bytes_of(g.dout_dtype), out = bytes_of(g.grad_dtype);
    cudaError_t e = cudaSuccess;
    // the dense table is cleared first: rows without an id stay so
    Fill fill{};
    if (!g.rows) {
        const size_t bytes = (size_t)g.table_rows * g.dim * out;
        if (g.grad_ld == g.dim && (uintptr_t)g.grad % 16 == 0 && bytes >= 16) fill = Fill{(uint4*)g.grad, (int64_t)(bytes / 16), (int)(bytes % 16)};
        else e = cudaMemset2DAsync(g.grad, (size_t)g.grad_ld * out, 0, (size_t)g.dim * out, (size_t)g.table_rows, s);
    }
    if (e == cudaSuccess) e = launch_key_sort(g.ids, nullptr, g.n, Rows{}, g.table_rows, ws + l.sort, keys, order, P.words, 2, fill, s);
    if (e == cudaSuccess && g.rows) {
        const int tiles = (int)(((int64_t)g.n.bound + ES_TILE - 1) / ES_TILE);
        e = launch_train(k_head_counts, (tiles + ES_THREADS / 32 - 1) / (ES_THREADS / 32), ES_THREADS, 0, s, keys, g.n, (uint32_t)g.table_rows, heads);
        if (e == cudaSuccess) e = launch_train(k_head_scan, 1, 1024, 0, s, tiles, heads, g.d_num_rows);
    }
    if (e != cudaSuccess) return e;
    const int ve = unit_elems(g.dout, g.dout_ld, in, g.grad, g.grad_ld, out, g.dim);
    if (in == 4 && out == 4) return run_sum_tt<float, float>(P, ve, s);
    if (in == 4) return run_sum_tt<float, bf16>(P, ve, s);
    if (out == 4) return run_sum_tt<bf16, float>(P, ve, s);
    return run_sum_tt<bf16, bf16>(P, ve, s);
}

}  // namespace gs
