// Rows kept in 8 bits: written by node id or as a range, with one scale per block of rows and head, and read back.
//
//   code = e4m3(x / s),  s = 2^e the smallest with |x| <= 448 s over the block's rows of a head;  read: s code.
//
// A write changes some rows of a block.  If it leaves others, the block's scale never falls: it is raised where the new rows need
// it, and the codes that stay are brought to it.  One warp does all of a block, so nobody else sees it half written.  Which row wins
// where an id occurs twice is settled by a pass of integer maxima before (claims: the highest position), which also lists the
// blocks that are written; the order of the list does not show in the result.  The kernels move bytes and little else: 2.03 M rows of 8 x 32
// read by id as bf16 255 us (1.04 GB written, what L2 misses of 0.5 GB read: 0.93 of a copy's rate).  262,144 rows written by id into blocks of
// 16 of 2.4 M: 100 us where no scale rises (191 MB of DRAM traffic), 160 where those of 16,418 of the 128,317 blocks do (250 MB).  That is
// latency, not bytes (warps active 36 %, issue slots 50 %): a block's place in the list, its claims, its scale and its rows are fetched one
// behind another.  As a range, bf16, 74 us: a block's rows are read once for its scale and once for its codes.
#include "gs_codes.cuh"
#include "gs_device.cuh"
#include "gs_train.h"

namespace gs {

constexpr int CD_THREADS = 256;

__device__ __forceinline__ int coded_count(const Count& c) {
    if (!c.d_n) return c.bound;
    const int n = __ldg(c.d_n);
    return n < 0 ? 0 : (n > c.bound ? c.bound : n);
}

// What a write by id keeps beside a store, all -1 between two writes: for every row the highest position that writes it; and, for
// blocks of several rows, for every block whether it is listed, the list of the blocks, its length and the blocks of threads that are done.
struct Claims {
    int32_t* rows;
    int32_t* listed;
    int32_t* list;
    int32_t* words;                  // [0] the list's last place, [1] threads' blocks done, less one
    __device__ __forceinline__ explicit Claims(const CodedWrite& P) {
        const int64_t blocks = (P.to.rows + (1 << P.to.shift) - 1) >> P.to.shift;
        rows = P.claims;
        listed = rows + P.to.rows;
        list = listed + blocks;
        words = list + blocks;
    }
};

__global__ void __launch_bounds__(CD_THREADS) k_coded_claim(const __grid_constant__ CodedWrite P) {
    chain_wait();
    const Claims K(P);
    __shared__ int s_count[CD_THREADS / 32], s_first;
    const int n = coded_count(P.n), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int64_t p0 = (int64_t)blockIdx.x * CD_THREADS; p0 < n; p0 += (int64_t)gridDim.x * CD_THREADS) {
        const int64_t p = p0 + threadIdx.x;
        const int id = p < n ? __ldg(P.ids + p) : -1;
        const bool in = id >= 0 && id < P.to.rows;
        if (in) atomicMax(K.rows + id, (int)p);
        if (!P.to.shift) continue;
        // places in the list, one addition for all threads
        const bool first = in && atomicExch(K.listed + (id >> P.to.shift), 0) < 0;
        const uint32_t who = __ballot_sync(FULL, first);
        __syncthreads();
        if (lane == 0) s_count[warp] = __popc(who);
        __syncthreads();
        if (threadIdx.x == 0) {
            int all = 0;
            for (int w = 0; w < CD_THREADS / 32; ++w) {
                const int c = s_count[w];
                s_count[w] = all;
                all += c;
            }
            s_first = all ? atomicAdd(K.words, all) + 1 : 0;
        }
        __syncthreads();
        if (first) K.list[s_first + s_count[warp] + __popc(who & ((1u << lane) - 1))] = id >> P.to.shift;
    }
}

// The largest finite magnitude of some elements, as the bits of an f32.  Infinities and NaN are looked for where they are met.
template <typename T, int VE> __device__ __forceinline__ uint32_t magnitude(const Raw<T, VE>& r) {
    uint32_t w[4], top = 0;
    constexpr int W = (int)sizeof(T) * VE / 4;
    if constexpr (W == 4) { w[0] = r.w.x; w[1] = r.w.y; w[2] = r.w.z; w[3] = r.w.w; }
    else if constexpr (W == 2) { w[0] = r.w.x; w[1] = r.w.y; }
    else w[0] = (uint32_t)r.w;
    if constexpr (sizeof(T) == 2) {
        // two at a time; the maximum passes NaN over
        __nv_bfloat162 two = __float2bfloat162_rn(0.f);
#pragma unroll
        for (int i = 0; i < (W ? W : 1); ++i) two = __hmax2(two, __habs2(*reinterpret_cast<const __nv_bfloat162*>(&w[i])));
        const uint32_t both = *reinterpret_cast<const uint32_t*>(&two);
        top = max(both & 0xFFFF0000u, both << 16);
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) top = max(top, w[i] & 0x7FFFFFFFu);
    }
    if (top < 0x7F800000u) return top;
    float x[VE];
    unpack<T, VE>(r, x);
    top = 0;
#pragma unroll
    for (int i = 0; i < VE; ++i) top = max(top, finite_magnitude(x[i]));
    return top;
}
template <typename T, int VE> __device__ __forceinline__ void put_codes(uint8_t* to, const Raw<T, VE>& r, float unscale) {
    float x[VE];
    unpack<T, VE>(r, x);
    *reinterpret_cast<typename CodeWord<VE>::type*>(to) = encode<VE>(x, unscale);
}

// The codes of a block's rows that stay, brought to a scale that is 2^steps larger; one head by tl lanes.
template <int VE> __device__ __forceinline__ void requantise(uint8_t* out, int64_t row_stride, uint64_t stays, uint32_t steps, int c0, int dim, int width) {
    using Word = typename CodeWord<VE>::type;
    constexpr int M = 4;
    const float ratio = steps < 64u ? scale_of(127u - steps) : 0.f;
    for (int c = c0; c < dim; c += width)
        for (uint64_t left = stays; left;) {
            Word w[M];
            uint8_t* at[M];
#pragma unroll
            for (int j = 0; j < M; ++j) {
                at[j] = left ? out + (int64_t)(__ffsll(left) - 1) * row_stride + c : nullptr;
                left &= left - 1;
                if (at[j]) w[j] = *reinterpret_cast<const Word*>(at[j]);
            }
#pragma unroll
            for (int j = 0; j < M; ++j) {
                if (!at[j]) continue;
                float x[VE];
                decode<VE>(w[j], x);
                *reinterpret_cast<Word*>(at[j]) = encode<VE>(x, ratio);
            }
        }
}

// Which rows of a block are written: lane i holds the positions that go to the block's rows i and 32 + i, -1 where a row stays.
struct BlockRows {
    int low, high;
    uint64_t written, stays;
    __device__ __forceinline__ BlockRows(int l, int h, int64_t room, int shift) : low(l), high(h) {
        const int rows = (int)(room < (1 << shift) ? room : 1 << shift);
        const uint64_t all = rows >= 64 ? ~0ull : (1ull << rows) - 1;
        written = __ballot_sync(FULL, low >= 0);
        if (shift > 5) written |= (uint64_t)__ballot_sync(FULL, high >= 0) << 32;
        stays = all & ~written;
    }
    __device__ __forceinline__ int position(int row) const { return __shfl_sync(FULL, row < 32 ? low : high, row & 31); }
};

// A block by one warp: any number of rows, heads and columns.
template <typename T, int VE> __device__ __forceinline__ void write_block(const CodedWrite& P, int64_t b, BlockRows B) {
    constexpr int U = 4;                                     // rows whose loads are in flight
    const CodedView& C = P.to;
    const int lane = threadIdx.x & 31, tl = P.tl, t = lane & (tl - 1), D = C.head_dim;
    // the next rows of a set, with their positions (-1: none)
    auto take = [&](uint64_t& left, int (&row)[U], int (&at)[U]) {
#pragma unroll
        for (int j = 0; j < U; ++j) {
            row[j] = left ? __ffsll(left) - 1 : 0;
            const int p = B.position(row[j]);
            at[j] = left ? p : -1;
            left &= left - 1;
        }
    };
    for (int h = lane / tl; h < P.head_tiles * (32 / tl); h += 32 / tl) {
        const bool mine = h < C.heads;
        const T* in = (const T*)P.in.data + (int64_t)(mine ? h : 0) * P.in.head_stride;
        uint8_t* scale = C.scales + b * C.scale_stride + (mine ? h : 0);
        const uint32_t before = B.stays ? *scale : 0u;
        uint32_t top = 0;
        for (uint64_t left = B.written; left;) {
            int row[U], at[U];
            take(left, row, at);
            for (int c = t * VE; c < D; c += tl * VE) {
                Raw<T, VE> r[U];
#pragma unroll
                for (int j = 0; j < U; ++j) r[j] = mine && at[j] >= 0 ? load_raw<T, VE>(in + (int64_t)at[j] * P.in.row_stride + c) : zero_raw<T, VE>();
#pragma unroll
                for (int j = 0; j < U; ++j) top = max(top, magnitude<T, VE>(r[j]));
            }
        }
        for (int o = 1; o < tl; o <<= 1) top = max(top, __shfl_xor_sync(FULL, top, o));
        const uint32_t after = max(scale_byte(top), before);
        const float unscale = unscale_of(after);
        uint8_t* out = C.codes + (b << C.shift) * C.row_stride + (int64_t)(mine ? h : 0) * C.pitch;
        for (uint64_t left = B.written; left;) {
            int row[U], at[U];
            take(left, row, at);
            if (!mine) continue;
#pragma unroll
            for (int j = 0; j < U; ++j) {
                if (at[j] < 0) continue;
                uint8_t* to = out + (int64_t)row[j] * C.row_stride;
                for (int c = t * VE; c < D; c += tl * VE) put_codes<T, VE>(to + c, load_raw<T, VE>(in + (int64_t)at[j] * P.in.row_stride + c), unscale);
                for (int c = D + t; c < C.pitch; c += tl) to[c] = 0;
            }
        }
        __syncwarp();                                        // the scale has been read by all lanes of the head
        if (!mine) continue;
        if (B.stays && after != before) requantise<VE>(out, C.row_stride, B.stays, after - before, t * VE, D, tl * VE);
        if (t == 0 && (!B.stays || after != before)) *scale = (uint8_t)after;
    }
}

// All warps of a kernel have read the list's length: the last block of threads to say so empties the list.
__device__ __forceinline__ void close_list(const Claims& K) {
    __syncthreads();
    if (threadIdx.x == 0 && atomicAdd(K.words + 1, 1) + 2 == (int)gridDim.x) K.words[0] = K.words[1] = -1;
}
// Block i of those that are written (row i, where a block is one), -1 if there is none, and the positions that go to its rows.
__device__ __forceinline__ int listed_block(const CodedWrite& P, const Claims& K, int64_t i, int n, int& low, int& high) {
    const int lane = threadIdx.x & 31, rows = 1 << P.to.shift;
    low = high = -1;
    if (i >= n) return -1;
    if (P.to.shift == 0) {
        const int id = __ldg(P.ids + i);
        if (id < 0 || id >= P.to.rows || __ldcg(K.rows + id) != (int)i) return -1;
        if (lane == 0) low = (int)i;
        return id;
    }
    const int b = __ldcg(K.list + i);
    const int64_t row = ((int64_t)b << P.to.shift) + lane;
    if (lane < rows && row < P.to.rows) low = __ldcg(K.rows + row);
    if (lane + 32 < rows && row + 32 < P.to.rows) high = __ldcg(K.rows + row + 32);
    return b;
}
// The claims of a block are free again.
__device__ __forceinline__ void release(const CodedWrite& P, const Claims& K, int64_t i, int b, int low, int high) {
    const int lane = threadIdx.x & 31;
    const int64_t row = ((int64_t)b << P.to.shift) + lane;
    if (low >= 0) K.rows[row] = -1;
    if (high >= 0) K.rows[row + 32] = -1;
    if (P.to.shift && lane == 0) K.listed[b] = K.list[i] = -1;
}

// Rows by id, Q blocks to a warp at a time, in stores whose heads the lanes hold in one piece each.  Of a block's rows R are held from
// the search for the scale to the codes (where a batch's nodes lie anywhere among all, few of a block are written).
template <typename T, int VE> __global__ void __launch_bounds__(CD_THREADS, 3) k_coded_write_few(const __grid_constant__ CodedWrite P) {
    constexpr int Q = 2, R = 4;
    chain_wait();
    const CodedView& C = P.to;
    const Claims K(P);
    const int n = C.shift ? __ldcg(K.words) + 1 : coded_count(P.n);             // blocks listed, or positions
    const int lane = threadIdx.x & 31, tl = P.tl, t = lane & (tl - 1), h = lane / tl, rows = 1 << C.shift;
    const bool mine = h < C.heads && t * VE < C.pitch, loads = mine && t * VE < C.head_dim;      // codes up to the pitch are zeros
    const char* in = reinterpret_cast<const char*>((const T*)P.in.data + (int64_t)(mine ? h : 0) * P.in.head_stride + (loads ? t * VE : 0));
    uint8_t* codes = C.codes + (int64_t)(mine ? h : 0) * C.pitch + (mine ? t * VE : 0);
    uint8_t* scales = C.scales + (mine ? h : 0);
    const uint32_t in_step = (uint32_t)P.in.row_stride * (uint32_t)sizeof(T), row_step = (uint32_t)C.row_stride, scale_step = (uint32_t)C.scale_stride;
    auto fetch = [&](uint32_t left, int low, Raw<T, VE> (&r)[R]) {
#pragma unroll
        for (int j = 0; j < R; ++j) {
            r[j] = zero_raw<T, VE>();
            if (!left) continue;
            const int p = __shfl_sync(FULL, low, __ffs(left) - 1);
            if (loads) r[j] = load_raw<T, VE>(reinterpret_cast<const T*>(in + (uint64_t)(uint32_t)p * in_step));
            left &= left - 1;
        }
    };
    auto after_r = [](uint32_t left) {                       // the set without its first R rows
#pragma unroll
        for (int j = 0; j < R; ++j) left &= left - 1;
        return left;
    };
    for (int64_t i = ((int64_t)blockIdx.x * (CD_THREADS / 32) + (threadIdx.x >> 5)) * Q; i < n; i += (int64_t)gridDim.x * (CD_THREADS / 32) * Q) {
        int b[Q], low[Q], high[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q) b[q] = listed_block(P, K, i + q, n, low[q], high[q]);
        Raw<T, VE> r[Q][R];
        uint32_t before[Q], written[Q], all[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            written[q] = __ballot_sync(FULL, low[q] >= 0);
            const uint32_t room = b[q] < 0 ? 0u : (uint32_t)C.rows - ((uint32_t)b[q] << C.shift);
            all[q] = room >= 32u ? FULL : (1u << room) - 1;
            if (rows < 32) all[q] &= (1u << rows) - 1;
            before[q] = all[q] != written[q] ? scales[(uint64_t)(uint32_t)b[q] * scale_step] : 0u;
            fetch(written[q], low[q], r[q]);
        }
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            if (b[q] < 0) continue;
            const bool many = after_r(written[q]) != 0;
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < R; ++j) top = max(top, magnitude<T, VE>(r[q][j]));
            for (uint32_t left = after_r(written[q]); left; left = after_r(left)) {
                fetch(left, low[q], r[q]);
#pragma unroll
                for (int j = 0; j < R; ++j) top = max(top, magnitude<T, VE>(r[q][j]));
            }
            for (int o = 1; o < tl; o <<= 1) top = max(top, __shfl_xor_sync(FULL, top, o));
            const uint32_t after = max(scale_byte(top), before[q]);
            const float unscale = unscale_of(after);
            uint8_t* out = codes + (uint64_t)((uint32_t)b[q] << C.shift) * row_step;
            for (uint32_t left = written[q]; left;) {
                if (many) fetch(left, low[q], r[q]);
#pragma unroll
                for (int j = 0; j < R; ++j) {
                    if (!left) break;
                    if (mine) put_codes<T, VE>(out + (uint64_t)(uint32_t)(__ffs(left) - 1) * row_step, r[q][j], unscale);
                    left &= left - 1;
                }
            }
            const uint32_t stays = all[q] & ~written[q];
            if (mine && stays && after != before[q]) requantise<VE>(out - t * VE, C.row_stride, stays, after - before[q], t * VE, C.head_dim, tl * VE);
            if (mine && t == 0 && (!stays || after != before[q])) scales[(uint64_t)(uint32_t)b[q] * scale_step] = (uint8_t)after;
            release(P, K, i + q, b[q], low[q], high[q]);
        }
    }
    if (C.shift) close_list(K);
}

// The same in any store, a block to a warp at a time.
template <typename T, int VE> __global__ void __launch_bounds__(CD_THREADS) k_coded_write_ids(const __grid_constant__ CodedWrite P) {
    chain_wait();
    const Claims K(P);
    const int n = P.to.shift ? __ldcg(K.words) + 1 : coded_count(P.n);
    for (int64_t i = (int64_t)blockIdx.x * (CD_THREADS / 32) + (threadIdx.x >> 5); i < n; i += (int64_t)gridDim.x * (CD_THREADS / 32)) {
        int low, high;
        const int b = listed_block(P, K, i, n, low, high);
        if (b < 0) continue;
        write_block<T, VE>(P, b, BlockRows(low, high, P.to.rows - ((int64_t)b << P.to.shift), P.to.shift));
        release(P, K, i, b, low, high);
    }
    if (P.to.shift) close_list(K);
}

// A range of rows: a warp per block.
template <typename T, int VE> __global__ void __launch_bounds__(CD_THREADS) k_coded_write_range(const __grid_constant__ CodedWrite P) {
    chain_wait();
    const int lane = threadIdx.x & 31, rows = 1 << P.to.shift;
    const int64_t first = P.first, room = P.to.rows - first;
    const int64_t n = coded_count(P.n) < room ? coded_count(P.n) : room;
    if (n <= 0) return;
    const int64_t b1 = (first + n - 1) >> P.to.shift;
    for (int64_t b = (first >> P.to.shift) + (int64_t)blockIdx.x * (CD_THREADS / 32) + (threadIdx.x >> 5); b <= b1; b += (int64_t)gridDim.x * (CD_THREADS / 32)) {
        const int64_t r0 = (b << P.to.shift) + lane - first, r1 = r0 + 32;
        write_block<T, VE>(P, b, BlockRows(lane < rows && r0 >= 0 && r0 < n ? (int)r0 : -1, lane + 32 < rows && r1 >= 0 && r1 < n ? (int)r1 : -1,
                                           P.to.rows - (b << P.to.shift), P.to.shift));
    }
}

// out[p, h, :] = scale * codes of row ids[p] (or first + p).  A group of lanes per row, U rows in flight; a lane keeps its piece
// of a row from row to row where the row has no more pieces than the group has lanes.
template <typename T, int VE, int U> __global__ void __launch_bounds__(CD_THREADS, 4) k_coded_read(const __grid_constant__ CodedRead P) {
    chain_wait();
    const CodedView& C = P.from;
    const int n = coded_count(P.n), lane = threadIdx.x & 31, tl = P.tl, t = lane & (tl - 1), rpw = 32 / tl;
    const int per_head = (C.head_dim + VE - 1) / VE, pieces = per_head * C.heads;
    const int64_t step_o = rpw * P.out.row_stride;
    const uint32_t step_c = (uint32_t)C.row_stride, step_s = (uint32_t)C.scale_stride;
    const int64_t tile = (int64_t)rpw * U, step = (int64_t)gridDim.x * (CD_THREADS / 32) * tile;
    for (int64_t p0 = ((int64_t)blockIdx.x * (CD_THREADS / 32) + (threadIdx.x >> 5)) * tile; p0 < n; p0 += step) {
        const int rows = (int)(n - p0 < tile ? n - p0 : tile) - lane / tl;      // of this group, rpw apart
        int row[U];                                          // -1: zeros
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int64_t p = p0 + j * rpw + lane / tl;
            row[j] = j * rpw >= rows ? -1 : (P.ids ? __ldg(P.ids + p) : (int)(P.first + p));
            if (row[j] >= C.rows) row[j] = -1;
        }
        for (int piece = t; piece < pieces; piece += tl) {
            const int h = piece / per_head, c = (piece - h * per_head) * VE;
            const uint8_t* codes = C.codes + (int64_t)h * C.pitch + c;
            const uint8_t* scales = C.scales + h;
            T* out = (T*)P.out.data + (p0 + lane / tl) * P.out.row_stride + (int64_t)h * P.out.head_stride + c;
            typename CodeWord<VE>::type w[U];
            uint32_t s[U];
#pragma unroll
            for (int j = 0; j < U; ++j) {
                w[j] = {};
                s[j] = 0;
                if (row[j] >= 0) {
                    w[j] = __ldg(reinterpret_cast<const typename CodeWord<VE>::type*>(codes + (uint64_t)(uint32_t)row[j] * step_c));
                    s[j] = __ldg(scales + (uint64_t)((uint32_t)row[j] >> C.shift) * step_s);
                }
            }
#pragma unroll
            for (int j = 0; j < U; ++j) {
                if (j * rpw >= rows) break;
                float x[VE];
                decode<VE>(w[j], x);
                const float scale = scale_of(s[j]);
#pragma unroll
                for (int i = 0; i < VE; ++i) x[i] *= scale;
                store_vec<T, VE>(out, x);
                out += step_o;
            }
        }
    }
}

// ---------------------------------------------------------------- launches
// Elements per access that the head dimension and the typed side allow (the codes are on pieces of 16 bytes).
static int coded_elems(gs_dtype dtype, int head_dim, const HeadView& v) {
    const int size = dtype == GS_BF16 ? 2 : 4;
    for (int ve = 16 / size; ve >= 4; ve /= 2)
        if (head_dim % ve == 0 && (uintptr_t)v.data % (ve * size) == 0 && (v.row_stride * size) % (ve * size) == 0 && (v.head_stride * size) % (ve * size) == 0) return ve;
    return 1;
}

template <typename T, int VE> static cudaError_t run_write(CodedWrite P, cudaStream_t s) {
    const int pieces = (P.to.pitch + VE - 1) / VE;
    P.tl = 1;
    while (P.tl < pieces && P.tl < 32) P.tl *= 2;
    P.head_tiles = (P.to.heads + 32 / P.tl - 1) / (32 / P.tl);
    if (!P.ids) {
        const int64_t blocks = ((int64_t)P.n.bound >> P.to.shift) + 2;
        int64_t grid = (blocks + CD_THREADS / 32 - 1) / (CD_THREADS / 32);
        if (grid > sm_count() * 32) grid = sm_count() * 32;
        return launch_train(k_coded_write_range<T, VE>, grid, CD_THREADS, 0, s, P);
    }
    int64_t grid = ((int64_t)P.n.bound + CD_THREADS - 1) / CD_THREADS;
    if (grid > sm_count() * 16) grid = sm_count() * 16;
    const cudaError_t e = launch_train(k_coded_claim, grid, CD_THREADS, 0, s, P);
    if (e != cudaSuccess) return e;
    // a piece of every head to the lanes, and blocks whose rows one ballot tells
    const bool few = P.head_tiles == 1 && P.to.pitch <= P.tl * VE && P.to.shift <= 5;
    const int64_t blocks = (P.to.rows + (1 << P.to.shift) - 1) >> P.to.shift, most = P.to.shift && blocks < P.n.bound ? blocks : P.n.bound;
    const int per = CD_THREADS / 32 * (few ? 2 : 1);
    grid = (most + per - 1) / per;
    if (grid > sm_count() * 3) grid = sm_count() * 3;        // what is resident: blocks of a few rows and of many come to every warp
    return few ? launch_train(k_coded_write_few<T, VE>, grid, CD_THREADS, 0, s, P) : launch_train(k_coded_write_ids<T, VE>, grid, CD_THREADS, 0, s, P);
}

cudaError_t launch_coded_write(const CodedWrite& P, cudaStream_t s) {
    const int ve = coded_elems(P.dtype, P.to.head_dim, P.in);
    if (P.dtype == GS_BF16) return ve == 8 ? run_write<bf16, 8>(P, s) : (ve == 4 ? run_write<bf16, 4>(P, s) : run_write<bf16, 1>(P, s));
    return ve == 4 ? run_write<float, 4>(P, s) : run_write<float, 1>(P, s);
}

template <typename T, int VE> static cudaError_t run_read(CodedRead P, cudaStream_t s) {
    constexpr int U = 8;
    const int64_t pieces = (int64_t)((P.from.head_dim + VE - 1) / VE) * P.from.heads;
    P.tl = 1;
    while (P.tl < pieces && P.tl < 32) P.tl *= 2;
    const int64_t tile = (int64_t)(32 / P.tl) * U * (CD_THREADS / 32);
    int64_t grid = ((int64_t)P.n.bound + tile - 1) / tile;
    if (grid > sm_count() * 64) grid = sm_count() * 64;
    return launch_train(k_coded_read<T, VE, U>, grid, CD_THREADS, 0, s, P);
}

cudaError_t launch_coded_read(const CodedRead& P, cudaStream_t s) {
    const int ve = coded_elems(P.dtype, P.from.head_dim, P.out);
    if (P.dtype == GS_BF16) return ve == 8 ? run_read<bf16, 8>(P, s) : (ve == 4 ? run_read<bf16, 4>(P, s) : run_read<bf16, 1>(P, s));
    return ve == 4 ? run_read<float, 4>(P, s) : run_read<float, 1>(P, s);
}

}  // namespace gs
