// Rows kept in 8 bits: written by node id or as a range, with one scale per block of rows and head, and read back.
//
//   code = e4m3(x / s),  s = 2^e the smallest with |x| <= 448 s over the block's rows of a head;  read: s code.
//
// A write changes some rows of a block.  If it leaves others, the block's scale never falls: it is raised where the new rows need
// it, and the codes that stay are brought to it.  One warp does all of a block, so nobody else sees it half written.  Which warp,
// and which row wins where an id occurs twice, is settled by a pass of integer maxima before (claims): the highest position.
// Both kernels move bytes and little else; the source rows are read twice by the write (for the scale, for the codes), the second
// time from the cache.
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

// claims[row] and, for blocks of several rows, claims[rows + block]: the highest position that writes there (-1: none).
__global__ void __launch_bounds__(CD_THREADS) k_coded_claim(const __grid_constant__ CodedWrite P) {
    chain_wait();
    const int n = coded_count(P.n);
    for (int64_t p = (int64_t)blockIdx.x * CD_THREADS + threadIdx.x; p < n; p += (int64_t)gridDim.x * CD_THREADS) {
        const int64_t id = __ldg(P.ids + p);
        if (id < 0 || id >= P.to.rows) continue;
        atomicMax(P.claims + id, (int)p);
        if (P.to.shift) atomicMax(P.claims + P.to.rows + (id >> P.to.shift), (int)p);
    }
}

// The block b by one warp.  Lane i holds the positions that are written to the block's rows i and 32 + i, -1 where a row stays.
template <typename T, int VE> __device__ __forceinline__ void write_block(const CodedWrite& P, int64_t b, int low, int high) {
    constexpr int U = 4;                                     // rows whose loads are in flight
    using Word = typename CodeWord<VE>::type;
    const CodedView& C = P.to;
    const int lane = threadIdx.x & 31, tl = P.tl, t = lane & (tl - 1), D = C.head_dim;
    const int64_t first = b << C.shift, room = C.rows - first;
    const int rows = (int)(room < (1 << C.shift) ? room : 1 << C.shift);
    const uint64_t all = rows == 64 ? ~0ull : (1ull << rows) - 1;
    const uint64_t written = (((uint64_t)__ballot_sync(FULL, high >= 0) << 32) | __ballot_sync(FULL, low >= 0)) & all, stays = all & ~written;
    // the next rows of a set, with their positions (-1: none)
    auto take = [&](uint64_t& left, int (&row)[U], int (&at)[U]) {
#pragma unroll
        for (int j = 0; j < U; ++j) {
            row[j] = left ? __ffsll(left) - 1 : 0;
            const int p = __shfl_sync(FULL, row[j] < 32 ? low : high, row[j] & 31);
            at[j] = left ? p : -1;
            left &= left - 1;
        }
    };
    for (int h = lane / tl; h < P.head_tiles * (32 / tl); h += 32 / tl) {
        const bool mine = h < C.heads;
        const T* in = (const T*)P.in.data + (int64_t)(mine ? h : 0) * P.in.head_stride;
        uint32_t top = 0, before = 0;
        if (mine && stays && t == 0) before = C.scales[b * C.scale_stride + h];
        for (uint64_t left = written; left;) {
            int row[U], at[U];
            take(left, row, at);
            for (int c = t * VE; c < D; c += tl * VE) {
                Raw<T, VE> r[U];
#pragma unroll
                for (int j = 0; j < U; ++j) r[j] = mine && at[j] >= 0 ? load_raw<T, VE>(in + (int64_t)at[j] * P.in.row_stride + c) : zero_raw<T, VE>();
#pragma unroll
                for (int j = 0; j < U; ++j) {
                    float x[VE];
                    unpack<T, VE>(r[j], x);
#pragma unroll
                    for (int i = 0; i < VE; ++i) {
                        const uint32_t m = finite_magnitude(x[i]);
                        top = m > top ? m : top;
                    }
                }
            }
        }
        for (int o = 1; o < tl; o <<= 1) {
            const uint32_t m = __shfl_xor_sync(FULL, top, o);
            top = m > top ? m : top;
        }
        before = __shfl_sync(FULL, before, lane & ~(tl - 1));
        const uint32_t need = scale_byte(top), after = need > before ? need : before;
        const float unscale = unscale_of(after);
        uint8_t* out = C.codes + first * C.row_stride + (int64_t)h * C.pitch;
        for (uint64_t left = written; left;) {
            int row[U], at[U];
            take(left, row, at);
            if (!mine) continue;
#pragma unroll
            for (int j = 0; j < U; ++j) {
                if (at[j] < 0) continue;
                uint8_t* to = out + (int64_t)row[j] * C.row_stride;
                for (int c = t * VE; c < D; c += tl * VE) {
                    float x[VE];
                    unpack<T, VE>(load_raw<T, VE>(in + (int64_t)at[j] * P.in.row_stride + c), x);
                    *reinterpret_cast<Word*>(to + c) = encode<VE>(x, unscale);
                }
                for (int c = D + t; c < C.pitch; c += tl) to[c] = 0;
            }
        }
        if (!mine) continue;
        if (stays && after != before) {                      // the codes that stay, brought to the new scale
            const float ratio = after - before < 64u ? scale_of(127u + before - after) : 0.f;
            for (int i = 0; i < rows; ++i) {
                if (!(stays >> i & 1)) continue;
                for (int c = t * VE; c < D; c += tl * VE) {
                    Word* w = reinterpret_cast<Word*>(out + (int64_t)i * C.row_stride + c);
                    float x[VE];
                    decode<VE>(*w, x);
                    *w = encode<VE>(x, ratio);
                }
            }
        }
        if (t == 0 && (!stays || after != before)) C.scales[b * C.scale_stride + h] = (uint8_t)after;
    }
}

// Rows by id: the warp takes 32 positions at a time and writes the blocks that they lead, one after the other.
template <typename T, int VE> __global__ void __launch_bounds__(CD_THREADS) k_coded_write_ids(const __grid_constant__ CodedWrite P) {
    chain_wait();
    const int n = coded_count(P.n), lane = threadIdx.x & 31;
    const int64_t step = (int64_t)gridDim.x * (CD_THREADS / 32) * P.take;
    for (int64_t p0 = ((int64_t)blockIdx.x * (CD_THREADS / 32) + (threadIdx.x >> 5)) * P.take; p0 < n; p0 += step) {
        const int64_t p = p0 + lane;
        int64_t block = -1;
        if (lane < P.take && p < n) {
            const int64_t id = __ldg(P.ids + p);
            if (id >= 0 && id < P.to.rows) {
                const int64_t b = id >> P.to.shift;
                if (__ldcg(P.claims + (P.to.shift ? P.to.rows + b : id)) == (int)p) block = b;
            }
        }
        for (uint32_t left = __ballot_sync(FULL, block >= 0); left; left &= left - 1) {
            const int64_t b = __shfl_sync(FULL, block, __ffs(left) - 1);
            const int64_t first = b << P.to.shift, room = P.to.rows - first;
            const int rows = (int)(room < (1 << P.to.shift) ? room : 1 << P.to.shift);
            int low = -1, high = -1;
            if (lane < rows) low = P.to.shift ? __ldcg(P.claims + first + lane) : (int)(p0 + __ffs(left) - 1);
            if (lane + 32 < rows) high = __ldcg(P.claims + first + lane + 32);
            write_block<T, VE>(P, b, low, high);
            if (low >= 0) P.claims[first + lane] = -1;
            if (high >= 0) P.claims[first + lane + 32] = -1;
            if (P.to.shift && lane == 0) P.claims[P.to.rows + b] = -1;
            __syncwarp();
        }
    }
}

// A range of rows: a warp per block.
template <typename T, int VE> __global__ void __launch_bounds__(CD_THREADS) k_coded_write_range(const __grid_constant__ CodedWrite P) {
    chain_wait();
    const int lane = threadIdx.x & 31;
    const int64_t first = P.first, room = P.to.rows - first;
    const int64_t n = coded_count(P.n) < room ? coded_count(P.n) : room;
    if (n <= 0) return;
    const int64_t b1 = (first + n - 1) >> P.to.shift;
    for (int64_t b = (first >> P.to.shift) + (int64_t)blockIdx.x * (CD_THREADS / 32) + (threadIdx.x >> 5); b <= b1; b += (int64_t)gridDim.x * (CD_THREADS / 32)) {
        const int64_t r0 = (b << P.to.shift) + lane - first, r1 = r0 + 32;
        const int rows = 1 << P.to.shift;
        write_block<T, VE>(P, b, lane < rows && r0 >= 0 && r0 < n ? (int)r0 : -1, lane + 32 < rows && r1 >= 0 && r1 < n ? (int)r1 : -1);
    }
}

// out[p, h, :] = scale * codes of row ids[p] (or first + p).  A group of lanes per row, U rows in flight; a lane keeps its piece
// of a row from row to row where the row has no more pieces than the group has lanes.
template <typename T, int VE, int U> __global__ void __launch_bounds__(CD_THREADS) k_coded_read(const __grid_constant__ CodedRead P) {
    chain_wait();
    const CodedView& C = P.from;
    const int n = coded_count(P.n), lane = threadIdx.x & 31, tl = P.tl, t = lane & (tl - 1), rpw = 32 / tl;
    const int per_head = (C.head_dim + VE - 1) / VE, pieces = per_head * C.heads;
    const int64_t tile = (int64_t)rpw * U, step = (int64_t)gridDim.x * (CD_THREADS / 32) * tile;
    for (int64_t p0 = ((int64_t)blockIdx.x * (CD_THREADS / 32) + (threadIdx.x >> 5)) * tile; p0 < n; p0 += step) {
        int64_t row[U];
        bool on[U];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int64_t p = p0 + j * rpw + lane / tl;
            on[j] = p < n;
            row[j] = !on[j] ? -1 : (P.ids ? (int64_t)__ldg(P.ids + p) : P.first + p);
            if (row[j] >= C.rows) row[j] = -1;
        }
        for (int piece = t; piece < pieces; piece += tl) {
            const int h = piece / per_head, c = (piece - h * per_head) * VE;
            typename CodeWord<VE>::type w[U];
            uint32_t s[U];
#pragma unroll
            for (int j = 0; j < U; ++j) {
                w[j] = {};
                s[j] = 0;
                if (row[j] >= 0) {
                    w[j] = __ldg(reinterpret_cast<const typename CodeWord<VE>::type*>(C.codes + row[j] * C.row_stride + (int64_t)h * C.pitch + c));
                    s[j] = __ldg(C.scales + (row[j] >> C.shift) * C.scale_stride + h);
                }
            }
#pragma unroll
            for (int j = 0; j < U; ++j) {
                if (!on[j]) continue;
                float x[VE];
                decode<VE>(w[j], x);
                const float scale = scale_of(s[j]);
#pragma unroll
                for (int i = 0; i < VE; ++i) x[i] *= scale;
                store_vec<T, VE>((T*)P.out.data + (p0 + j * rpw + lane / tl) * P.out.row_stride + (int64_t)h * P.out.head_stride + c, x);
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
    const int pieces = (P.to.head_dim + VE - 1) / VE;
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
    // few positions: fewer of them to a warp, so that all SMs have some
    P.take = 32;
    while (P.take > 1 && (int64_t)P.n.bound < sm_count() * 8 * (int64_t)P.take) P.take /= 2;
    grid = ((int64_t)P.n.bound + (CD_THREADS / 32) * P.take - 1) / ((CD_THREADS / 32) * P.take);
    if (grid > sm_count() * 32) grid = sm_count() * 32;
    return launch_train(k_coded_write_ids<T, VE>, grid, CD_THREADS, 0, s, P);
}

cudaError_t launch_coded_write(const CodedWrite& P, cudaStream_t s) {
    const int ve = coded_elems(P.dtype, P.to.head_dim, P.in);
    if (P.dtype == GS_BF16) return ve == 8 ? run_write<bf16, 8>(P, s) : (ve == 4 ? run_write<bf16, 4>(P, s) : run_write<bf16, 1>(P, s));
    return ve == 4 ? run_write<float, 4>(P, s) : run_write<float, 1>(P, s);
}

template <typename T, int VE> static cudaError_t run_read(CodedRead P, cudaStream_t s) {
    constexpr int U = 4;
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
