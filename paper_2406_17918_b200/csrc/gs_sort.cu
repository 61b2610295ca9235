// Stable sort of (key, payload) pairs by key: the order in which gradients of repeated ids, and the edges of a
// block seen from their sources, are summed.  Least-significant-digit radix sort with 8-bit digits over the bits the
// keys have.  One kernel counts the digits of every pass; each pass is then one kernel in which a tile of 4096 pairs
// finds its place behind the earlier tiles by looking back over their published digit counts (tiles are handed out
// by a counter, so the tiles a block waits for are held by blocks that already run; every wait is bounded all the
// same).  The pairs are put in digit order in shared memory first, so that they leave in runs.  Equal keys keep
// their input order: results do not depend on the schedule.
#include "gs_device.cuh"
#include "gs_train.h"

namespace gs {

constexpr int KS_THREADS = 256;
constexpr int KS_ROUNDS = 16;
constexpr int KS_TILE = KS_THREADS * KS_ROUNDS;
constexpr int KS_WARPS = KS_THREADS / 32;
constexpr int KS_SMALL = 4096;               // up to here one block sorts everything in shared memory
constexpr int KS_SMALL_THREADS = 1024;
constexpr unsigned KS_WAIT_LIMIT = 1u << 22; // polls of one predecessor's word before the block gives up

__device__ int g_sort_gave_up;

struct KeySort {
    const int32_t* keys;
    const int32_t* payload;
    Count n;
    uint32_t key_limit;
    int passes, shift;
    int32_t* hist;           // [4][256]
    int32_t* ticket;         // [4]
    uint32_t* state;         // this pass: [tiles][256]: 2 flag bits, 30 bits of count
    const unsigned long long* src;
    unsigned long long* dst;      // passes before the last: key << 32 | payload
    uint32_t* out_keys;           // last pass
    int32_t* out_payload;
};

__device__ __forceinline__ int count_of(const Count& c) {
    if (!c.d_n) return c.bound;
    const int n = __ldcg(c.d_n);
    return n < 0 ? 0 : (n > c.bound ? c.bound : n);
}

__device__ __forceinline__ uint32_t clamp_key(int32_t k, uint32_t limit) {
    return (uint32_t)k < limit ? (uint32_t)k : limit;
}

__device__ __forceinline__ unsigned long long first_word(const KeySort& P, int i) {
    return ((unsigned long long)clamp_key(__ldg(P.keys + i), P.key_limit) << 32) | (uint32_t)(P.payload ? __ldcg(P.payload + i) : i);
}

__global__ void __launch_bounds__(KS_THREADS) k_key_hist(KeySort P) {
    constexpr int U = 4;
    __shared__ int h[4][256];
    chain_wait();
    const int n = count_of(P.n);
    for (int i = threadIdx.x; i < 1024; i += KS_THREADS) (&h[0][0])[i] = 0;
    __syncthreads();
    for (int64_t i = (int64_t)blockIdx.x * KS_THREADS * U + threadIdx.x; i < n; i += (int64_t)gridDim.x * KS_THREADS * U) {
        uint32_t k[U];
#pragma unroll
        for (int j = 0; j < U; ++j) k[j] = i + j * KS_THREADS < n ? clamp_key(__ldg(P.keys + i + j * KS_THREADS), P.key_limit) : 0xFFFFFFFFu;
#pragma unroll
        for (int j = 0; j < U; ++j)
            if (i + j * KS_THREADS < n)
                for (int p = 0; p < P.passes; ++p) atomicAdd(&h[p][(k[j] >> (8 * p)) & 255u], 1);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 256 * P.passes; i += KS_THREADS) {
        const int c = (&h[0][0])[i];
        if (c) atomicAdd(P.hist + i, c);
    }
}

// Lanes whose digit equals this lane's, from one ballot per bit (a match instruction takes time for every distinct
// digit in the warp: 2 M keys, 50 us a pass).
__device__ __forceinline__ uint32_t same_digit(uint32_t d) {
    uint32_t same = FULL;
#pragma unroll
    for (int b = 0; b < 8; ++b) {
        const uint32_t set = __ballot_sync(FULL, (d >> b) & 1u);
        same &= (d >> b) & 1u ? set : ~set;
    }
    return same;
}

// Ranks a warp's keys round by round: rank[r] = keys of the same digit before this one in the warp's share,
// cnt[d] = the warp's count of digit d at the end.
template <int ROUNDS>
__device__ __forceinline__ void rank_rounds(const unsigned long long (&key)[ROUNDS], int shift, int* cnt, int (&rank)[ROUNDS]) {
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const uint32_t d = (uint32_t)(key[r] >> shift) & 255u;
        const uint32_t same = same_digit(d), before = __popc(same & lanemask_lt());
        const int base = cnt[d];
        rank[r] = base + before;
        __syncwarp();
        if (before == 0) cnt[d] = base + __popc(same);
        __syncwarp();
    }
}

__global__ void __launch_bounds__(KS_THREADS, 3) k_key_pass(KeySort P, int first, int last) {
    __shared__ unsigned long long pairs[KS_TILE];
    __shared__ int cnt[KS_WARPS][256];
    __shared__ int local_start[256];     // first place of a digit inside the tile
    __shared__ int out_base[256];        // output position of the tile's pair j of digit d is out_base[d] + j
    __shared__ int warp_sums[33];
    __shared__ int s_tile;
    chain_wait();
    const int n = count_of(P.n);
    const int tiles = (int)(((int64_t)n + KS_TILE - 1) / KS_TILE);
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, d = threadIdx.x;
    int total;
    const int digit_base = block_exclusive_scan<KS_THREADS>(__ldcg(P.hist + d), warp_sums, &total);
    for (;;) {
        __syncthreads();
        if (threadIdx.x == 0) s_tile = atomicAdd(P.ticket, 1);
        for (int t = threadIdx.x; t < KS_WARPS * 256; t += KS_THREADS) (&cnt[0][0])[t] = 0;
        __syncthreads();
        const int tile = s_tile;
        if (tile >= tiles) return;
        unsigned long long key[KS_ROUNDS];
        int rank[KS_ROUNDS];
        const int64_t wbase = (int64_t)tile * KS_TILE + wid * (KS_ROUNDS * 32);
#pragma unroll
        for (int r = 0; r < KS_ROUNDS; ++r) {
            const int64_t i = wbase + r * 32 + lane;
            key[r] = i < n ? (first ? first_word(P, (int)i) : __ldcg(P.src + i)) : ~0ull;   // padding sorts last, behind position n
        }
        rank_rounds(key, P.shift, cnt[wid], rank);
        __syncthreads();
        int sum = 0;
#pragma unroll
        for (int w = 0; w < KS_WARPS; ++w) {
            const int c = cnt[w][d];
            cnt[w][d] = sum;
            sum += c;
        }
        volatile uint32_t* st = P.state + (size_t)tile * 256 + d;
        *st = (tile == 0 ? 2u << 30 : 1u << 30) | (uint32_t)sum;
        const int lstart = block_exclusive_scan<KS_THREADS>(sum, warp_sums, &total);
        local_start[d] = lstart;
        int before = 0;
        unsigned polls = 0;
        for (int t = tile - 1; t >= 0;) {
            const uint32_t w = *((volatile uint32_t*)P.state + (size_t)t * 256 + d);
            if (w == 0) {
                if (++polls > KS_WAIT_LIMIT) {
                    atomicExch(&g_sort_gave_up, 1);
                    break;
                }
                continue;
            }
            before += (int)(w & 0x3FFFFFFFu);
            if (w >> 31) break;
            --t;
            polls = 0;
        }
        if (tile) *st = (2u << 30) | (uint32_t)(before + sum);
        out_base[d] = digit_base + before - lstart;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < KS_ROUNDS; ++r) {
            const uint32_t dg = (uint32_t)(key[r] >> P.shift) & 255u;
            pairs[local_start[dg] + cnt[wid][dg] + rank[r]] = key[r];
        }
        __syncthreads();
        for (int j = threadIdx.x; j < KS_TILE; j += KS_THREADS) {
            const unsigned long long w = pairs[j];
            const int64_t at = (int64_t)out_base[(uint32_t)(w >> P.shift) & 255u] + j;
            if (at < 0 || at >= n) continue;
            if (last) {
                P.out_keys[at] = (uint32_t)(w >> 32);
                P.out_payload[at] = (int32_t)(uint32_t)w;
            } else {
                P.dst[at] = w;
            }
        }
    }
}

// All passes in one block.
__global__ void __launch_bounds__(KS_SMALL_THREADS) k_key_sort_small(KeySort P) {
    constexpr int R = KS_SMALL / KS_SMALL_THREADS, W = KS_SMALL_THREADS / 32;
    extern __shared__ unsigned long long small_pairs[];              // [KS_SMALL], then cnt[W][256]
    int* cnt = reinterpret_cast<int*>(small_pairs + KS_SMALL);
    __shared__ int start[256];
    __shared__ int warp_sums[33];
    chain_wait();
    const int n = count_of(P.n);
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    unsigned long long key[R];
    int rank[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int i = wid * (R * 32) + r * 32 + lane;
        key[r] = i < n ? first_word(P, i) : ~0ull;
    }
    for (int p = 0; p < P.passes; ++p) {
        const int shift = 32 + 8 * p;
        for (int t = threadIdx.x; t < W * 256; t += KS_SMALL_THREADS) cnt[t] = 0;
        __syncthreads();
        rank_rounds(key, shift, cnt + wid * 256, rank);
        __syncthreads();
        int sum = 0;
        if (threadIdx.x < 256) {
            for (int w = 0; w < W; ++w) {
                const int c = cnt[w * 256 + threadIdx.x];
                cnt[w * 256 + threadIdx.x] = sum;
                sum += c;
            }
        }
        int total;
        const int s = block_exclusive_scan<KS_SMALL_THREADS>(sum, warp_sums, &total);
        if (threadIdx.x < 256) start[threadIdx.x] = s;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint32_t dg = (uint32_t)(key[r] >> shift) & 255u;
            small_pairs[start[dg] + cnt[wid * 256 + dg] + rank[r]] = key[r];
        }
        __syncthreads();
        if (p + 1 < P.passes) {
#pragma unroll
            for (int r = 0; r < R; ++r) key[r] = small_pairs[wid * (R * 32) + r * 32 + lane];
        }
        __syncthreads();
    }
    for (int j = threadIdx.x; j < n; j += KS_SMALL_THREADS) {
        P.out_keys[j] = (uint32_t)(small_pairs[j] >> 32);
        P.out_payload[j] = (int32_t)(uint32_t)small_pairs[j];
    }
}

static int64_t ks_tiles(int64_t n) { return (n + KS_TILE - 1) / KS_TILE; }

size_t key_sort_bytes(int64_t n) {
    return align_up((size_t)n * 8, 256) * 2 + align_up((1024 + 4) * 4 + (size_t)ks_tiles(n) * 4 * 1024, 256) + 256;
}

cudaError_t launch_key_sort(const int32_t* keys, const int32_t* payload, Count n, int64_t key_limit, void* workspace,
                            uint32_t* out_keys, int32_t* out_payload, cudaStream_t s) {
    KeySort P{};
    P.keys = keys;
    P.payload = payload;
    P.n = n;
    P.key_limit = (uint32_t)key_limit;
    P.out_keys = out_keys;
    P.out_payload = out_payload;
    int bits = 1;
    while (bits < 32 && (key_limit >> bits)) ++bits;
    P.passes = (bits + 7) / 8;
    if (n.bound <= KS_SMALL) {
        constexpr int smem = KS_SMALL * 8 + (KS_SMALL_THREADS / 32) * 256 * 4;
        const cudaError_t e = cudaFuncSetAttribute(k_key_sort_small, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
        return launch_train(k_key_sort_small, 1, KS_SMALL_THREADS, smem, s, P);
    }
    const size_t buf = align_up((size_t)n.bound * 8, 256);
    unsigned long long* a = (unsigned long long*)workspace;
    unsigned long long* b = (unsigned long long*)((char*)workspace + buf);
    const int64_t tiles = ks_tiles(n.bound);
    int32_t* words = (int32_t*)((char*)workspace + 2 * buf);
    int32_t* hist = words;
    int32_t* ticket = words + 1024;
    uint32_t* state = (uint32_t*)(words + 1028);
    cudaError_t e = cudaMemsetAsync(words, 0, (1028 + (size_t)tiles * 256 * P.passes) * 4, s);
    if (e != cudaSuccess) return e;
    P.hist = hist;
    int64_t grid = (n.bound + KS_THREADS * 4 - 1) / (KS_THREADS * 4);
    if (grid > sm_count() * 8) grid = sm_count() * 8;
    e = launch_train(k_key_hist, grid, KS_THREADS, 0, s, P);
    grid = tiles < sm_count() * 3 ? tiles : sm_count() * 3;
    for (int p = 0; p < P.passes && e == cudaSuccess; ++p) {
        P.shift = 32 + 8 * p;
        P.hist = hist + 256 * p;
        P.ticket = ticket + p;
        P.state = state + (size_t)tiles * 256 * p;
        P.src = (p & 1) ? a : b;
        P.dst = (p & 1) ? b : a;
        e = launch_train(k_key_pass, grid, KS_THREADS, 0, s, P, (int)(p == 0), (int)(p + 1 == P.passes));
    }
    return e;
}

// ---------------------------------------------------------------- row offsets of the sorted list
__device__ __forceinline__ int lower_bound_key(const uint32_t* keys, int lo, int hi, uint32_t key) {
    while (lo < hi) {
        const int mid = (int)(((unsigned)lo + (unsigned)hi) >> 1);
        if (__ldca(keys + mid) < key) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

// The same by a whole warp: 32 probes per step.
__device__ __forceinline__ int lower_bound_warp(const uint32_t* keys, int n, uint32_t key) {
    int lo = 0, hi = n;                                    // the answer lies in [lo, hi]
    const int lane = threadIdx.x & 31;
    while (lo < hi) {
        const int step = (hi - lo + 31) / 32, at = lo + lane * step;
        const uint32_t less = __ballot_sync(FULL, at < hi && __ldcg(keys + at) < key);   // a prefix of the lanes
        const int k = __popc(less);
        if (k == 0) return lo;
        hi = k < 32 && lo + k * step < hi ? lo + k * step : hi;
        lo = lo + (k - 1) * step + 1;
    }
    return lo;
}

constexpr int RS_THREADS = 256, RS_ROWS = 1024;

// A block finds the range of its rows first, so that the rows' own searches stay in a narrow window.
__global__ void __launch_bounds__(RS_THREADS) k_row_starts(const uint32_t* __restrict__ keys, Count nc, Count rc, int32_t* __restrict__ starts) {
    __shared__ int range[2];
    chain_wait();
    const int n = count_of(nc);
    const int64_t rows = (int64_t)count_of(rc) + 1;      // one more than the rows: the end of the last
    for (int64_t r0 = (int64_t)blockIdx.x * RS_ROWS; r0 < rows; r0 += (int64_t)gridDim.x * RS_ROWS) {
        __syncthreads();
        if (threadIdx.x < 64) {
            const int64_t r = r0 + (threadIdx.x >= 32 ? RS_ROWS : 0);
            const int at = lower_bound_warp(keys, n, (uint32_t)r);
            if ((threadIdx.x & 31) == 0) range[threadIdx.x >> 5] = at;
        }
        __syncthreads();
        const int lo = range[0], hi = range[1];
#pragma unroll
        for (int j = 0; j < RS_ROWS / RS_THREADS; ++j) {
            const int64_t r = r0 + j * RS_THREADS + threadIdx.x;
            if (r < rows) starts[r] = lower_bound_key(keys, lo, hi, (uint32_t)r);
        }
    }
}

cudaError_t launch_row_starts(const uint32_t* keys, Count n, Count rows, int32_t* starts, cudaStream_t s) {
    int64_t blocks = ((int64_t)rows.bound + 1 + RS_ROWS - 1) / RS_ROWS;
    if (blocks > sm_count() * 32) blocks = sm_count() * 32;
    return launch_train(k_row_starts, blocks, RS_THREADS, 0, s, keys, n, rows, starts);
}

cudaError_t train_gave_up(cudaStream_t s, int* h_sort) {
    cudaError_t e = cudaMemcpyFromSymbolAsync(h_sort, g_sort_gave_up, sizeof(int), 0, cudaMemcpyDeviceToHost, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    return e;
}

}  // namespace gs
