// Stable sort of (key, payload) pairs by key: the order in which gradients of repeated ids, and the edges of a
// block seen from their sources, are summed.  Least-significant-digit radix sort, digits of up to 9 bits.  A pass is three
// kernels: the digit counts of every tile; every digit's offsets into the
// tiles; and the scatter, in which each warp ranks its pairs by ballots, the tile is put in digit order in shared memory and
// leaves in runs.  Equal keys keep their input order, and no kernel waits for another block: results do not depend on the
// schedule.  2.03 M pairs of 26 bits: 95 us.  (One kernel per 8-bit digit, tiles looking back over their predecessors'
// counts: 150 us, the polls of the waiting tiles held up the others; digits of 11 bits and tiles of 8192: 138 us, one
// block per SM, with as many passes at 26 bits; not tried at 19 to 22 bits, where they would save one.)
#include <cooperative_groups.h>

#include "gs_device.cuh"
#include "gs_train.h"

namespace gs {

constexpr int KS_THREADS = 256;
constexpr int KS_WARPS = KS_THREADS / 32;
constexpr int KS_MAX_BITS = 9, KS_MAX_BINS = 1 << KS_MAX_BITS, KS_MAX_PASSES = (32 + KS_MAX_BITS - 1) / KS_MAX_BITS;
constexpr int KS_ROUNDS_SMALL = 4, KS_ROUNDS_LARGE = 16;   // pairs per thread of a tile
constexpr int64_t KS_LARGE = (int64_t)1 << 19;             // from here on there are tiles enough for the large ones
constexpr int KS_SMALL = 4096;               // up to here one block sorts everything in shared memory
constexpr int KS_SMALL_THREADS = 1024;
constexpr int KC_BLOCKS = 8;                 // up to KC_MAX pairs a cluster of blocks sorts in its shared memory
constexpr int KC_ROUNDS = 8, KC_TILE = 1024 * KC_ROUNDS, KC_MAX = KC_BLOCKS * KC_TILE;
constexpr int KC_BITS = 9, KC_BINS = 1 << KC_BITS;

struct KeySort {
    const int32_t* keys;
    const int32_t* payload;
    Count n;
    Rows within;                  // positions outside these rows take the value key_limit too
    uint32_t key_limit;
    int passes, bits, shift;      // digits; shift: of this pass's digit inside the key
    int tiles;                    // of the bound
    int32_t* totals;              // [bins] pairs per digit
    int32_t* counts;              // [bins][tiles], then the digits' offsets
    const unsigned long long* src;
    unsigned long long* dst;      // passes before the last: key << 32 | payload
    uint32_t* out_keys;           // last pass
    int32_t* out_payload;
    int32_t* zero;                // words that the first kernel clears for the caller
    int zero_words;
};

__device__ __forceinline__ int count_of(const Count& c) {
    if (!c.d_n) return c.bound;
    const int n = __ldcg(c.d_n);
    return n < 0 ? 0 : (n > c.bound ? c.bound : n);
}

__device__ __forceinline__ uint32_t clamp_key(int32_t k, uint32_t limit) {
    return (uint32_t)k < limit ? (uint32_t)k : limit;
}

// The positions [x, y) that the rows hold.
__device__ __forceinline__ int2 span_of(const Rows& r) {
    if (!r.offsets) return make_int2(0, 0x7FFFFFFF);
    return make_int2(__ldcg(r.offsets), __ldcg(r.offsets + count_of(r.n)));
}

__device__ __forceinline__ uint32_t first_key(const KeySort& P, int2 span, int i) {
    return i >= span.x && i < span.y ? clamp_key(__ldg(P.keys + i), P.key_limit) : P.key_limit;
}

__device__ __forceinline__ unsigned long long first_word(const KeySort& P, int2 span, int i) {
    return ((unsigned long long)first_key(P, span, i) << 32) | (uint32_t)(P.payload ? __ldcg(P.payload + i) : i);
}

// Lanes whose digit equals this lane's, from one ballot per bit (a match instruction takes time for every distinct
// digit in the warp).
__device__ __forceinline__ uint32_t same_digit(uint32_t d, int bits) {
    uint32_t same = FULL;
#pragma unroll
    for (int b = 0; b < KS_MAX_BITS; ++b) {
        if (b >= bits) break;
        const uint32_t set = __ballot_sync(FULL, (d >> b) & 1u);
        same &= (d >> b) & 1u ? set : ~set;
    }
    return same;
}

// Ranks a warp's keys round by round: rank[r] = keys of the same digit before this one in the warp's share,
// cnt[d] = the warp's count of digit d at the end.
template <int ROUNDS, typename C>
__device__ __forceinline__ void rank_rounds(const unsigned long long (&key)[ROUNDS], int shift, int bits, C* cnt, int (&rank)[ROUNDS]) {
    const uint32_t mask = (1u << bits) - 1u;
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const uint32_t d = (uint32_t)(key[r] >> shift) & mask;
        const uint32_t same = same_digit(d, bits), before = __popc(same & lanemask_lt());
        const int base = cnt[d];
        rank[r] = base + before;
        __syncwarp();
        if (before == 0) cnt[d] = (C)(base + __popc(same));
        __syncwarp();
    }
}

template <int ROUNDS>
__global__ void __launch_bounds__(KS_THREADS) k_key_count(KeySort P, int first) {
    __shared__ int h[KS_MAX_BINS];
    chain_wait();
    const int n = count_of(P.n), bins = 1 << P.bits;
    const int2 span = span_of(P.within);
    if (first && blockIdx.x == 0)
        for (int i = threadIdx.x; i < P.zero_words; i += KS_THREADS) P.zero[i] = 0;
    for (int tile = blockIdx.x; tile < P.tiles; tile += gridDim.x) {
        __syncthreads();
        for (int i = threadIdx.x; i < bins; i += KS_THREADS) h[i] = 0;
        __syncthreads();
        uint32_t key[ROUNDS];
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const int64_t i = (int64_t)tile * (KS_THREADS * ROUNDS) + r * KS_THREADS + threadIdx.x;
            key[r] = i < n ? (first ? first_key(P, span, (int)i) : (uint32_t)(__ldcg(P.src + i) >> 32)) : 0;
        }
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const int64_t i = (int64_t)tile * (KS_THREADS * ROUNDS) + r * KS_THREADS + threadIdx.x;
            if (i < n) atomicAdd(&h[(key[r] >> P.shift) & (bins - 1)], 1);
        }
        __syncthreads();
        for (int i = threadIdx.x; i < bins; i += KS_THREADS) {
            P.counts[(size_t)i * P.tiles + tile] = h[i];
            if (h[i]) atomicAdd(P.totals + i, h[i]);
        }
    }
}

// A warp per digit: the digit's first place, then its offset in every tile.
__global__ void __launch_bounds__(256) k_key_scan(KeySort P) {
    __shared__ int warp_sums[33];
    __shared__ int starts[8];
    chain_wait();
    const int bins = 1 << P.bits, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int d0 = blockIdx.x * 8; d0 < bins; d0 += gridDim.x * 8) {
        int below = 0, sum;
        for (int i = threadIdx.x; i < d0; i += 256) below += __ldcg(P.totals + i);
        __syncthreads();
        block_exclusive_scan<256>(below, warp_sums, &sum);
        if (threadIdx.x == 0) {
            for (int j = 0; j < 8; ++j) {
                starts[j] = sum;
                if (d0 + j < bins) sum += __ldcg(P.totals + d0 + j);
            }
        }
        __syncthreads();
        const int d = d0 + warp;
        if (d < bins) {
            int at = starts[warp];
            int32_t* row = P.counts + (size_t)d * P.tiles;
            constexpr int PER = 8;                            // words per lane in flight
            for (int base = 0; base < P.tiles; base += 32 * PER) {
                int c[PER];
#pragma unroll
                for (int j = 0; j < PER; ++j) {
                    const int i = base + j * 32 + lane;
                    c[j] = i < P.tiles ? __ldcg(row + i) : 0;
                }
#pragma unroll
                for (int j = 0; j < PER; ++j) {
                    int incl = c[j];
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) {
                        const int y = __shfl_up_sync(FULL, incl, o);
                        if (lane >= o) incl += y;
                    }
                    const int i = base + j * 32 + lane;
                    if (i < P.tiles) row[i] = at + incl - c[j];
                    at += __shfl_sync(FULL, incl, 31);
                }
            }
        }
    }
}

template <int ROUNDS> constexpr int scatter_smem() { return KS_THREADS * ROUNDS * 8 + KS_WARPS * KS_MAX_BINS * 2 + KS_MAX_BINS * 8; }

template <int ROUNDS>
__global__ void __launch_bounds__(KS_THREADS, ROUNDS <= 4 ? 5 : 3) k_key_scatter(KeySort P, int first, int last) {
    extern __shared__ unsigned long long pairs[];                    // [tile], then the counters
    constexpr int TILE = KS_THREADS * ROUNDS, PER = (KS_MAX_BINS + KS_THREADS - 1) / KS_THREADS;
    uint16_t* cnt = reinterpret_cast<uint16_t*>(pairs + TILE);       // [warps][bins]
    int* local_start = reinterpret_cast<int*>(cnt + KS_WARPS * KS_MAX_BINS);   // first place of a digit inside the tile
    int* out_base = local_start + KS_MAX_BINS;                       // the tile's pair j of digit d goes to out_base[d] + j
    __shared__ int warp_sums[33];
    chain_wait();
    const int n = count_of(P.n), bins = 1 << P.bits, per = (bins + KS_THREADS - 1) / KS_THREADS;
    const int2 span = span_of(P.within);
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, shift = 32 + P.shift;
    for (int tile = blockIdx.x; tile < P.tiles; tile += gridDim.x) {
        if ((int64_t)tile * TILE >= n) return;
        __syncthreads();
        for (int i = threadIdx.x; i < KS_WARPS * bins / 2; i += KS_THREADS) {
            const int w = i / (bins / 2);
            reinterpret_cast<uint32_t*>(cnt + w * KS_MAX_BINS)[i - w * (bins / 2)] = 0;
        }
        unsigned long long key[ROUNDS];
        int rank[ROUNDS];
        const int64_t wbase = (int64_t)tile * TILE + wid * (ROUNDS * 32);
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const int64_t i = wbase + r * 32 + lane;
            key[r] = i < n ? (first ? first_word(P, span, (int)i) : __ldcg(P.src + i)) : ~0ull;   // padding sorts last, behind position n
        }
        __syncthreads();
        rank_rounds(key, shift, P.bits, cnt + wid * KS_MAX_BINS, rank);
        __syncthreads();
        int sums[PER], all = 0;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            sums[j] = 0;
            const int d = (int)threadIdx.x * per + j;
            if (j < per && d < bins) {
                int sum = 0;
#pragma unroll
                for (int w = 0; w < KS_WARPS; ++w) {
                    const int c = cnt[w * KS_MAX_BINS + d];
                    cnt[w * KS_MAX_BINS + d] = (uint16_t)sum;
                    sum += c;
                }
                sums[j] = sum;
                all += sum;
            }
        }
        int total;
        int at = block_exclusive_scan<KS_THREADS>(all, warp_sums, &total);
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int d = (int)threadIdx.x * per + j;
            if (j < per && d < bins) {
                local_start[d] = at;
                out_base[d] = __ldcg(P.counts + (size_t)d * P.tiles + tile) - at;
                at += sums[j];
            }
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const uint32_t d = (uint32_t)(key[r] >> shift) & (uint32_t)(bins - 1);
            pairs[local_start[d] + cnt[wid * KS_MAX_BINS + d] + rank[r]] = key[r];
        }
        __syncthreads();
        for (int j = threadIdx.x; j < TILE; j += KS_THREADS) {
            const unsigned long long w = pairs[j];
            const int64_t to = (int64_t)out_base[(uint32_t)(w >> shift) & (uint32_t)(bins - 1)] + j;
            if (to < 0 || to >= n) continue;                          // padding
            if (last) {
                P.out_keys[to] = (uint32_t)(w >> 32);
                P.out_payload[to] = (int32_t)(uint32_t)w;
            } else {
                P.dst[to] = w;
            }
        }
    }
}

// The rest of the grid clears memory for the caller meanwhile: a sort of so few pairs keeps a few SMs busy.
__device__ __forceinline__ void fill_zero(const Fill& f, int block, int blocks) {
    const uint4 zero = make_uint4(0, 0, 0, 0);
    for (int64_t i = (int64_t)block * blockDim.x + threadIdx.x; i < f.pieces; i += (int64_t)blocks * blockDim.x) __stcs(f.p + i, zero);
    if (block == 0 && (int)threadIdx.x < f.tail) reinterpret_cast<char*>(f.p + f.pieces)[threadIdx.x] = 0;
}

// All passes in one block; the others clear memory.
__global__ void __launch_bounds__(KS_SMALL_THREADS) k_key_sort_small(KeySort P, Fill f) {
    constexpr int R = KS_SMALL / KS_SMALL_THREADS, W = KS_SMALL_THREADS / 32, BINS = KC_BINS;
    extern __shared__ unsigned long long pairs[];                    // [KS_SMALL], then cnt[W][BINS]
    uint16_t* cnt = reinterpret_cast<uint16_t*>(pairs + KS_SMALL);
    __shared__ int start[BINS];
    __shared__ int warp_sums[33];
    chain_wait();
    if (blockIdx.x > 0) {
        fill_zero(f, blockIdx.x - 1, gridDim.x - 1);
        return;
    }
    const int n = count_of(P.n);
    const int2 span = span_of(P.within);
    for (int i = threadIdx.x; i < P.zero_words; i += KS_SMALL_THREADS) P.zero[i] = 0;
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    unsigned long long key[R];
    int rank[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int i = wid * (R * 32) + r * 32 + lane;
        key[r] = i < n ? first_word(P, span, i) : ~0ull;
    }
    const uint32_t mask = (1u << P.bits) - 1u;
    for (int p = 0; p < P.passes; ++p) {
        const int shift = 32 + P.bits * p;
        for (int t = threadIdx.x; t < W * BINS / 2; t += KS_SMALL_THREADS) reinterpret_cast<uint32_t*>(cnt)[t] = 0;
        __syncthreads();
        rank_rounds(key, shift, P.bits, cnt + wid * BINS, rank);
        __syncthreads();
        int sum = 0;
        if (threadIdx.x < BINS) {
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const int c = cnt[w * BINS + threadIdx.x];
                cnt[w * BINS + threadIdx.x] = (uint16_t)sum;
                sum += c;
            }
        }
        int total;
        const int s = block_exclusive_scan<KS_SMALL_THREADS>(sum, warp_sums, &total);
        if (threadIdx.x < BINS) start[threadIdx.x] = s;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const uint32_t dg = (uint32_t)(key[r] >> shift) & mask;
            pairs[start[dg] + cnt[wid * BINS + dg] + rank[r]] = key[r];
        }
        __syncthreads();
        if (p + 1 < P.passes) {
#pragma unroll
            for (int r = 0; r < R; ++r) key[r] = pairs[wid * (R * 32) + r * 32 + lane];
        }
        __syncthreads();
    }
    for (int j = threadIdx.x; j < n; j += KS_SMALL_THREADS) {
        P.out_keys[j] = (uint32_t)(pairs[j] >> 32);
        P.out_payload[j] = (int32_t)(uint32_t)pairs[j];
    }
}

__global__ void __launch_bounds__(KS_SMALL_THREADS) k_fill(Fill f) {
    chain_wait();
    fill_zero(f, blockIdx.x, gridDim.x);
}

// All passes in one cluster (40,961 ids of 18 bits: 33 us, the clearing of 87 MB beside it; bound by the ballots of the ranks): every block ranks its share, the blocks read one another's digit counts, and every pair goes
// straight to its place in the shared memory of the block that holds it next.
__global__ void __cluster_dims__(KC_BLOCKS, 1, 1) __launch_bounds__(1024) k_key_sort_cluster(KeySort P, Fill f) {
    namespace cg = cooperative_groups;
    constexpr int W = 32;
    extern __shared__ unsigned long long pairs[];                    // two buffers of KC_TILE, then the counters
    uint16_t* cnt = reinterpret_cast<uint16_t*>(pairs + 2 * KC_TILE);           // [W][KC_BINS]
    int* totals = reinterpret_cast<int*>(cnt + W * KC_BINS);         // this block's pairs per digit
    int* place = totals + KC_BINS;                                   // first place of this block's pairs of a digit
    __shared__ int warp_sums[33];
    chain_wait();
    if (blockIdx.x >= KC_BLOCKS) {                                   // whole clusters
        fill_zero(f, blockIdx.x - KC_BLOCKS, gridDim.x - KC_BLOCKS);
        return;
    }
    cg::cluster_group cluster = cg::this_cluster();
    const int n = count_of(P.n), me = blockIdx.x, bins = 1 << P.bits;
    const int2 span = span_of(P.within);
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    if (me == 0)
        for (int i = threadIdx.x; i < P.zero_words; i += 1024) P.zero[i] = 0;
    unsigned long long key[KC_ROUNDS];
    int rank[KC_ROUNDS];
#pragma unroll
    for (int r = 0; r < KC_ROUNDS; ++r) {
        const int i = me * KC_TILE + wid * (KC_ROUNDS * 32) + r * 32 + lane;
        key[r] = i < n ? first_word(P, span, i) : ~0ull;                   // padding sorts last, behind position n
    }
    for (int p = 0; p < P.passes; ++p) {
        const int shift = 32 + P.bits * p;
        unsigned long long* to = pairs + (p & 1) * KC_TILE;
        for (int i = threadIdx.x; i < W * KC_BINS / 2; i += 1024) reinterpret_cast<uint32_t*>(cnt)[i] = 0;
        __syncthreads();
        rank_rounds(key, shift, P.bits, cnt + wid * KC_BINS, rank);
        __syncthreads();
        if (threadIdx.x < bins) {
            int sum = 0;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const int c = cnt[w * KC_BINS + threadIdx.x];
                cnt[w * KC_BINS + threadIdx.x] = (uint16_t)sum;
                sum += c;
            }
            totals[threadIdx.x] = sum;
        }
        // in digit order first, so that neighbouring threads send runs, not single pairs, to the other blocks
        const int mine = threadIdx.x < bins ? totals[threadIdx.x] : 0;
        int total;
        const int local = block_exclusive_scan<1024>(mine, warp_sums, &total);
        if (threadIdx.x < bins) place[threadIdx.x] = local;
        cluster.sync();                                              // the counts are there; the last pass's pairs are read
        unsigned long long* staged = pairs + (~p & 1) * KC_TILE;
#pragma unroll
        for (int r = 0; r < KC_ROUNDS; ++r) {
            const uint32_t d = (uint32_t)(key[r] >> shift) & (uint32_t)(bins - 1);
            staged[place[d] + cnt[wid * KC_BINS + d] + rank[r]] = key[r];
        }
        int before = 0, all = 0;
        if (threadIdx.x < bins) {
#pragma unroll
            for (int c = 0; c < KC_BLOCKS; ++c) {
                const int t = cluster.map_shared_rank(totals, c)[threadIdx.x];
                if (c < me) before += t;
                all += t;
            }
        }
        const int start = block_exclusive_scan<1024>(all, warp_sums, &total);
        if (threadIdx.x < bins) place[threadIdx.x] = start + before - local;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < KC_ROUNDS; ++r) {
            const int j = r * 1024 + threadIdx.x;
            const unsigned long long w = staged[j];
            const int at = place[(uint32_t)(w >> shift) & (uint32_t)(bins - 1)] + j;
            cluster.map_shared_rank(to, at / KC_TILE)[at % KC_TILE] = w;
        }
        cluster.sync();                                              // all pairs have arrived, all counts are read
#pragma unroll
        for (int r = 0; r < KC_ROUNDS; ++r) key[r] = to[wid * (KC_ROUNDS * 32) + r * 32 + lane];
    }
#pragma unroll
    for (int r = 0; r < KC_ROUNDS; ++r) {
        const int i = me * KC_TILE + wid * (KC_ROUNDS * 32) + r * 32 + lane;
        if (i < n) {
            P.out_keys[i] = (uint32_t)(key[r] >> 32);
            P.out_payload[i] = (int32_t)(uint32_t)key[r];
        }
    }
}

static int64_t ks_tile(int64_t n) { return KS_THREADS * (n < KS_LARGE ? KS_ROUNDS_SMALL : KS_ROUNDS_LARGE); }
static int64_t ks_tiles(int64_t n) { return (n + ks_tile(n) - 1) / ks_tile(n); }

size_t key_sort_bytes(int64_t n) {
    return align_up((size_t)n * 8, 256) * 2 + align_up((size_t)KS_MAX_PASSES * KS_MAX_BINS * 4, 256) + align_up((size_t)KS_MAX_BINS * ks_tiles(n) * 4, 256) + 256;
}

template <int ROUNDS> static cudaError_t run_pass(const KeySort& P, bool first, bool last, cudaStream_t s) {
    static std::atomic<uint64_t> allowed{0};
    cudaError_t e = allow_smem(k_key_scatter<ROUNDS>, scatter_smem<ROUNDS>(), allowed);
    if (e == cudaSuccess) e = launch_train(k_key_count<ROUNDS>, P.tiles, KS_THREADS, 0, s, P, (int)first);
    if (e == cudaSuccess) e = launch_train(k_key_scan, ((1 << P.bits) + 7) / 8, 256, 0, s, P);
    if (e == cudaSuccess) e = launch_train(k_key_scatter<ROUNDS>, P.tiles, KS_THREADS, scatter_smem<ROUNDS>(), s, P, (int)first, (int)last);
    return e;
}

cudaError_t launch_key_sort(const int32_t* keys, const int32_t* payload, Count n, Rows within, int64_t key_limit, void* workspace,
                            uint32_t* out_keys, int32_t* out_payload, int32_t* zero, int zero_words, Fill fill, cudaStream_t s) {
    KeySort P{};
    P.keys = keys;
    P.payload = payload;
    P.n = n;
    P.within = within;
    P.key_limit = (uint32_t)key_limit;
    P.out_keys = out_keys;
    P.out_payload = out_payload;
    P.zero = zero;
    P.zero_words = zero_words;
    int bits = 1;
    while (bits < 32 && (key_limit >> bits)) ++bits;
    // blocks that clear memory beside the sort: enough for all SMs, each with a few kilobytes at least
    int64_t fillers = fill.pieces / 4096;
    if (fillers > sm_count() - KC_BLOCKS) fillers = sm_count() - KC_BLOCKS;
    fillers = (fillers + (fill.pieces > 0)) / KC_BLOCKS * KC_BLOCKS + (fill.pieces > 0 ? KC_BLOCKS : 0);
    cudaError_t e = cudaSuccess;
    if (n.bound > KS_SMALL && n.bound <= KC_MAX && limit_grid(KC_BLOCKS + fillers) == KC_BLOCKS + fillers) {
        constexpr int smem = 2 * KC_TILE * 8 + 32 * KC_BINS * 2 + 2 * KC_BINS * 4;
        static std::atomic<uint64_t> allowed{0};
        P.passes = (bits + KC_BITS - 1) / KC_BITS;
        P.bits = (bits + P.passes - 1) / P.passes;
        e = allow_smem(k_key_sort_cluster, smem, allowed);
        if (e != cudaSuccess) return e;
        return launch_train(k_key_sort_cluster, KC_BLOCKS + fillers, 1024, smem, s, P, fill);
    }
    if (n.bound <= KS_SMALL && limit_grid(1 + fillers) == 1 + fillers) {
        constexpr int smem = KS_SMALL * 8 + (KS_SMALL_THREADS / 32) * KC_BINS * 2;
        P.passes = (bits + KC_BITS - 1) / KC_BITS;
        P.bits = (bits + P.passes - 1) / P.passes;
        static std::atomic<uint64_t> allowed{0};
        e = allow_smem(k_key_sort_small, smem, allowed);
        if (e != cudaSuccess) return e;
        return launch_train(k_key_sort_small, 1 + fillers, KS_SMALL_THREADS, smem, s, P, fill);
    }
    if (fill.pieces > 0) e = launch_train(k_fill, fillers, KS_SMALL_THREADS, 0, s, fill);
    if (e != cudaSuccess) return e;
    P.passes = (bits + KS_MAX_BITS - 1) / KS_MAX_BITS;
    P.bits = (bits + P.passes - 1) / P.passes;
    P.tiles = (int)ks_tiles(n.bound);
    const size_t buf = align_up((size_t)n.bound * 8, 256);
    char* ws = (char*)workspace;
    unsigned long long* a = (unsigned long long*)ws;
    unsigned long long* b = (unsigned long long*)(ws + buf);
    int32_t* totals = (int32_t*)(ws + 2 * buf);
    P.counts = (int32_t*)(ws + 2 * buf + align_up((size_t)KS_MAX_PASSES * KS_MAX_BINS * 4, 256));
    e = cudaMemsetAsync(totals, 0, (size_t)P.passes * KS_MAX_BINS * 4, s);
    for (int p = 0; p < P.passes && e == cudaSuccess; ++p) {
        P.shift = P.bits * p;
        P.totals = totals + KS_MAX_BINS * p;
        P.src = (p & 1) ? a : b;
        P.dst = (p & 1) ? b : a;
        const bool first = p == 0, last = p + 1 == P.passes;
        e = n.bound < KS_LARGE ? run_pass<KS_ROUNDS_SMALL>(P, first, last, s) : run_pass<KS_ROUNDS_LARGE>(P, first, last, s);
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

}  // namespace gs
