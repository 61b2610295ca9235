// Softmax cross entropy against a table on the tensor cores: bf16 operands of up to 256 columns.
//
// A block keeps a tile of 128 rows of x in shared memory (hidden rows for the forward pass and dh, table rows for dw)
// and lets tiles of 128 rows of y stream by (TMA, 128-byte swizzle).  Unit u of a block:
//   S = X Y^T (tcgen05, 128 x 128, f32 in tensor memory)  ->  a softmax warpgroup turns S into statistics, or into
//   Z = dz in bf16 that overwrites S in tensor memory     ->  O += Z Y, the same shared-memory tile of Y as the second
// operand, read along its other dimension.  Rounding Z to bf16 costs up to 2^-8 of each term, as the gradient's own
// rounding to bf16 does; the entries of labels are rounded in two parts (LabelUnits).
// Roles: one warp issues the loads, one the products S, one the products O, one the copies of finished tiles out; sixteen
// warps weigh, eight to a unit (a thread per row and 64 columns), the two groups of eight in turn, so that S of one unit is
// multiplied while another is exponentiated.  S of a later unit may overwrite a Z once the product that read it has ended.
// Work is cut into equal runs of units, one per SM; a row of tiles shared by runs is joined from f32 partials.
// Bound: forward by the exponentials (one per logit; special-function and multiply-add units share them), backward by the
// reads of X, Y and Y again from shared memory beside them.  8,192 x 169,343 x 128: forward 357 us (0.99 PFLOP/s), dh 481 us and
// dw 571 us (1.5 and 1.2 PFLOP/s over their two products).
#include <atomic>
#include <type_traits>

#include "gs_device.cuh"
#include "gs_tc.cuh"
#include "gs_train.cuh"
#include "gs_train.h"
#include "gs_xent.h"

namespace gs {

constexpr int XT = XENT_TC_TILE;
constexpr int XT_THREADS = 640;            // 4 warps of roles, 4 softmax warpgroups: two per unit, 64 columns each
constexpr int XT_CHUNK = XT * 128;         // bytes of a tile's 64 columns
constexpr int XT_MAX_STAGES = 8;
constexpr long long XT_UNIT_CLOCKS = 1000000;   // more than five hundred times what a unit takes
constexpr float XT_LOG2E = 1.4426950408889634f;

__device__ int g_xent_gave_up;

__device__ __forceinline__ float xt_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// 2^x for x <= 0 by the multiply-add units, two at a time: x = n + f with n the nearest integer (taken from the low bits
// of x + 1.5 * 2^23), 2^f by a polynomial on [-1/2, 1/2] (minimax in relative error with the constant 1 fixed, found by
// reweighted least squares: 1.9e-7 with degree 5, 2.9e-6 with degree 4), 2^n from its exponent bits.  x is cut at -126; NaN
// passes through.  The special-function units give 16 exponentials per clock and SM; every third pair or so comes from here.
template <int DEGREE> __device__ __forceinline__ f32x2 exp2_by_fma(f32x2 x) {
    constexpr float C5[5] = {0.6931470036506653f, 0.24022242426872253f, 0.05550733581185341f, 0.009671512991189957f, 0.001326472731307149f};
    constexpr float C4[4] = {0.6931241750717163f, 0.24024099111557007f, 0.055906426161527634f, 0.009582852944731712f};
    float lo, hi;
    split(x, lo, hi);
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(lo) : "f"(-126.f));
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(hi) : "f"(-126.f));
    x = pair(lo, hi);
    const f32x2 magic = pair(12583039.f, 12583039.f), minus = pair(-12583039.f, -12583039.f), one = pair(1.f, 1.f), neg = pair(-1.f, -1.f);
    const f32x2 r = add2(x, magic);                       // 1.5 * 2^23 + 127 + n
    const f32x2 f = fma2(add2(r, minus), neg, x);
    f32x2 p;
    if constexpr (DEGREE == 5) {
        p = pair(C5[4], C5[4]);
#pragma unroll
        for (int i = 3; i >= 0; --i) p = fma2(p, f, pair(C5[i], C5[i]));
    } else {
        p = pair(C4[3], C4[3]);
#pragma unroll
        for (int i = 2; i >= 0; --i) p = fma2(p, f, pair(C4[i], C4[i]));
    }
    p = fma2(p, f, one);
    split(r, lo, hi);
    return mul2(p, pair(__uint_as_float(__float_as_uint(lo) << 23), __uint_as_float(__float_as_uint(hi) << 23)));
}

// 2^x of pair j of 16: the multiply-add units take 4 of 16 pairs forward, 2 of 16 backward (there the tensor cores set
// the pace).  Measured side by side at 8,192 x 169,343 x 128 (an earlier forward, 369 us): forward 369 us with 4, 387 with 5,
// 396 with 6 pairs, 443 with none; backward 1,083 us with 2, 1,078 with none (64 columns: 902 and 969), 1,098 with 4.
constexpr int FMA_PAIRS_FORWARD = 0x2222, FMA_PAIRS_BACKWARD = 0x0202;
template <bool FORWARD> __device__ __forceinline__ f32x2 exp2_pair(f32x2 x, int j) {
    if (((FORWARD ? FMA_PAIRS_FORWARD : FMA_PAIRS_BACKWARD) >> j) & 1) return exp2_by_fma<FORWARD ? 5 : 4>(x);
    float lo, hi;
    split(x, lo, hi);
    return pair(xt_exp2(lo), xt_exp2(hi));
}

struct XentTc {
    Xent a;
    Runs runs;
    int nx, ny;
    int on;                      // columns of O: dim rounded up to 16
    int stages, xbufs;           // tiles of y and of x in shared memory
    int sbufs, obufs;            // buffers of S and of O in tensor memory: O(i) starts at column 128 sbufs + i * on_pitch
    int on_pitch;
    int out, out_pitch;          // backward: OUT_*, bytes between the staged rows
    float2* stats;               // forward: [parts + tiles_x][XENT_TC_STATS][XT]
    float* picked;
    float* partial;              // backward: [2 parts][XT][on]
    const uint32_t* marks;       // backward: [tiles of hidden rows][mark_words] bits, the tiles of the table with a label of these rows
    int mark_words;
    const float* row_info;       // dw: [tiles of hidden rows][3][XT]: -lse (base 2), upstream gradient times scale, label
};
constexpr int XT_INFO = 3 * XT * 4;        // bytes of a tile's row_info
// How a finished tile of bf16 gradients leaves: lane by lane; or through shared memory and then by bulk copies, a row each
// (rows on 16 bytes) or the whole tile at once (rows without gaps, wherever they start).
enum { OUT_DIRECT = 0, OUT_ROWS = 1, OUT_TILE = 2 };

// The block's runs, cut at rows of tiles.
struct Segments {
    const Runs& r;
    int64_t run, t, end;
    int step;
    __device__ Segments(const Runs& runs, int first, int step_) : r(runs), run(first), step(step_) {
        t = run < r.parts ? r.start(run) : 0;
        end = run < r.parts ? r.start(run + 1) : 0;
    }
    // Next segment: row xi, tiles [y0, y0 + n) of it; false when the block is done.
    __device__ bool next(int64_t& run_out, int64_t& xi, int& y0, int& n) {
        while (t >= end) {
            run += step;
            if (run >= r.parts) return false;
            t = r.start(run);
            end = r.start(run + 1);
        }
        xi = t / r.tiles_y;
        const int64_t last = (xi + 1) * r.tiles_y < end ? (xi + 1) * r.tiles_y : end;
        y0 = (int)(t - xi * r.tiles_y);
        n = (int)(last - t);
        t = last;
        run_out = run;
        return true;
    }
};

// 16 columns of a gradient row (fewer at its end), in 16-byte pieces where the address allows.
__device__ __forceinline__ void store_columns(void* to, gs_dtype t, int64_t at, const float (&f)[16], int left) {
    if (t == GS_BF16) {
        bf16* p = static_cast<bf16*>(to) + at;
        if (left >= 16 && ((uintptr_t)p & 15) == 0) return store_vec<bf16, 16>(p, f);
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (j < left) p[j] = from_f32<bf16>(f[j]);
    } else {
        float* p = static_cast<float*>(to) + at;
        if (left >= 16 && ((uintptr_t)p & 15) == 0) return store_vec<float, 16>(p, f);
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (j < left) p[j] = f[j];
    }
}

enum { TC_FORWARD = 0, TC_DHIDDEN = 1, TC_DTABLE = 2 };

__device__ __forceinline__ float4 shared_f4(uint32_t a) {
    float4 r;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(r.x), "=f"(r.y), "=f"(r.z), "=f"(r.w) : "r"(a));
    return r;
}
__device__ __forceinline__ int shared_i(uint32_t a) {
    int r;
    asm volatile("ld.shared.s32 %0, [%1];" : "=r"(r) : "r"(a));
    return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ float min3(float a, float b, float c) {
    float r;
    asm("min.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// Where a unit holds entries of labels.  p - 1 of a small p lies just under one, where bf16 drops p: up to 2^-9 of the
// entry, the same way in every row of a label, so that nothing averages it out (512 columns: 0.003 of the table's gradient,
// where rounding it takes 0.0017).  The 16 columns of Z around such an entry are multiplied in two parts, the second what the
// rounding took from the first, in the columns of S beside it.  Only those 16: frequent labels lie together in the
// table, and the block that has them would be the last (8,192 x 169,343 x 128, labels by a squared law: both gradients
// 1,030 us without the second part, 1,112 with it, 1,238 with all 128 columns of every such unit).
// The warps that write Z and the one that multiplies it find the places alike: marked units from memory, 32 of a segment at
// a time, the columns from the labels.
struct LabelUnits {
    uint32_t mask;
    // before unit i of a segment of n units, by all lanes of a warp: whether it is marked
    template <int M> __device__ bool marked(int i, int64_t xi, int y0, int n, const uint32_t* marks, int words) {
        if ((i & 31) == 0) {
            const int y = i + (threadIdx.x & 31);
            const int64_t hidden = M == TC_DHIDDEN ? xi : y0 + y, table = M == TC_DHIDDEN ? y0 + y : xi;
            mask = __ballot_sync(FULL, y < n && (__ldcg(marks + hidden * words + (table >> 5)) >> (table & 31) & 1));
        }
        return mask >> (i & 31) & 1;
    }
    // Bit 4 k: columns 16 k .. 16 k + 15 of tile y hold a label's entry.  dh: the labels of the rows of tile xi; dw: the
    // columns are the hidden rows whose info lies at `at`.
    template <int M> static __device__ uint32_t columns(const Xent& a, int64_t xi, int y, uint32_t at) {
        const int lane = threadIdx.x & 31;
        uint32_t m = 0;
        if (M == TC_DHIDDEN) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t x = xi * XT + lane * 4 + j;
                const int lab = x < a.rows ? __ldg(a.labels + x) : -1;
                if (lab >= 0 && lab < a.vocab && lab / XT == y) m |= 1u << (lab % XT / 16 * 4);
            }
            return __reduce_or_sync(FULL, m);
        }
        int lab[4];
        asm volatile("ld.shared.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(lab[0]), "=r"(lab[1]), "=r"(lab[2]), "=r"(lab[3]) : "r"(at + (2 * XT + lane * 4) * 4));
        const int from = (int)(xi * XT);
#pragma unroll
        for (int j = 0; j < 4; ++j) m |= (uint32_t)(lab[j] - from) < (uint32_t)XT;       // -1 is in no tile
        m = __ballot_sync(FULL, m);                                                      // four lanes to 16 columns
        m |= m >> 1;
        m |= m >> 2;
        return m & 0x11111111u;
    }
};

// CHUNKS: 64-column pieces of a row, known at compile time so that the issuing warp's code is straight.
template <int M, int CHUNKS>
__global__ void __launch_bounds__(XT_THREADS, 1) k_xent_tc(const __grid_constant__ XentTc P, const __grid_constant__ CUtensorMap xmap,
                                                           const __grid_constant__ CUtensorMap ymap) {
    extern __shared__ unsigned char tiles[];
    __shared__ __align__(8) unsigned long long bars[2 * XT_MAX_STAGES + 24];
    __shared__ uint32_t s_tmem;
    __shared__ volatile int s_stop;
    const int SBUFS = M == TC_FORWARD ? 4 : P.sbufs;
    const int warp = __shfl_sync(FULL, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    constexpr uint32_t tile_bytes = CHUNKS * XT_CHUNK;
    const uint32_t xbase = (tc::smem_addr(tiles) + 1023) & ~1023u, ring = xbase + P.xbufs * tile_bytes;
    const uint32_t info = ring + P.stages * tile_bytes;      // dw: row_info of the stages' tiles
    const uint32_t staging = info + (M == TC_DTABLE ? P.stages * XT_INFO : 0);
    const uint32_t b0 = tc::smem_addr(bars);
    auto full = [&](int i) { return b0 + 8 * i; };
    auto empty = [&](int i) { return b0 + 8 * (XT_MAX_STAGES + i); };
    const uint32_t b1 = b0 + 16 * XT_MAX_STAGES;
    auto s_full = [&](int i) { return b1 + 8 * i; };         // 4: S of a unit is in tensor memory
    auto p_full = [&](int i) { return b1 + 32 + 8 * i; };    // 4: Z is written (forward: S may be overwritten)
    auto x_full = [&](int i) { return b1 + 64 + 8 * i; };    // 2
    auto x_free = [&](int i) { return b1 + 80 + 8 * i; };    // 2
    auto o_full = [&](int i) { return b1 + 96 + 8 * i; };    // 2
    auto o_free = [&](int i) { return b1 + 112 + 8 * i; };   // 2
    auto z_free = [&](int i) { return b1 + 128 + 8 * i; };   // 4: Z of a unit has been multiplied (backward)
    const uint32_t staged = b1 + 176, unstaged = b1 + 184;   // the tile is in shared memory; its copies have read it
    auto drained = [&](int i) { return b1 + 160 + 8 * i; };  // 2: the products of a role that gives up

    if (threadIdx.x == 0) {
        s_stop = 0;
        for (int i = 0; i < P.stages; ++i) {
            tc::mbar_init(full(i), 1);
            tc::mbar_init(empty(i), 1);
        }
        for (int i = 0; i < 4; ++i) {
            tc::mbar_init(s_full(i), 1);
            tc::mbar_init(p_full(i), 256);
            tc::mbar_init(z_free(i), 1);
        }
        for (int i = 0; i < 2; ++i) {
            tc::mbar_init(x_full(i), 1);
            tc::mbar_init(x_free(i), 1);
            tc::mbar_init(o_full(i), 1);
            tc::mbar_init(o_free(i), 512);
        }
        tc::mbar_init(staged, 512);
        tc::mbar_init(unstaged, 32);
        tc::mbar_init(drained(0), 1);
        tc::mbar_init(drained(1), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 2) tc::tmem_alloc(tc::smem_addr(&s_tmem), 512);
    chain_wait();                                          // what is set up above may overlap the kernel before
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t tmem = __shfl_sync(FULL, s_tmem, 0);
    // a whole tile of 128 rows can leave in one copy; its last, shorter neighbour goes lane by lane
    auto stages_tile = [&](int64_t i) { return P.out == OUT_ROWS || (P.out == OUT_TILE && (i + 1) * XT <= P.nx); };
    // A role that gives up: its products still write tensor memory, which must not be freed under them.
    auto drain = [&](uint32_t bar) {
        if (tc::elect_one()) {
            atomicExch(&g_xent_gave_up, 1);
            tc::commit(bar);
        }
        __syncwarp();
        const long long begin = clock64();
        while (!tc::mbar_try(bar, 0) && clock64() - begin < tc::WAIT_CLOCKS) {}
    };
    Segments seg(P.runs, blockIdx.x, gridDim.x);
    int64_t run, xi;
    int y0, n;

    if (warp == 0) {
        {                                                  // ---- loads
            int st = 0, issued = 0, segs = 0;
            uint32_t ph = 0;
            bool ok = true;
            while (ok && seg.next(run, xi, y0, n)) {
                const int xb = segs % P.xbufs;
                if (segs >= P.xbufs) ok = __all_sync(FULL, tc::mbar_wait(x_free(xb), (uint32_t)(segs / P.xbufs - 1) & 1, &s_stop));
                if (!ok) break;
                if (tc::elect_one()) {
                    tc::mbar_expect(x_full(xb), tile_bytes);
                    for (int c = 0; c < CHUNKS; ++c) tc::tma_load(xbase + xb * tile_bytes + c * XT_CHUNK, &xmap, c * 64, (int)(xi * XT), x_full(xb));
                }
                __syncwarp();
                ++segs;
                for (int i = 0; i < n; ++i) {
                    if (issued >= P.stages) ok = __all_sync(FULL, tc::mbar_wait(empty(st), ph ^ 1, &s_stop));
                    if (!ok) break;
                    if (tc::elect_one()) {
                        tc::mbar_expect(full(st), tile_bytes + (M == TC_DTABLE ? XT_INFO : 0));
                        if (M == TC_DTABLE) tc::bulk_load(info + st * XT_INFO, P.row_info + (int64_t)(y0 + i) * (XT_INFO / 4), XT_INFO, full(st));
                        for (int c = 0; c < CHUNKS; ++c) tc::tma_load(ring + st * tile_bytes + c * XT_CHUNK, &ymap, c * 64, (y0 + i) * XT, full(st));
                    }
                    __syncwarp();
                    ++issued;
                    if (++st == P.stages) {
                        st = 0;
                        ph ^= 1;
                    }
                }
            }
            if (!ok) atomicExch(&g_xent_gave_up, 1);
            // no copy may be in flight when the block ends, whatever became of the other roles
            const long long begin = clock64();
            for (int j = issued > P.stages ? issued - P.stages : 0; j < issued; ++j)
                while (!tc::mbar_try(full(j % P.stages), (uint32_t)(j / P.stages) & 1) && clock64() - begin < tc::WAIT_CLOCKS) {}
            for (int j = segs > P.xbufs ? segs - P.xbufs : 0; j < segs; ++j)
                while (!tc::mbar_try(x_full(j % P.xbufs), (uint32_t)(j / P.xbufs) & 1) && clock64() - begin < tc::WAIT_CLOCKS) {}
        }
    } else if (warp == 1) {                                // ---- first products: S
        const uint32_t inst = tc::instruction(XT, false);
        const uint64_t xd = tc::operand(xbase, 16, 1024), yd = tc::operand(ring, 16, 1024);
        constexpr uint32_t tile_step = tile_bytes >> 4;    // in the operands' units of 16 bytes
        int st = 0, b = 0, segs = 0;
        uint32_t ph = 0, bph = 0;
        bool ok = true, reuse = false;
        auto wait = [&](uint32_t bar, uint32_t parity) { ok = ok && __all_sync(FULL, tc::mbar_wait(bar, parity, &s_stop)); };
        while (ok && seg.next(run, xi, y0, n)) {
            const int xb = segs % P.xbufs;
            wait(x_full(xb), (uint32_t)(segs / P.xbufs) & 1);
            ++segs;
            for (int i = 0; i < n; ++i) {
                wait(full(st), ph);
                if (reuse) wait(M == TC_FORWARD ? p_full(b) : z_free(b), bph ^ 1);
                if (!ok) break;
                tc::fence_after();
                const uint64_t a = xd + (uint32_t)xb * tile_step, y = yd + (uint32_t)st * tile_step;
                const uint32_t d = tmem + b * XT;
                if (tc::elect_one()) {
#pragma unroll
                    for (int k = 0; k < CHUNKS * 4; ++k)       // columns behind dim are zero in both operands
                        tc::mma_ss(d, a + (k >> 2) * (XT_CHUNK >> 4) + (k & 3) * 2, y + (k >> 2) * (XT_CHUNK >> 4) + (k & 3) * 2, inst, k > 0);
                    tc::commit(s_full(b));
                    if (i + 1 == n) tc::commit(x_free(xb));
                    if (M == TC_FORWARD) tc::commit(empty(st));
                }
                __syncwarp();
                if (++st == P.stages) {
                    st = 0;
                    ph ^= 1;
                }
                if (++b == SBUFS) {
                    b = 0;
                    bph ^= 1;
                    reuse = true;
                }
            }
        }
        if (!ok) drain(drained(0));
    } else if (warp == 3 && M != TC_FORWARD) {             // ---- second products: O
        const uint32_t inst = tc::instruction(P.on, true);
        const uint64_t zd = tc::operand(ring, XT_CHUNK, 1024);
        constexpr uint32_t tile_step = tile_bytes >> 4;
        int st = 0, b = 0, ob = 0, segs = 0;
        uint32_t ph = 0, bph = 0, oph = 1;                 // oph: parity of the use of O before this one; the first use waits for none
        bool ok = true;
        auto wait = [&](uint32_t bar, uint32_t parity) { ok = ok && __all_sync(FULL, tc::mbar_wait(bar, parity, &s_stop)); };
        LabelUnits units;
        while (ok && seg.next(run, xi, y0, n)) {
            const uint32_t o = tmem + SBUFS * XT + ob * P.on_pitch;
            for (int i = 0; i < n; ++i) {
                const bool marked = units.marked<M>(i, xi, y0, n, P.marks, P.mark_words);
                wait(full(st), ph);                        // long complete: the tile must be visible to this thread too
                const uint32_t labels = marked && ok ? LabelUnits::columns<M>(P.a, xi, y0 + i, info + st * XT_INFO) : 0;
                wait(p_full(b), bph);
                if (i == 0 && segs >= P.obufs) wait(o_free(ob), oph);
                if (!ok) break;
                tc::fence_after();
                const uint32_t z = tmem + b * XT;
                const uint64_t y = zd + (uint32_t)st * tile_step;
                if (tc::elect_one()) {
#pragma unroll
                    for (int k = 0; k < XT / 16; ++k)      // Z lies in four pieces, each over the columns of S it came from
                        tc::mma_ts(o, z + (k >> 1) * 32 + (k & 1) * 8, y + k * 128, inst, i > 0 || k > 0);
                    if (labels) {
#pragma unroll
                        for (int k = 0; k < XT / 16; ++k)
                            if (labels >> 4 * k & 1) tc::mma_ts(o, z + (k >> 1) * 32 + 16 + (k & 1) * 8, y + k * 128, inst, true);
                    }
                    tc::commit(empty(st));
                    tc::commit(z_free(b));
                    if (i + 1 == n) tc::commit(o_full(ob));
                }
                __syncwarp();
                if (++st == P.stages) {
                    st = 0;
                    ph ^= 1;
                }
                if (++b == SBUFS) {
                    b = 0;
                    bph ^= 1;
                }
            }
            ++segs;
            if (++ob == P.obufs) {
                ob = 0;
                oph ^= 1;
            }
        }
        if (!ok) drain(drained(1));
    } else if (warp == 2 && M != TC_FORWARD && P.out != OUT_DIRECT) {       // ---- copies of finished tiles
        bool ok = true;
        uint32_t parity = 0;
        char* grad = (char*)(M == TC_DHIDDEN ? P.a.dhidden : P.a.dtable);
        const int64_t ld = (M == TC_DHIDDEN ? P.a.dhidden_ld : P.a.dtable_ld) * 2;
        long long units = 0;                               // since the last finished tile
        while (ok && seg.next(run, xi, y0, n)) {
            units += n;
            if (y0 != 0 || n != P.runs.tiles_y || !stages_tile(xi)) continue;
            // the other roles wait for units, this one for whole rows of them: a table of 320 M rows takes over two seconds
            ok = __all_sync(FULL, tc::mbar_wait(staged, parity, &s_stop, tc::WAIT_CLOCKS + units * XT_UNIT_CLOCKS));
            units = 0;
            if (!ok) break;
            parity ^= 1;
            if (P.out == OUT_ROWS) {
                for (int r = lane; r < XT && xi * XT + r < P.nx; r += 32) tc::bulk_store(grad + (xi * XT + r) * ld, staging + r * P.out_pitch, P.a.dim * 2);
            } else if (lane == 0) {
                tc::bulk_store(grad + xi * XT * ld, staging, XT * P.a.dim * 2);
            }
            tc::bulk_commit();
            tc::bulk_wait_read();
            tc::mbar_arrive(unstaged);
        }
        tc::bulk_wait_all();
        if (!ok && lane == 0) atomicExch(&g_xent_gave_up, 1);
    } else if (warp >= 4) {                                // ---- softmax
        const int sw = warp - 4, wg = sw >> 2, half = wg & 1, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // this warp's 32 lanes of tensor memory
        const float c2 = P.a.scale * XT_LOG2E;
        bool ok = true;
        uint32_t ph = 0, bph = 0, oph = 0;
        int st = 0, b = 0, ob = 0, mine = wg >> 1, tiles_out = 0;   // mine: 0 at this pair's units
        // The sum of a finished segment.  It is taken after the first unit of the next one, when the last products have long ended.
        bool pending = false, whole = false;
        int64_t e_run = 0, e_xi = 0;
        auto epilogue = [&]() {
            pending = false;
            const int64_t x = e_xi * XT + row;
            ok = tc::mbar_wait(o_full(ob), oph, &s_stop);
            ok = __all_sync(FULL, ok);
            if (!ok) return;
            tc::fence_after();
            float factor = 1.f;
            if (M == TC_DHIDDEN && x < P.nx) {
                const int lab = __ldg(P.a.labels + x);
                factor = lab >= 0 && lab < P.a.vocab ? __ldg(P.a.dloss + x) * P.a.scale : 0.f;
            }
            const bool zero = M == TC_DHIDDEN && factor == 0.f;
            float* part = P.partial + (P.runs.slot(e_run, e_xi) * XT + row) * P.on;
            void* grad = M == TC_DHIDDEN ? P.a.dhidden : P.a.dtable;
            const int64_t grad_ld = M == TC_DHIDDEN ? P.a.dhidden_ld : P.a.dtable_ld;
            const bool stage = whole && stages_tile(e_xi);
            if (stage && tiles_out > 0) {                  // the copies of the tile before must have read the rows
                ok = __all_sync(FULL, tc::mbar_wait(unstaged, (uint32_t)(tiles_out - 1) & 1, &s_stop));
                if (!ok) return;
            }
            tiles_out += stage;
            for (int c = wg * 16; c < P.on; c += 64) {
                uint32_t q[16];
                __syncwarp();
                tc::ld16(tmem + SBUFS * XT + ob * P.on_pitch + lanes + c, q);
                tc::wait_ld(q);
                float f[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) f[j] = zero ? 0.f : __uint_as_float(q[j]) * factor;
                if (!whole) {
                    if (x < P.nx) store_vec<float, 16>(part + c, f);
                } else if (stage) {
                    const uint32_t to = staging + row * P.out_pitch + c * 2;
                    uint32_t w[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) w[j] = pack_bf16(f[2 * j], f[2 * j + 1]);
                    if (P.out == OUT_ROWS) {
                        if (c < P.a.dim) asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
                        if (c + 8 < P.a.dim) asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + 16), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
                    } else {
                        const int left = P.a.dim - c;
                        if (P.a.dim % 2 == 0) {
#pragma unroll
                            for (int j = 0; j < 8; ++j)
                                if (2 * j < left) asm volatile("st.shared.b32 [%0], %1;" ::"r"(to + 4 * j), "r"(w[j]) : "memory");
                        } else {
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                if (2 * j < left) asm volatile("st.shared.b16 [%0], %1;" ::"r"(to + 4 * j), "h"((uint16_t)w[j]) : "memory");
                                if (2 * j + 1 < left) asm volatile("st.shared.b16 [%0], %1;" ::"r"(to + 4 * j + 2), "h"((uint16_t)(w[j] >> 16)) : "memory");
                            }
                        }
                    }
                } else if (x < P.nx) {
                    store_columns(grad, P.a.grad_dtype, x * grad_ld + c, f, P.a.dim - c);
                }
            }
            tc::fence_before();
            tc::mbar_arrive(o_free(ob));
            if (stage) {
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");    // the copy engine sees the rows
                tc::mbar_arrive(staged);
            }
            if (++ob == P.obufs) {
                ob = 0;
                oph ^= 1;
            }
        };
        while (ok && seg.next(run, xi, y0, n)) {
            const int64_t x = xi * XT + row;
            float lse2 = 0.f, m = -INFINITY, l = 0.f;
            int label = -1;
            if (M != TC_DTABLE && x < P.nx) {
                const int lab = __ldg(P.a.labels + x);
                label = lab >= 0 && lab < P.a.vocab ? lab : -1;
                if (M == TC_DHIDDEN) lse2 = __ldg(P.a.lse + x) * XT_LOG2E;
            }
            LabelUnits units;
            for (int i = 0; i < n && ok; ++i, mine ^= 1, st = st + 1 == P.stages ? 0 : st + 1, ph ^= st == 0, b = b + 1 == SBUFS ? 0 : b + 1, bph ^= b == 0) {
                const bool marked = M != TC_FORWARD && units.marked<M>(i, xi, y0, n, P.marks, P.mark_words);
                if (mine) continue;
                const int ybase = (y0 + i) * XT + half * 64;
                const uint32_t cols = info + st * XT_INFO + half * 64 * 4;      // dw: row_info of this warp's columns
                if (M == TC_DTABLE) {
                    ok = tc::mbar_wait(full(st), ph, &s_stop);
                    if (!__all_sync(FULL, ok)) {
                        ok = false;
                        break;
                    }
                }
                ok = tc::mbar_wait(s_full(b), bph, &s_stop);
                ok = __all_sync(FULL, ok);
                if (!ok) break;
                tc::fence_after();
                const uint32_t sa = tmem + b * XT + half * 64 + lanes;
                // backward: 32 columns of S become Z
                auto weigh = [&](auto labels, int c) {
                    constexpr bool LABELS = decltype(labels)::value;
                    uint32_t q[32];
                    tc::ld32(sa + 32 * c, q);
                    tc::wait_ld(q);
                    const int col = ybase + c * 32;
                    f32x2 f[16];
                    const f32x2 c22 = pair(c2, c2);
                    uint32_t mask = 0;                 // this row's label entries among the 32 columns
                    if (M == TC_DHIDDEN) {
                        const f32x2 r2 = pair(-lse2, -lse2);
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            f[j] = exp2_pair<false>(fma2(pair(__uint_as_float(q[2 * j]), __uint_as_float(q[2 * j + 1])), c22, r2), j);
                        if (LABELS) {
                            if (label >= col && label < col + 32) mask = 1u << (label - col);
#pragma unroll
                            for (int j = 0; j < 16; ++j) f[j] = add2(f[j], pair(mask >> 2 * j & 1 ? -1.f : 0.f, mask >> (2 * j + 1) & 1 ? -1.f : 0.f));
                        }
                        if (col + 32 > P.ny) {
#pragma unroll
                            for (int j = 0; j < 16; ++j) {
                                float lo, hi;
                                split(f[j], lo, hi);
                                f[j] = pair(col + 2 * j < P.ny ? lo : 0.f, col + 2 * j + 1 < P.ny ? hi : 0.f);
                            }
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 16; j += 2) {
                            const float4 ls = shared_f4(cols + (c * 32 + 2 * j) * 4);
                            f[j] = exp2_pair<false>(fma2(pair(__uint_as_float(q[2 * j]), __uint_as_float(q[2 * j + 1])), c22, pair(ls.x, ls.y)), j);
                            f[j + 1] = exp2_pair<false>(fma2(pair(__uint_as_float(q[2 * j + 2]), __uint_as_float(q[2 * j + 3])), c22, pair(ls.z, ls.w)), j + 1);
                        }
                        if (LABELS) {
                            const int lab = shared_i(cols + (2 * XT + c * 32 + lane) * 4) - ((int)(xi * XT) + (warp & 3) * 32);
                            mask = __ballot_sync(FULL, lab >= 0 && lab < 32);      // columns whose label is this lane's row
#pragma unroll
                            for (int k = 0; k < 5; ++k) {
                                const uint32_t ones = __ballot_sync(FULL, lab >> k & 1);
                                mask &= lane >> k & 1 ? ones : ~ones;
                            }
#pragma unroll
                            for (int j = 0; j < 16; ++j) f[j] = add2(f[j], pair(mask >> 2 * j & 1 ? -1.f : 0.f, mask >> (2 * j + 1) & 1 ? -1.f : 0.f));
                        }
#pragma unroll
                        for (int j = 0; j < 16; j += 2) {
                            const float4 g = shared_f4(cols + (XT + c * 32 + 2 * j) * 4);
                            f[j] = mul2(f[j], pair(g.x, g.y));
                            f[j + 1] = mul2(f[j + 1], pair(g.z, g.w));
                        }
                    }
                    uint32_t z[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        float lo, hi;
                        split(f[j], lo, hi);
                        z[j] = pack_bf16(lo, hi);
                    }
                    __syncwarp();
                    tc::st16(sa + 32 * c, z);           // over columns of S that this warp has read
                    if (LABELS) {                      // what the rounding took
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            float lo, hi;
                            split(f[j], lo, hi);
                            lo -= __uint_as_float(z[j] << 16);
                            hi -= __uint_as_float(z[j] & 0xFFFF0000u);
                            // nothing to add where an entry left the range
                            z[j] = pack_bf16(fabsf(lo) <= 3e38f ? lo : 0.f, fabsf(hi) <= 3e38f ? hi : 0.f);
                        }
                        __syncwarp();
                        tc::st16(sa + 32 * c + 16, z);
                    }
                };
                if constexpr (M != TC_FORWARD) {
                    if (marked) {
                        const uint32_t labels = LabelUnits::columns<M>(P.a, xi, y0 + i, info + st * XT_INFO) >> half * 16;
#pragma unroll 1
                        for (int c = 0; c < 2; ++c) {
                            if (labels >> 8 * c & 0x11) weigh(std::true_type{}, c);
                            else weigh(std::false_type{}, c);
                        }
                    } else {
                        weigh(std::false_type{}, 0);
                        weigh(std::false_type{}, 1);
                    }
                }
#pragma unroll
                for (int c = 0; c < (M == TC_FORWARD ? 2 : 0); ++c) {
                    uint32_t q[32];
                    tc::ld32(sa + 32 * c, q);
                    tc::wait_ld(q);
                    const int col = ybase + c * 32;
                    if (c == 1) {                      // S is in registers: the buffer may be overwritten
                        tc::fence_before();
                        tc::mbar_arrive(p_full(b));
                    }
                    float cc = c2;
                    if (col + 32 > P.ny) {             // behind the table's last row
                        cc = 1.f;
#pragma unroll
                        for (int j = 0; j < 32; ++j) q[j] = col + j < P.ny ? __float_as_uint(__uint_as_float(q[j]) * c2) : 0xFF800000u;
                    }
                    if (__any_sync(FULL, label >= col && label < col + 32)) {
                        float z = 0.f;
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (col + j == label) z = __uint_as_float(q[j]) * cc;
                        if (label >= col && label < col + 32) P.picked[x] = z;
                        __syncwarp();
                    }
                    float e[4];                        // the largest product with cc comes from the largest or the smallest S
#pragma unroll
                    for (int j = 0; j < 4; ++j) e[j] = __uint_as_float(q[j]);
                    if (cc >= 0.f) {
#pragma unroll
                        for (int j = 4; j < 32; j += 8)
#pragma unroll
                            for (int k = 0; k < 4; ++k) e[k] = j < 28 ? max3(e[k], __uint_as_float(q[j + k]), __uint_as_float(q[(j + k + 4) & 31])) : fmaxf(e[k], __uint_as_float(q[j + k]));
                        e[0] = fmaxf(max3(e[0], e[1], e[2]), e[3]);
                    } else {
#pragma unroll
                        for (int j = 4; j < 32; j += 8)
#pragma unroll
                            for (int k = 0; k < 4; ++k) e[k] = j < 28 ? min3(e[k], __uint_as_float(q[j + k]), __uint_as_float(q[(j + k + 4) & 31])) : fminf(e[k], __uint_as_float(q[j + k]));
                        e[0] = fminf(min3(e[0], e[1], e[2]), e[3]);
                    }
                    const float top = fmaxf(m, e[0] * cc), ref = top == -INFINITY ? 0.f : top;
                    const f32x2 c22 = pair(cc, cc), r2 = pair(-ref, -ref);
                    f32x2 sum[2] = {0, 0};
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        sum[j & 1] = add2(sum[j & 1], exp2_pair<true>(fma2(pair(__uint_as_float(q[2 * j]), __uint_as_float(q[2 * j + 1])), c22, r2), j));
                    float lo, hi;
                    split(add2(sum[0], sum[1]), lo, hi);
                    l = l * xt_exp2(m - ref) + (lo + hi);
                    m = top;
                }
                if (M != TC_FORWARD) {
                    tc::wait_st();
                    tc::fence_before();
                    tc::mbar_arrive(p_full(b));
                    if (pending) epilogue();
                }
            }
            if (!ok) break;
            if (M == TC_FORWARD) {
                P.stats[((run + xi) * XENT_TC_STATS + wg) * XT + row] = make_float2(m, l);
                continue;
            }
            if (pending) epilogue();
            pending = true;
            whole = y0 == 0 && n == P.runs.tiles_y;
            e_run = run;
            e_xi = xi;
        }
        if (M != TC_FORWARD && ok && pending) epilogue();
        if (!ok && lane == 0) atomicExch(&g_xent_gave_up, 1);
    }
    __syncwarp();
    tc::fence_before();
    __syncthreads();
    if (warp == 2) {
        tc::fence_after();
        tc::tmem_free(tmem, 512);
    }
}

// Columns c .. c + 7 of a row, zeros behind its end, read in units of U.
template <typename U> __device__ __forceinline__ uint4 eight_columns(const bf16* row, int c, int dim) {
    constexpr int PER = sizeof(U) / 2;
    union {
        U u[8 / PER];
        uint4 w;
    } v;
#pragma unroll
    for (int j = 0; j < 8 / PER; ++j) v.u[j] = c + j * PER < dim ? __ldcs(reinterpret_cast<const U*>(row + c) + j) : U{};
    return v.w;
}

// What the backward kernels need of the hidden rows, tile by tile (rows behind the last have no gradient): row_info, the marks of
// the table's tiles in which their labels lie, and a copy in which rows without a label are zeros.  Such a row's weights
// are zeros, but it may hold infinities or NaN, and the products take whole tiles.  The copy has a pitch that tile loads can address;
// it is read in units of U.  8,192 rows of 128: 4.7 us, 2.6 without the copy.
constexpr int XI_THREADS = 512;
template <typename U> __global__ void __launch_bounds__(XI_THREADS) k_xent_row_info(Xent a, float* __restrict__ info, uint32_t* __restrict__ marks, int words,
                                                                                    int pitch, bf16* __restrict__ copy) {
    __shared__ bool s_valid[XT];
    chain_wait();
    const int per_row = pitch / 8;
    for (int64_t t = blockIdx.x; t * XT < a.rows; t += gridDim.x) {
        for (int i = threadIdx.x; i < words; i += XI_THREADS) marks[t * words + i] = 0;
        __syncthreads();
        if (threadIdx.x < XT) {
            const int64_t n = t * XT + threadIdx.x;
            const int lab = n < a.rows ? a.labels[n] : -1;
            const bool valid = lab >= 0 && lab < a.vocab;
            float* p = info + t * 3 * XT + threadIdx.x;
            p[0] = valid ? a.lse[n] * -XT_LOG2E : 0.f;
            p[XT] = valid ? a.dloss[n] * a.scale : 0.f;
            reinterpret_cast<int*>(p)[2 * XT] = valid ? lab : -1;
            if (valid) atomicOr(marks + t * words + (lab >> 5) / XT, 1u << (lab / XT & 31));
            s_valid[threadIdx.x] = valid;
        }
        __syncthreads();
        const int left = a.rows - t * XT < XT ? (int)(a.rows - t * XT) : XT;
#pragma unroll 4
        for (int i = threadIdx.x; i < left * per_row; i += XI_THREADS) {
            const int r = i / per_row, c = (i - r * per_row) * 8;
            const bf16* from = (const bf16*)a.hidden + (t * XT + r) * a.hidden_ld;
            *reinterpret_cast<uint4*>(copy + (t * XT + r) * pitch + c) = s_valid[r] ? eight_columns<U>(from, c, a.dim) : make_uint4(0, 0, 0, 0);
        }
    }
}

// Rows repacked to a pitch that tile loads can address (a multiple of 16 bytes): 8 columns per thread, read in units of U.
template <typename U> __global__ void __launch_bounds__(256) k_xent_pack(const bf16* __restrict__ src, int64_t ld, int64_t rows, int dim, int pitch, bf16* __restrict__ dst) {
    chain_wait();
    const int per_row = pitch / 8, rows_per_block = 256 / per_row;
    const int r_in = threadIdx.x / per_row, c = (threadIdx.x - r_in * per_row) * 8;
    if (r_in >= rows_per_block) return;
    for (int64_t r = (int64_t)blockIdx.x * rows_per_block + r_in; r < rows; r += (int64_t)gridDim.x * rows_per_block) {
        *reinterpret_cast<uint4*>(dst + r * pitch + c) = eight_columns<U>(src + r * ld, c, dim);
    }
}

// ---------------------------------------------------------------- launches
typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static EncodeTiled encode_tiled() {
    static std::atomic<EncodeTiled> found{nullptr};
    EncodeTiled f = found.load(std::memory_order_relaxed);
    if (!f) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &r) != cudaSuccess || r != cudaDriverEntryPointSuccess) return nullptr;
        f = (EncodeTiled)p;
        found.store(f, std::memory_order_relaxed);
    }
    return f;
}

// Rows of `dim` bf16, tiles of 64 columns by 128 rows; what lies outside reads as zero.
static cudaError_t row_map(CUtensorMap* map, const void* base, int64_t rows, int dim, int64_t ld) {
    const EncodeTiled f = encode_tiled();
    if (!f) return cudaErrorSymbolNotFound;
    const cuuint64_t dims[2] = {(cuuint64_t)dim, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * 2};
    const cuuint32_t box[2] = {64, XT}, step[2] = {1, 1};
    return f(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
               ? cudaSuccess
               : cudaErrorInvalidValue;
}

static bool tile_rows_ok(const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && (ld * 2) % 16 == 0; }
static int packed_pitch(int dim) { return (dim + 7) / 8 * 8; }

bool xent_tc_takes(const Xent& a) {
    if (a.dtype != GS_BF16 || a.dim > XENT_TC_MAX_DIM) return false;
    return a.dim % 8 != 0 || (tile_rows_ok(a.hidden, a.hidden_ld) && tile_rows_ok(a.table, a.table_ld));
}

// Words of marks per tile of hidden rows: a bit per tile of the table.
static int mark_words(const Xent& a) { return (int)((a.vocab + 32 * XT - 1) / (32 * XT)); }

struct TcLayout {
    size_t hidden, table, rest, total;
};

static TcLayout tc_layout(const Xent& a) {
    TcLayout l{};
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t o = off; off = align_up(off + bytes, 256); return o; };
    l.hidden = take((size_t)a.rows * packed_pitch(a.dim) * 2);       // for the backward pass, or as the table
    if (a.dim % 8) l.table = take((size_t)a.vocab * packed_pitch(a.dim) * 2);       // what tile loads may not be able to address is copied
    l.rest = off;
    const int64_t parts = sm_count(), tx = (a.rows + XT - 1) / XT;
    const size_t fwd = align_up((size_t)(parts + tx) * XENT_TC_STATS * XT * 8, 256) + align_up((size_t)a.rows * 4, 256);
    const size_t bwd = align_up((size_t)2 * parts * XT * ((a.dim + 15) / 16 * 16) * 4, 256) + (size_t)tx * (XT_INFO + (size_t)mark_words(a) * 4);
    take(fwd > bwd ? fwd : bwd);
    l.total = off;
    return l;
}

size_t xent_tc_workspace(const Xent& a) { return tc_layout(a).total; }

cudaError_t xent_gave_up(cudaStream_t s, int* h_flag) {
    cudaError_t e = cudaMemcpyFromSymbolAsync(h_flag, g_xent_gave_up, sizeof(int), 0, cudaMemcpyDeviceToHost, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    return e;
}

struct Operands {
    void* hidden;
    void* table;
    int64_t hidden_ld, table_ld;
    char* rest;
    CUtensorMap hidden_map, table_map;
};

// Units in which rows can be read: the largest power of two that divides address, pitch and length, at most `most` bytes.
static int read_unit(const void* p, int64_t ld, int dim, int most) {
    const uint64_t all = (uint64_t)(uintptr_t)p | (uint64_t)ld * 2 | (uint64_t)dim * 2;
    while (most > 2 && all % most) most /= 2;
    return most;
}

// BACKWARD: the hidden rows are the copy that k_xent_row_info makes.
template <bool BACKWARD> static cudaError_t prepare_operands(const Xent& a, void* workspace, Operands* o, cudaStream_t s) {
    const TcLayout l = tc_layout(a);
    char* ws = (char*)workspace;
    o->hidden = const_cast<void*>(a.hidden);
    o->table = const_cast<void*>(a.table);
    o->hidden_ld = a.hidden_ld;
    o->table_ld = a.table_ld;
    o->rest = ws + l.rest;
    cudaError_t e = cudaSuccess;
    const int pitch = packed_pitch(a.dim);
    auto pack = [&](const void* src, int64_t ld, int64_t rows, char* dst) {
        const int rows_per_block = 256 / (pitch / 8);
        int64_t blocks = (rows + rows_per_block - 1) / rows_per_block;
        if (blocks > sm_count() * 32) blocks = sm_count() * 32;
        const int unit = read_unit(src, ld, a.dim, 8);
        if (e != cudaSuccess) return;
        if (unit == 8) e = launch_train(k_xent_pack<uint2>, blocks, 256, 0, s, (const bf16*)src, ld, rows, a.dim, pitch, (bf16*)dst);
        else if (unit == 4) e = launch_train(k_xent_pack<uint32_t>, blocks, 256, 0, s, (const bf16*)src, ld, rows, a.dim, pitch, (bf16*)dst);
        else e = launch_train(k_xent_pack<uint16_t>, blocks, 256, 0, s, (const bf16*)src, ld, rows, a.dim, pitch, (bf16*)dst);
    };
    if (BACKWARD || !tile_rows_ok(a.hidden, a.hidden_ld)) {
        if (!BACKWARD) pack(a.hidden, a.hidden_ld, a.rows, ws + l.hidden);
        o->hidden = ws + l.hidden;
        o->hidden_ld = pitch;
    }
    if (!tile_rows_ok(a.table, a.table_ld)) {
        pack(a.table, a.table_ld, a.vocab, ws + l.table);
        o->table = ws + l.table;
        o->table_ld = pitch;
    }
    if (e == cudaSuccess) e = row_map(&o->hidden_map, o->hidden, a.rows, a.dim, o->hidden_ld);
    if (e == cudaSuccess) e = row_map(&o->table_map, o->table, a.vocab, a.dim, o->table_ld);
    return e;
}

template <int M> static cudaError_t run_tc(const Xent& a, const Operands& o, XentTc& P, cudaStream_t s) {
    constexpr bool ON_X = M != TC_DTABLE;
    P.a = a;
    P.nx = ON_X ? a.rows : (int)a.vocab;
    P.ny = ON_X ? (int)a.vocab : a.rows;
    P.runs = make_runs(P.nx, XT, P.ny, XT, sm_count());
    const int chunks = (a.dim + 63) / 64, tile = chunks * XT_CHUNK;
    P.xbufs = chunks == 1 || (chunks == 2 && M == TC_FORWARD) ? 2 : 1;
    P.on = (a.dim + 15) / 16 * 16;
    // 512 columns of tensor memory: three S and one O of up to 128 columns (two of up to 64), or two S and one O of up to
    // 256.  Two S and two O of 128 columns, whose next row's products need not wait for the store of this one's: dw of
    // 169,343 x 128 with 128 hidden rows 56.4 | 57.2 us, but 512 rows 67.0 | 65.9, 1,024 rows 94.5 | 85.9, 8,192 rows 582 | 503.
    P.on_pitch = chunks == 1 ? 64 : 128;
    P.sbufs = chunks <= 2 ? 3 : 2;
    P.obufs = chunks == 1 ? 2 : 1;
    // shared memory: X, the ring of Y, row info, and rows on their way out where X and three or more tiles of Y leave room
    int staging = 0;
    P.out = OUT_DIRECT;                    // each gradient by its own address and pitch
    P.out_pitch = 0;
    if (M != TC_FORWARD && chunks <= 2 && a.grad_dtype == GS_BF16) {
        const void* grad = M == TC_DHIDDEN ? a.dhidden : a.dtable;
        const int64_t ld = M == TC_DHIDDEN ? a.dhidden_ld : a.dtable_ld;
        if (tile_rows_ok(grad, ld) && a.dim % 8 == 0) P.out = OUT_ROWS;
        else if (((uintptr_t)grad & 15) == 0 && ld == a.dim) P.out = OUT_TILE;
        P.out_pitch = a.dim * 2 + (P.out == OUT_ROWS ? 16 : 0);      // 16 bytes apart: neighbouring rows in different banks
        if (P.out != OUT_DIRECT) staging = XT * P.out_pitch;
    }
    P.stages = ((M == TC_FORWARD ? 192 : 216) * 1024 - staging) / (tile + (M == TC_DTABLE ? XT_INFO : 0)) - P.xbufs;
    if (P.stages > XT_MAX_STAGES) P.stages = XT_MAX_STAGES;
    // at least 120 KB, so that an SM holds one block: a block takes all of the tensor memory
    int smem = (P.xbufs + P.stages) * tile + 1024 + (M == TC_DTABLE ? P.stages * XT_INFO : 0) + staging;
    if (smem < (120 << 10)) smem = 120 << 10;
    auto kernel = chunks == 1 ? k_xent_tc<M, 1> : (chunks == 2 ? k_xent_tc<M, 2> : (chunks == 3 ? k_xent_tc<M, 3> : k_xent_tc<M, 4>));
    static std::atomic<uint64_t> allowed[4];
    const cudaError_t e = allow_smem(kernel, 226 << 10, allowed[chunks - 1]);
    if (e != cudaSuccess) return e;
    return launch_train(kernel, P.runs.parts, XT_THREADS, smem, s, P, ON_X ? o.hidden_map : o.table_map, ON_X ? o.table_map : o.hidden_map);
}

cudaError_t launch_xent_tc_forward(const Xent& a, void* workspace, Runs* runs, const float2** stats, const float** picked, cudaStream_t s) {
    Operands o;
    cudaError_t e = prepare_operands<false>(a, workspace, &o, s);
    if (e != cudaSuccess) return e;
    XentTc P{};
    const int64_t tx = (a.rows + XT - 1) / XT;
    P.stats = (float2*)o.rest;
    P.picked = (float*)(o.rest + align_up((size_t)(sm_count() + tx) * XENT_TC_STATS * XT * 8, 256));
    e = run_tc<TC_FORWARD>(a, o, P, s);
    *runs = P.runs;
    *stats = P.stats;
    *picked = P.picked;
    return e;
}

cudaError_t launch_xent_tc_backward(const Xent& a, void* workspace, cudaStream_t s) {
    Operands o;
    cudaError_t e = prepare_operands<true>(a, workspace, &o, s);
    if (e != cudaSuccess) return e;
    XentTc P{};
    P.partial = (float*)o.rest;
    float* row_info = (float*)(o.rest + align_up((size_t)2 * sm_count() * XT * ((a.dim + 15) / 16 * 16) * 4, 256));
    P.row_info = row_info;
    P.mark_words = mark_words(a);
    uint32_t* marks = (uint32_t*)(row_info + (int64_t)((a.rows + XT - 1) / XT) * (XT_INFO / 4));
    P.marks = marks;
    auto info = [&](auto kernel) {
        return launch_train(kernel, (a.rows + XT - 1) / XT, XI_THREADS, 0, s, a, row_info, marks, P.mark_words, (int)o.hidden_ld, (bf16*)o.hidden);
    };
    switch (read_unit(a.hidden, a.hidden_ld, a.dim, 16)) {
        case 16: e = info(k_xent_row_info<uint4>); break;
        case 8: e = info(k_xent_row_info<uint2>); break;
        case 4: e = info(k_xent_row_info<uint32_t>); break;
        default: e = info(k_xent_row_info<uint16_t>);
    }
    if (e == cudaSuccess) e = run_tc<TC_DHIDDEN>(a, o, P, s);
    if (e != cudaSuccess) return e;
    e = launch_xent_join(a, true, P.runs, XT, P.on, P.partial, s);
    if (e != cudaSuccess) return e;
    e = run_tc<TC_DTABLE>(a, o, P, s);
    if (e != cudaSuccess) return e;
    return launch_xent_join(a, false, P.runs, XT, P.on, P.partial, s);
}

}  // namespace gs
