// Softmax cross entropy of hidden rows against every row of a table, without keeping the logits.
//
//   z_nv = scale h_n . w_v,  lse_n = log sum_v exp z_nv,  loss_n = lse_n - z_n,label(n)
//   dz_nv = g_n scale (exp(z_nv - lse_n) - [v = label(n)]),  dh_n = sum_v dz_nv w_v,  dw_v = sum_n dz_nv h_n
// (g_n the upstream gradient; a label outside the table: loss 0 and no gradient.)  The logits exist one tile at a
// time.  The backward pass recomputes them from lse, once for dh (a tile of hidden rows stays, the table streams by)
// and once for dw (a tile of table rows stays, the hidden rows stream by): 8 N V d operations, no atomics.
//
// bf16 operands of up to 256 columns go to the tensor cores (gs_xent_tc.cu).  k_xent_simt takes the rest, f32 above
// all, with products in 32 bits on the CUDA cores: exact enough for f32 operands, which the tensor cores' types are
// not.  It serves both directions: x are the rows that stay, y the rows that stream.
#include "gs_device.cuh"
#include "gs_train.cuh"
#include "gs_train.h"
#include "gs_xent.h"

namespace gs {

constexpr float XE_LOG2E = 1.4426950408889634f, XE_LN2 = 0.6931471805599453f;
constexpr int XS_TILE = 64;          // rows of x and of y per tile
constexpr int XS_THREADS = 256;
constexpr int XS_K = 32;             // depth of one staged slice of the products
constexpr int XS_COLS = 128;         // gradient columns per block

__device__ __forceinline__ float xe_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

enum XentMode { XE_FORWARD, XE_DHIDDEN, XE_DTABLE };

struct XentSimt {
    Xent a;
    Runs runs;
    float2* stats;        // forward: [parts + tiles_x][XS_TILE] running maximum (base 2) and sum
    float* picked;        // forward: [rows] the label's logit, base 2
    float* partial;       // backward: [2 parts][XS_TILE][dim]
};

template <typename T, XentMode M>
__global__ void __launch_bounds__(XS_THREADS) k_xent_simt(const __grid_constant__ XentSimt P) {
    __shared__ float xs[XS_K][XS_TILE + 4], ys[XS_K][XS_TILE + 4];
    __shared__ float zs[XS_TILE][XS_TILE + 1];
    __shared__ float s_lse[XS_TILE], s_g[XS_TILE];
    __shared__ int s_label[XS_TILE];
    constexpr bool ON_X = M != XE_DTABLE;          // the hidden rows are x
    const Xent& a = P.a;
    const T* X = (const T*)(ON_X ? a.hidden : a.table);
    const T* Y = (const T*)(ON_X ? a.table : a.hidden);
    const int64_t xld = ON_X ? a.hidden_ld : a.table_ld, yld = ON_X ? a.table_ld : a.hidden_ld;
    const int nx = ON_X ? a.rows : (int)a.vocab, ny = ON_X ? (int)a.vocab : a.rows, d = a.dim;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int col0 = blockIdx.y * XS_COLS;
    const float c2 = a.scale * XE_LOG2E;
    for (int64_t run = blockIdx.x; run < P.runs.parts; run += gridDim.x) {
        int64_t t = P.runs.start(run);
        const int64_t end = P.runs.start(run + 1);
        while (t < end) {
            const int64_t xi = t / P.runs.tiles_y;
            const int64_t last = (xi + 1) * P.runs.tiles_y < end ? (xi + 1) * P.runs.tiles_y : end;
            const int x0 = (int)(xi * XS_TILE);
            float m[4], l[4], acc[4][8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                m[i] = -INFINITY;
                l[i] = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) acc[i][j] = 0.f;
            }
            const bool whole = t == xi * P.runs.tiles_y && last == (xi + 1) * P.runs.tiles_y;
            for (; t < last; ++t) {
                const int y0 = (int)((t - xi * P.runs.tiles_y) * XS_TILE);
                __syncthreads();
                if (threadIdx.x < XS_TILE) {       // what belongs to the tile's hidden rows
                    const int n = (ON_X ? x0 : y0) + threadIdx.x;
                    const int lab = n < a.rows ? __ldg(a.labels + n) : -1;
                    const bool valid = lab >= 0 && lab < a.vocab;
                    s_label[threadIdx.x] = valid ? lab : -1;
                    if (M != XE_FORWARD) {
                        s_lse[threadIdx.x] = n < a.rows ? __ldg(a.lse + n) * XE_LOG2E : 0.f;
                        s_g[threadIdx.x] = valid ? __ldg(a.dloss + n) * a.scale : 0.f;
                    }
                }
                float s[4][4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
                for (int k0 = 0; k0 < d; k0 += XS_K) {
                    __syncthreads();
                    for (int i = threadIdx.x; i < XS_TILE * XS_K; i += XS_THREADS) {
                        const int r = i / XS_K, k = i % XS_K;
                        const bool on = k0 + k < d;
                        xs[k][r] = on && x0 + r < nx ? to_f32(X[(int64_t)(x0 + r) * xld + k0 + k]) : 0.f;
                        ys[k][r] = on && y0 + r < ny ? to_f32(Y[(int64_t)(y0 + r) * yld + k0 + k]) : 0.f;
                    }
                    __syncthreads();
#pragma unroll 8
                    for (int k = 0; k < XS_K; ++k) {
                        float xv[4], yv[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            xv[i] = xs[k][ty * 4 + i];
                            yv[i] = ys[k][tx + 16 * i];
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int j = 0; j < 4; ++j) s[i][j] = fmaf(xv[i], yv[j], s[i][j]);
                    }
                }
                if (M == XE_FORWARD) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int lab = s_label[ty * 4 + i];
                        float top = m[i];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int v = y0 + tx + 16 * j;
                            s[i][j] = v < ny ? s[i][j] * c2 : -INFINITY;
                            if (v == lab) P.picked[x0 + ty * 4 + i] = s[i][j];
                            top = fmaxf(top, s[i][j]);
                        }
#pragma unroll
                        for (int o = 8; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(FULL, top, o));
                        const float ref = top == -INFINITY ? 0.f : top;
                        float sum = 0.f;
#pragma unroll
                        for (int j = 0; j < 4; ++j) sum += xe_exp2(s[i][j] - ref);
                        l[i] = l[i] * xe_exp2(m[i] - ref) + sum;       // this thread's columns; joined at the end
                        m[i] = top;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const int xr = ty * 4 + i, yr = tx + 16 * j, n = ON_X ? xr : yr, v = ON_X ? y0 + yr : x0 + xr;
                            const bool on = x0 + xr < nx && y0 + yr < ny;
                            const float p = xe_exp2(fmaf(s[i][j], c2, -s_lse[n])) - (s_label[n] == v ? 1.f : 0.f);
                            zs[xr][yr] = on && s_g[n] != 0.f ? p * s_g[n] : 0.f;
                        }
                    for (int k0 = 0; k0 < XS_TILE; k0 += 16) {        // 16 rows of y, 128 columns at a time
                        __syncthreads();
                        float* yc = &xs[0][0];                         // [16][132], over xs
                        for (int i = threadIdx.x; i < 16 * XS_COLS; i += XS_THREADS) {
                            const int r = i / XS_COLS, c = i % XS_COLS;
                            // a hidden row without a label may hold anything: zeros
                            const bool on = y0 + k0 + r < ny && col0 + c < d && (ON_X || s_label[k0 + r] >= 0);
                            yc[r * (XS_COLS + 4) + c] = on ? to_f32(Y[(int64_t)(y0 + k0 + r) * yld + col0 + c]) : 0.f;
                        }
                        __syncthreads();
#pragma unroll
                        for (int k = 0; k < 16; ++k) {
                            float yv[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) yv[j] = yc[k * (XS_COLS + 4) + tx + 16 * j];
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const float z = zs[ty * 4 + i][k0 + k];
#pragma unroll
                                for (int j = 0; j < 8; ++j) acc[i][j] = fmaf(z, yv[j], acc[i][j]);
                            }
                        }
                    }
                }
            }
            if (M == XE_FORWARD) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float sum = l[i];
#pragma unroll
                    for (int o = 8; o; o >>= 1) sum += __shfl_xor_sync(FULL, sum, o);
                    if (tx == 0) P.stats[(run + xi) * XS_TILE + ty * 4 + i] = make_float2(m[i], sum);
                }
            } else {
                float* part = P.partial + P.runs.slot(run, xi) * XS_TILE * d;
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int r = ty * 4 + i, c = col0 + tx + 16 * j;
                        if (c >= d || x0 + r >= nx) continue;
                        if (!whole) part[(int64_t)r * d + c] = acc[i][j];
                        else if (M == XE_DHIDDEN) a.store_dhidden(x0 + r, c, acc[i][j]);
                        else a.store_dtable(x0 + r, c, acc[i][j]);
                    }
            }
        }
    }
}

// lse and loss of every row from the runs' statistics: a warp per row, its lanes over the entries.
__global__ void __launch_bounds__(256) k_xent_finish(Xent a, Runs runs, int tile, int per, const float2* __restrict__ stats, const float* __restrict__ picked) {
    chain_wait();
    const int lane = threadIdx.x & 31;
    for (int64_t n = (int64_t)blockIdx.x * 8 + threadIdx.x / 32; n < a.rows; n += (int64_t)gridDim.x * 8) {
        const int64_t i = n / tile;
        const int64_t c0 = runs.run_of(i * runs.tiles_y), c1 = runs.run_of((i + 1) * runs.tiles_y - 1);
        float m = -INFINITY, l = 0.f;
        for (int64_t c = (c0 + i) * per + lane; c < (c1 + i + 1) * per; c += 32) {      // `per` entries of a run
            const float2 s = __ldcg(stats + c * tile + n % tile);
            const float top = fmaxf(m, s.x), ref = top == -INFINITY ? 0.f : top;
            l = l * xe_exp2(m - ref) + s.y * xe_exp2(s.x - ref);
            m = top;
        }
        for (int o = 16; o; o >>= 1) {
            const float mo = __shfl_xor_sync(FULL, m, o), lo = __shfl_xor_sync(FULL, l, o);
            const float top = fmaxf(m, mo), ref = top == -INFINITY ? 0.f : top;
            l = l * xe_exp2(m - ref) + lo * xe_exp2(mo - ref);
            m = top;
        }
        if (lane == 0) {
            const int lab = a.labels[n];
            const bool valid = lab >= 0 && lab < a.vocab;
            const float log2l = log2f(l);
            a.lse_out[n] = (m + log2l) * XE_LN2;
            a.loss[n] = valid ? ((m - __ldcg(picked + n)) + log2l) * XE_LN2 : 0.f;
        }
    }
}

// Rows of tiles that several runs share: their partial sums in order.  The run before the first that starts inside, c,
// left slot 2c - 1, the runs c, c + 1, .. up to the row's end 2c, 2c + 2, ..
template <XentMode M> __global__ void __launch_bounds__(256) k_xent_join(Xent a, const __grid_constant__ JoinList list, int tile, int pitch, const float* __restrict__ partial) {
    chain_wait();
    const JoinList::Entry j = list.e[blockIdx.x];
    const int64_t nx = M == XE_DHIDDEN ? a.rows : a.vocab, x0 = (int64_t)j.row * tile, step = (int64_t)tile * pitch;
    const int rows = nx - x0 < tile ? (int)(nx - x0) : tile;
    for (int e = blockIdx.y * 256 + threadIdx.x; e < rows * pitch; e += gridDim.y * 256) {
        const int r = e / pitch, col = e - r * pitch;
        if (col >= a.dim) continue;
        const float* p = partial + (2 * (int64_t)j.first - 1) * step + e;
        float acc = __ldcg(p);
        p += step;
#pragma unroll 8
        for (int k = 0; k < j.runs; ++k, p += 2 * step) acc += __ldcg(p);
        if (M == XE_DHIDDEN) a.store_dhidden(x0 + r, col, acc);
        else a.store_dtable(x0 + r, col, acc);
    }
}

// ---------------------------------------------------------------- launches
static int64_t simt_parts() { return sm_count() * 2 < MAX_JOINS ? sm_count() * 2 : MAX_JOINS; }
static Runs simt_runs(int64_t x, int64_t y) { return make_runs(x, XS_TILE, y, XS_TILE, simt_parts()); }

static size_t simt_workspace(const Xent& a) {
    const Runs f = simt_runs(a.rows, a.vocab), t = simt_runs(a.vocab, a.rows);
    const size_t fwd = align_up((size_t)(f.parts + f.tiles_x) * XS_TILE * 8, 256) + align_up((size_t)a.rows * 4, 256);
    const size_t bwd = (size_t)2 * (f.parts > t.parts ? f.parts : t.parts) * XS_TILE * a.dim * 4;
    return fwd > bwd ? fwd : bwd;
}

size_t xent_workspace(const Xent& a) {
    const size_t simt = simt_workspace(a), tc = a.dtype == GS_BF16 && a.dim <= XENT_TC_MAX_DIM ? xent_tc_workspace(a) : 0;
    return align_up(simt > tc ? simt : tc, 256);
}

template <typename T, XentMode M> static void run_simt(XentSimt& P, cudaStream_t s) {
    const int cols = M == XE_FORWARD ? 1 : (P.a.dim + XS_COLS - 1) / XS_COLS;
    k_xent_simt<T, M><<<dim3((unsigned)limit_grid(P.runs.parts), (unsigned)cols), XS_THREADS, 0, s>>>(P);
    count_launches(1);
}

template <XentMode M> static void run_join(const Xent& a, const Runs& runs, int tile, int pitch, const float* partial, cudaStream_t s) {
    JoinList list;
    const int n = list_joins(runs, &list);
    if (!n) return;
    // few shared rows: spread each over many blocks
    int64_t by = (tile * pitch + 255) / 256, few = sm_count() * 8 / n + 1;
    if (by > few) by = few;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)n, (unsigned)by);
    cfg.blockDim = dim3(256);
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    cudaLaunchKernelEx(&cfg, k_xent_join<M>, a, list, tile, pitch, partial);
    count_launches(1);
}

cudaError_t launch_xent_join(const Xent& a, bool hidden, const Runs& runs, int tile, int pitch, const float* partial, cudaStream_t s) {
    if (hidden) run_join<XE_DHIDDEN>(a, runs, tile, pitch, partial, s);
    else run_join<XE_DTABLE>(a, runs, tile, pitch, partial, s);
    return cudaGetLastError();
}

cudaError_t launch_xent_forward(const Xent& a, void* workspace, cudaStream_t s) {
    const int64_t finish = limit_grid((a.rows + 7) / 8 < sm_count() * 8 ? (a.rows + 7) / 8 : sm_count() * 8);
    if (xent_tc_takes(a)) {
        Runs runs;
        const float2* stats;
        const float* picked;
        const cudaError_t e = launch_xent_tc_forward(a, workspace, &runs, &stats, &picked, s);
        if (e != cudaSuccess) return e;
        return launch_train(k_xent_finish, finish, 256, 0, s, a, runs, XENT_TC_TILE, XENT_TC_STATS, stats, picked);
    }
    XentSimt P{};
    P.a = a;
    P.runs = simt_runs(a.rows, a.vocab);
    P.stats = (float2*)workspace;
    P.picked = (float*)((char*)workspace + align_up((size_t)(P.runs.parts + P.runs.tiles_x) * XS_TILE * 8, 256));
    if (a.dtype == GS_BF16) run_simt<bf16, XE_FORWARD>(P, s);
    else run_simt<float, XE_FORWARD>(P, s);
    k_xent_finish<<<(int)finish, 256, 0, s>>>(a, P.runs, XS_TILE, 1, P.stats, P.picked);
    count_launches(1);
    return cudaGetLastError();
}

cudaError_t launch_xent_backward(const Xent& a, void* workspace, cudaStream_t s) {
    if (xent_tc_takes(a)) return launch_xent_tc_backward(a, workspace, s);
    XentSimt P{};
    P.a = a;
    P.partial = (float*)workspace;
    P.runs = simt_runs(a.rows, a.vocab);
    if (a.dtype == GS_BF16) run_simt<bf16, XE_DHIDDEN>(P, s);
    else run_simt<float, XE_DHIDDEN>(P, s);
    run_join<XE_DHIDDEN>(a, P.runs, XS_TILE, a.dim, P.partial, s);
    P.runs = simt_runs(a.vocab, a.rows);
    if (a.dtype == GS_BF16) run_simt<bf16, XE_DTABLE>(P, s);
    else run_simt<float, XE_DTABLE>(P, s);
    run_join<XE_DTABLE>(a, P.runs, XS_TILE, a.dim, P.partial, s);
    return cudaGetLastError();
}

}  // namespace gs
