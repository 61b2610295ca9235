// Softmax attention of a block's destinations over their listed sources, forward and backward.
//
// For destination i, query head h, key/value head g(h) and the edges j of row i:
//   s = scale q_ih . k_jg,  lse_ih = log sum_j exp s,  o_ih = sum_j p v_jg,  p = exp(s - lse_ih);
//   delta = do . o,  ds = p (do . v - delta) scale,  dq_i = sum_j ds k_j,  dk_j = sum_i ds q_i,  dv_j = sum_i p do_i.
// The forward keeps a running maximum and sum.  The backward recomputes p from lse in the pass that sums dq; the ring kernels
// leave p and ds there, 8 bytes per edge and head, for the pass in source order, which then needs neither k nor v
// (4.36 M edges of 4 heads of 32: 605 us, 848 with the dot products taken again).
//
// Every edge gathers whole rows, so the kernels are bound by the gathered bytes: a group of tl lanes holds one
// (row, head) with one wide load per lane and operand, U edges are in flight per group, and groups of one row's heads are
// neighbours in a warp, so that an edge's row is read in one piece.  dk and dv are summed in source order over the
// reversed block (a stable sort), each row by one group: no atomics, the result does not depend on the schedule.
// A row longer than AT_CHUNK edges (hubs) is cut into chunks; the chunks' results are joined in order.
// Operands in pieces of 16 or 8 bytes go to the ring kernels (gs_attend_ring.cuh); the kernels of this file take one element
// at a time, whatever the alignment and the head dimension, and let `slots` groups share a row when rows are too few.
// 4.36 M edges of 4 heads of 32, bf16 (512 bytes gathered per edge): forward 347 us (6.4 TB/s gathered), dq 458 us, dk and dv
// 605 us, the reversed block 218 us.
#include <initializer_list>
#include <type_traits>

#include "gs_device.cuh"
#include "gs_train.cuh"
#include "gs_train.h"

namespace gs {

constexpr int AT_THREADS = 256;
constexpr int AT_CHUNK = 64;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

__device__ __forceinline__ float fast_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// lse in base 2, as the backward passes take it.  A row whose scores are all -inf has lse = -inf like a masked one and no
// part in any gradient: +inf instead makes its probabilities exp(-inf) = 0.  An edge of probability zero has no part in a
// sum, not even one of 0 times the infinity that made its score; looking at every edge for it takes 4 to 16 %, so it is done
// where a sum came out not finite.
__device__ __forceinline__ float backward_lse(float lse) { return lse == -INFINITY ? INFINITY : lse * LOG2E; }

// delta = do . o is taken from `out`, which a caller of bf16 holds rounded: off by up to 2^-8 of sum |do||o|, which ds of a
// row of few edges, or of one probability near 1, does not bear (2.5 times the error of dq and dk at 179 rows of mostly one
// to three edges).  The dq pass therefore also sums r = sum p (dp - delta), which is 0 for the right delta, and sum p k, and corrects
// itself: dq = sum p (dp - delta) k - r sum p k.  The pass behind it adds r to delta (the "shift").  262,144 rows of 4 x 32:
// dq 410 -> 457 us, dk and dv 552 -> 606 (ds rewritten at a row's end instead: 609 and 552).  f32: nothing to correct.
template <typename T> constexpr bool rounded_out = sizeof(T) == 2;
// Floats of a chunk's part of dq, per head: the sum; and sum p k and r.
template <typename T> __device__ __forceinline__ int dq_part(int dim) { return rounded_out<T> ? 2 * dim + 1 : dim; }

enum AttendKind { AT_FORWARD, AT_DQ, AT_DKV };

struct Attend {
    BlockAttention a;
    const int32_t* starts;      // row offsets and columns: the block's, or the reversed block's
    const int32_t* cols;
    Count rows, columns;
    int edge_bound;
    int tl, slots, units_per_row;
    int tiles;                  // ring kernels: warp-sized tiles of units a warp takes at a time
    int split;                  // rows above AT_CHUNK edges go to the chunk list
    int dst_split;              // the same of the dq pass, for the pass behind it
    int chunk_mode;             // this launch works through the chunk list
    int32_t* words;             // [0] chunks, [1] long rows
    int32_t* look;              // set by the dq pass if there are edges of probability zero to look for (ring kernels)
    int2* items;                // chunk -> (row, chunk of the row)
    int4* longs;                // long row -> (row, first chunk, chunks, -)
    float* partial;
    float2* stat;               // [dst][q heads]: lse in base 2, delta (one-element kernels)
    float* shift;               // [dst][q heads]: what is missing in the dq pass's delta (ring kernels; else NULL)
    float2* pd;                 // [edges][q heads]: p and ds before the scale, from the dq pass (ring kernels)
    const int32_t* edges;       // source-order pass: the edge each column came from
};

__device__ __forceinline__ int length_of(const Count& c) {
    if (!c.d_n) return c.bound;
    const int n = __ldcg(c.d_n);
    return n < 0 ? 0 : (n > c.bound ? c.bound : n);
}

// What one group of lanes works on: a (row, unit of heads) and its range of edges.
struct Work {
    int row, unit, item, begin, end;
    bool live;
};

// Chunks of a long row join the list once, from the row's first unit.
__device__ __forceinline__ void list_long_row(const Attend& P, int row, int len) {
    const int nc = (len + AT_CHUNK - 1) / AT_CHUNK;
    const int first = atomicAdd(P.words, nc);
    P.longs[atomicAdd(P.words + 1, 1)] = make_int4(row, first, nc, 0);
    for (int c = 0; c < nc; ++c) P.items[first + c] = make_int2(row, c);
}

__device__ __forceinline__ Work find_work(const Attend& P, int64_t u, int64_t units, bool first_lane) {
    Work w;
    w.live = u < units;
    w.row = w.unit = w.item = w.begin = w.end = 0;
    if (!w.live) return w;
    const int r = (int)(u / P.units_per_row);
    w.unit = (int)(u - (int64_t)r * P.units_per_row);
    w.row = r;
    int first = 0;
    if (P.chunk_mode) {
        w.item = r;
        const int2 it = P.items[r];
        w.row = it.x;
        first = it.y * AT_CHUNK;
    }
    int b = __ldg(P.starts + w.row), e = __ldg(P.starts + w.row + 1);
    b = b < 0 ? 0 : b;
    e = e > P.edge_bound ? P.edge_bound : e;
    if (e < b) e = b;
    if (P.chunk_mode) {
        w.begin = b + first;
        w.end = w.begin + AT_CHUNK < e ? w.begin + AT_CHUNK : e;
    } else {
        w.begin = b;
        w.end = e;
        if (P.split && e - b > AT_CHUNK) {
            if (w.unit == 0 && first_lane) list_long_row(P, w.row, e - b);
            w.end = b;
            w.live = false;
        }
    }
    return w;
}

template <int N> __device__ __forceinline__ void group_sum(float (&x)[N], int tl) {
    for (int o = 1; o < tl; o <<= 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] += __shfl_xor_sync(FULL, x[i], o);
    }
}

// The lane's elements of one head row: NV pieces of VE, tl pieces apart.
template <typename T, int VE, int NV> struct Piece {
    Raw<T, VE> r[NV];
    __device__ __forceinline__ void load(const T* row, int t, int tl, int dim, bool on) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (t + j * tl) * VE;
            r[j] = on && c < dim ? load_raw<T, VE>(row + c) : zero_raw<T, VE>();
        }
    }
    __device__ __forceinline__ void get(float (&x)[NV * VE]) const {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float y[VE];
            unpack<T, VE>(r[j], y);
#pragma unroll
            for (int i = 0; i < VE; ++i) x[j * VE + i] = y[i];
        }
    }
};

template <typename T, int VE, int NV>
__device__ __forceinline__ void store_piece(T* row, int t, int tl, int dim, const float (&x)[NV * VE]) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (t + j * tl) * VE;
        if (c < dim) {
            float y[VE];
#pragma unroll
            for (int i = 0; i < VE; ++i) y[i] = x[j * VE + i];
            store_vec<T, VE>(row + c, y);
        }
    }
}

template <int VE, int NV> __device__ __forceinline__ void store_partial(float* row, int t, int tl, int dim, const float (&x)[NV * VE]) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (t + j * tl) * VE;
        if (c < dim) {
#pragma unroll
            for (int i = 0; i < VE; ++i) row[c + i] = x[j * VE + i];
        }
    }
}

template <typename T, int VE, int NV, int G, int U>
__global__ void __launch_bounds__(AT_THREADS) k_attend_forward(const __grid_constant__ Attend P) {
    constexpr int E = VE * NV;
    const int lane = threadIdx.x & 31, t = lane & (P.tl - 1), slot = (lane / P.tl) & (P.slots - 1);
    const int width = P.tl * P.slots, per_block = AT_THREADS / width;
    const int rows = P.chunk_mode ? __ldcg(P.words) : length_of(P.rows), cols = length_of(P.columns);
    const int64_t units = (int64_t)rows * P.units_per_row;
    const float c2 = P.a.scale * LOG2E;
    const int D = P.a.head_dim;
    const T* kbase = (const T*)P.a.k.data;
    const T* vbase = (const T*)P.a.v.data;
    for (int64_t base = (int64_t)blockIdx.x * per_block; base < units; base += (int64_t)gridDim.x * per_block) {
        const Work w = find_work(P, base + threadIdx.x / width, units, t == 0 && slot == 0);
        const int h0 = w.unit * G, g = h0 / (P.a.q_heads / P.a.kv_heads);
        float q[G][E], acc[G][E], m[G], l[G];
#pragma unroll
        for (int i = 0; i < G; ++i) {
            Piece<T, VE, NV> p;
            p.load((const T*)P.a.q.data + (int64_t)w.row * P.a.q.row_stride + (int64_t)(h0 + i) * P.a.q.head_stride, t, P.tl, D, w.live);
            p.get(q[i]);
            m[i] = -INFINITY;
            l[i] = 0.f;
#pragma unroll
            for (int c = 0; c < E; ++c) acc[i][c] = 0.f;
        }
        const int mine = (w.end - w.begin + P.slots * U - 1) / (P.slots * U);
        const int trips = __reduce_max_sync(FULL, mine);
        for (int it = 0; it < trips; ++it) {
            Piece<T, VE, NV> kp[U], vp[U];
            bool on[U];
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const int e = w.begin + (it * U + j) * P.slots + slot;
                const int col = e < w.end ? __ldg(P.cols + e) : -1;
                on[j] = (uint32_t)col < (uint32_t)cols;
                kp[j].load(kbase + (int64_t)col * P.a.k.row_stride + (int64_t)g * P.a.k.head_stride, t, P.tl, D, on[j]);
                vp[j].load(vbase + (int64_t)col * P.a.v.row_stride + (int64_t)g * P.a.v.head_stride, t, P.tl, D, on[j]);
            }
            float s[U * G];
#pragma unroll
            for (int j = 0; j < U; ++j) {
                float k[E];
                kp[j].get(k);
#pragma unroll
                for (int i = 0; i < G; ++i) {
                    float x = 0.f;
#pragma unroll
                    for (int c = 0; c < E; ++c) x = fmaf(q[i][c], k[c], x);
                    s[j * G + i] = x;
                }
            }
            group_sum<U * G>(s, P.tl);
            float p[U * G];
#pragma unroll
            for (int i = 0; i < G; ++i) {
                float top = m[i];
#pragma unroll
                for (int j = 0; j < U; ++j) {
                    s[j * G + i] = on[j] ? s[j * G + i] * c2 : -INFINITY;
                    top = fmaxf(top, s[j * G + i]);
                }
                const float ref = top == -INFINITY ? 0.f : top;     // nothing seen yet: all weights are zero
                const float corr = fast_exp2(m[i] - ref);
                m[i] = top;
                l[i] *= corr;
#pragma unroll
                for (int j = 0; j < U; ++j) {
                    p[j * G + i] = fast_exp2(s[j * G + i] - ref);
                    l[i] += p[j * G + i];
                }
#pragma unroll
                for (int c = 0; c < E; ++c) acc[i][c] *= corr;
            }
#pragma unroll
            for (int j = 0; j < U; ++j) {
                float v[E];
                vp[j].get(v);
#pragma unroll
                for (int i = 0; i < G; ++i)
#pragma unroll
                    for (int c = 0; c < E; ++c) acc[i][c] = fmaf(p[j * G + i], v[c], acc[i][c]);
            }
        }
        for (int o = P.tl; o < width; o <<= 1) {                      // join the slots of a row
#pragma unroll
            for (int i = 0; i < G; ++i) {
                const float mo = __shfl_xor_sync(FULL, m[i], o), lo = __shfl_xor_sync(FULL, l[i], o);
                const float top = fmaxf(m[i], mo), ref = top == -INFINITY ? 0.f : top;
                const float ca = fast_exp2(m[i] - ref), cb = fast_exp2(mo - ref);
                m[i] = top;
                l[i] = l[i] * ca + lo * cb;
#pragma unroll
                for (int c = 0; c < E; ++c) acc[i][c] = acc[i][c] * ca + __shfl_xor_sync(FULL, acc[i][c], o) * cb;
            }
        }
        if (!w.live || slot) continue;
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const int h = h0 + i;
            if (P.chunk_mode) {
                float* part = P.partial + ((int64_t)w.item * P.a.q_heads + h) * (D + 2);
                store_partial<VE, NV>(part, t, P.tl, D, acc[i]);
                if (t == 0) {
                    part[D] = m[i];
                    part[D + 1] = l[i];
                }
            } else {
                const bool none = l[i] == 0.f;                        // no edge left by the mask: zero row, log of an empty sum
                const float inv = none ? 0.f : 1.f / l[i];
#pragma unroll
                for (int c = 0; c < E; ++c) acc[i][c] = none ? 0.f : acc[i][c] * inv;
                store_piece<T, VE, NV>((T*)P.a.out.data + (int64_t)w.row * P.a.out.row_stride + (int64_t)h * P.a.out.head_stride, t, P.tl, D, acc[i]);
                if (t == 0) P.a.lse[(int64_t)w.row * P.a.q_heads + h] = none ? -INFINITY : m[i] * LN2 + logf(l[i]);
            }
        }
    }
}

// One block per (long row, query head); bound by the latency of a few dependent reads per warp (313 chunks of 24 columns and
// 8 heads beside 1.28 M edges: 28 us): the chunks' sums rescaled to the common maximum; each warp adds a contiguous share of
// the chunks, the shares are added in order.
template <typename T> __global__ void __launch_bounds__(AT_THREADS) k_attend_forward_join(const __grid_constant__ Attend P) {
    constexpr int W = AT_THREADS / 32;
    __shared__ float s_m[W], s_l[W], s_acc[W][256];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, D = P.a.head_dim;
    const int64_t units = (int64_t)__ldcg(P.words + 1) * P.a.q_heads, stride = (int64_t)P.a.q_heads * (D + 2);
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int4 row = P.longs[u / P.a.q_heads];
        const int h = (int)(u % P.a.q_heads);
        const float* part = P.partial + (int64_t)row.y * stride + (int64_t)h * (D + 2);
        const int per = (row.z + W - 1) / W, c0 = warp * per, c1 = c0 + per < row.z ? c0 + per : row.z;
        float m = -INFINITY, l = 0.f;
        for (int c = c0 + lane; c < c1; c += 32) m = fmaxf(m, part[c * stride + D]);
        for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(FULL, m, o));
        __syncthreads();                                       // the previous unit's sums are read
        if (lane == 0) s_m[warp] = m;
        __syncthreads();
        for (int w = 0; w < W; ++w) m = fmaxf(m, s_m[w]);
        const float ref = m == -INFINITY ? 0.f : m;
        for (int c = c0 + lane; c < c1; c += 32) l += part[c * stride + D + 1] * fast_exp2(part[c * stride + D] - ref);
        for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(FULL, l, o);
        if (lane == 0) s_l[warp] = l;
        for (int col = lane; col < D; col += 32) {
            float acc = 0.f;
#pragma unroll 4
            for (int c = c0; c < c1; ++c) acc = fmaf(part[c * stride + col], fast_exp2(part[c * stride + D] - ref), acc);
            s_acc[warp][col] = acc;
        }
        __syncthreads();
        l = 0.f;
        for (int w = 0; w < W; ++w) l += s_l[w];
        const bool none = l == 0.f;
        T* out = (T*)P.a.out.data + (int64_t)row.x * P.a.out.row_stride + (int64_t)h * P.a.out.head_stride;
        for (int col = threadIdx.x; col < D; col += AT_THREADS) {
            float acc = 0.f;
            for (int w = 0; w < W; ++w) acc += s_acc[w][col];
            out[col] = from_f32<T>(none ? 0.f : acc / l);
        }
        if (threadIdx.x == 0) P.a.lse[(int64_t)row.x * P.a.q_heads + h] = none ? -INFINITY : m * LN2 + logf(l);
    }
}

// dq, and the statistics the source-order pass needs per (destination, head).  Bound like the forward pass by the gathers of
// k and v, here in single elements.
template <typename T, int VE, int NV, int G, int U>
__global__ void __launch_bounds__(AT_THREADS) k_attend_dq(const __grid_constant__ Attend P) {
    constexpr int E = VE * NV;
    const int lane = threadIdx.x & 31, t = lane & (P.tl - 1), slot = (lane / P.tl) & (P.slots - 1);
    const int width = P.tl * P.slots, per_block = AT_THREADS / width;
    const int rows = P.chunk_mode ? __ldcg(P.words) : length_of(P.rows), cols = length_of(P.columns);
    const int64_t units = (int64_t)rows * P.units_per_row;
    const float c2 = P.a.scale * LOG2E;
    const int D = P.a.head_dim;
    const T* kbase = (const T*)P.a.k.data;
    const T* vbase = (const T*)P.a.v.data;
    for (int64_t base = (int64_t)blockIdx.x * per_block; base < units; base += (int64_t)gridDim.x * per_block) {
        const int64_t u = base + threadIdx.x / width;
        const Work w = find_work(P, u, units, t == 0 && slot == 0);
        const bool in = u < units;
        const int h0 = w.unit * G, g = h0 / (P.a.q_heads / P.a.kv_heads);
        constexpr bool SHIFTED = rounded_out<T>;
        float q[G][E], go[G][E], acc[G][E], lse2[G], delta[G];
        float pk[SHIFTED ? G : 1][SHIFTED ? E : 1], miss[G];
#pragma unroll
        for (int i = 0; i < G; ++i) {
            Piece<T, VE, NV> p;
            float o[E];
            p.load((const T*)P.a.out.data + (int64_t)w.row * P.a.out.row_stride + (int64_t)(h0 + i) * P.a.out.head_stride, t, P.tl, D, in);
            p.get(o);
            p.load((const T*)P.a.dout.data + (int64_t)w.row * P.a.dout.row_stride + (int64_t)(h0 + i) * P.a.dout.head_stride, t, P.tl, D, in);
            p.get(go[i]);
            p.load((const T*)P.a.q.data + (int64_t)w.row * P.a.q.row_stride + (int64_t)(h0 + i) * P.a.q.head_stride, t, P.tl, D, in);
            p.get(q[i]);
            delta[i] = 0.f;
#pragma unroll
            for (int c = 0; c < E; ++c) {
                delta[i] = fmaf(go[i][c], o[c], delta[i]);
                acc[i][c] = 0.f;
                if constexpr (SHIFTED) pk[i][c] = 0.f;
            }
            miss[i] = 0.f;
            lse2[i] = in ? backward_lse(__ldg(P.a.lse + (int64_t)w.row * P.a.q_heads + h0 + i)) : 0.f;
        }
        group_sum<G>(delta, P.tl);
        if (in && !P.chunk_mode && slot == 0 && t == 0) {
#pragma unroll
            for (int i = 0; i < G; ++i) P.stat[(int64_t)w.row * P.a.q_heads + h0 + i] = make_float2(lse2[i], delta[i]);
        }
        const int mine = (w.end - w.begin + P.slots * U - 1) / (P.slots * U);
        const int trips = __reduce_max_sync(FULL, mine);
        auto walk = [&](auto look) {
            for (int it = 0; it < trips; ++it) {
                Piece<T, VE, NV> kp[U], vp[U];
                bool on[U];
#pragma unroll
                for (int j = 0; j < U; ++j) {
                    const int e = w.begin + (it * U + j) * P.slots + slot;
                    const int col = e < w.end ? __ldg(P.cols + e) : -1;
                    on[j] = (uint32_t)col < (uint32_t)cols;
                    kp[j].load(kbase + (int64_t)col * P.a.k.row_stride + (int64_t)g * P.a.k.head_stride, t, P.tl, D, on[j]);
                    vp[j].load(vbase + (int64_t)col * P.a.v.row_stride + (int64_t)g * P.a.v.head_stride, t, P.tl, D, on[j]);
                }
                float s[2 * U * G];
#pragma unroll
                for (int j = 0; j < U; ++j) {
                    float k[E], v[E];
                    kp[j].get(k);
                    vp[j].get(v);
#pragma unroll
                    for (int i = 0; i < G; ++i) {
                        float x = 0.f, y = 0.f;
#pragma unroll
                        for (int c = 0; c < E; ++c) {
                            x = fmaf(q[i][c], k[c], x);
                            y = fmaf(go[i][c], v[c], y);
                        }
                        s[j * G + i] = x;
                        s[U * G + j * G + i] = y;
                    }
                }
                group_sum<2 * U * G>(s, P.tl);
#pragma unroll
                for (int j = 0; j < U; ++j) {
                    float k[E];
                    kp[j].get(k);
#pragma unroll
                    for (int i = 0; i < G; ++i) {
                        const float p = on[j] ? fast_exp2(fmaf(s[j * G + i], c2, -lse2[i])) : 0.f;
                        const float ds = on[j] ? p * (s[U * G + j * G + i] - delta[i]) : 0.f;
                        if (decltype(look)::value && p == 0.f) continue;
#pragma unroll
                        for (int c = 0; c < E; ++c) {
                            acc[i][c] = fmaf(ds, k[c], acc[i][c]);
                            if constexpr (SHIFTED) pk[i][c] = fmaf(p, k[c], pk[i][c]);
                        }
                        miss[i] += ds;
                    }
                }
            }
        };
        walk(std::false_type{});
        bool finite = true;
#pragma unroll
        for (int i = 0; i < G; ++i)
#pragma unroll
            for (int c = 0; c < E; ++c) finite = finite && acc[i][c] * 0.f == 0.f;
        if (!__all_sync(FULL, finite)) {                              // once more, without the edges of probability zero
#pragma unroll
            for (int i = 0; i < G; ++i) {
                miss[i] = 0.f;
#pragma unroll
                for (int c = 0; c < E; ++c) {
                    acc[i][c] = 0.f;
                    if constexpr (SHIFTED) pk[i][c] = 0.f;
                }
            }
            walk(std::true_type{});
        }
        for (int o = P.tl; o < width; o <<= 1) {
#pragma unroll
            for (int i = 0; i < G; ++i) {
                if constexpr (SHIFTED) miss[i] += __shfl_xor_sync(FULL, miss[i], o);
#pragma unroll
                for (int c = 0; c < E; ++c) {
                    acc[i][c] += __shfl_xor_sync(FULL, acc[i][c], o);
                    if constexpr (SHIFTED) pk[i][c] += __shfl_xor_sync(FULL, pk[i][c], o);
                }
            }
        }
        if (!w.live || slot) continue;
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const int h = h0 + i;
            if (P.chunk_mode) {
                float* part = P.partial + ((int64_t)w.item * P.a.q_heads + h) * dq_part<T>(D);
                store_partial<VE, NV>(part, t, P.tl, D, acc[i]);
                if constexpr (SHIFTED) {
                    store_partial<VE, NV>(part + D, t, P.tl, D, pk[i]);
                    if (t == 0) part[2 * D] = miss[i];
                }
            } else {
                if (SHIFTED && t == 0) P.stat[(int64_t)w.row * P.a.q_heads + h] = make_float2(lse2[i], delta[i] + miss[i]);
#pragma unroll
                for (int c = 0; c < E; ++c) {
                    if constexpr (SHIFTED) acc[i][c] = fmaf(-miss[i], pk[i][c], acc[i][c]);
                    acc[i][c] *= P.a.scale;
                }
                store_piece<T, VE, NV>((T*)P.a.dq.data + (int64_t)w.row * P.a.dq.row_stride + (int64_t)h * P.a.dq.head_stride, t, P.tl, D, acc[i]);
            }
        }
    }
}

// dk and dv of one (source, key/value head): over the destinations that list it, and over the query heads that share it.
template <typename T, int VE, int NV, int G, int U>
__global__ void __launch_bounds__(AT_THREADS) k_attend_dkv(const __grid_constant__ Attend P) {
    constexpr int E = VE * NV;
    const int lane = threadIdx.x & 31, t = lane & (P.tl - 1), slot = (lane / P.tl) & (P.slots - 1);
    const int width = P.tl * P.slots, per_block = AT_THREADS / width;
    const int rows = P.chunk_mode ? __ldcg(P.words) : length_of(P.rows), cols = length_of(P.columns);
    const int64_t units = (int64_t)rows * P.units_per_row;
    const float c2 = P.a.scale * LOG2E;
    const int D = P.a.head_dim, group = P.a.q_heads / P.a.kv_heads;
    const T* qbase = (const T*)P.a.q.data;
    const T* gbase = (const T*)P.a.dout.data;
    for (int64_t base = (int64_t)blockIdx.x * per_block; base < units; base += (int64_t)gridDim.x * per_block) {
        const Work w = find_work(P, base + threadIdx.x / width, units, t == 0 && slot == 0);
        const int g = w.unit;
        float k[E], v[E], dk[E], dv[E];
        {
            Piece<T, VE, NV> p;
            const bool any = w.live && w.end > w.begin;
            p.load((const T*)P.a.k.data + (int64_t)w.row * P.a.k.row_stride + (int64_t)g * P.a.k.head_stride, t, P.tl, D, any);
            p.get(k);
            p.load((const T*)P.a.v.data + (int64_t)w.row * P.a.v.row_stride + (int64_t)g * P.a.v.head_stride, t, P.tl, D, any);
            p.get(v);
        }
#pragma unroll
        for (int c = 0; c < E; ++c) dk[c] = dv[c] = 0.f;
        const int mine = (w.end - w.begin + P.slots * U - 1) / (P.slots * U);
        const int trips = __reduce_max_sync(FULL, mine);
        auto walk = [&](auto look) {
            for (int h0 = g * group; h0 < (g + 1) * group; h0 += G) {
                for (int it = 0; it < trips; ++it) {
                    Piece<T, VE, NV> qp[U][G], gp[U][G];
                    float2 st[U][G];
                    bool on[U];
#pragma unroll
                    for (int j = 0; j < U; ++j) {
                        const int e = w.begin + (it * U + j) * P.slots + slot;
                        const int col = e < w.end ? __ldg(P.cols + e) : -1;
                        on[j] = (uint32_t)col < (uint32_t)cols;
#pragma unroll
                        for (int i = 0; i < G; ++i) {
                            qp[j][i].load(qbase + (int64_t)col * P.a.q.row_stride + (int64_t)(h0 + i) * P.a.q.head_stride, t, P.tl, D, on[j]);
                            gp[j][i].load(gbase + (int64_t)col * P.a.dout.row_stride + (int64_t)(h0 + i) * P.a.dout.head_stride, t, P.tl, D, on[j]);
                            st[j][i] = on[j] ? __ldg(P.stat + (int64_t)col * P.a.q_heads + h0 + i) : make_float2(0.f, 0.f);
                        }
                    }
                    float s[2 * U * G];
#pragma unroll
                    for (int j = 0; j < U; ++j)
#pragma unroll
                        for (int i = 0; i < G; ++i) {
                            float q[E], go[E], x = 0.f, y = 0.f;
                            qp[j][i].get(q);
                            gp[j][i].get(go);
#pragma unroll
                            for (int c = 0; c < E; ++c) {
                                x = fmaf(q[c], k[c], x);
                                y = fmaf(go[c], v[c], y);
                            }
                            s[j * G + i] = x;
                            s[U * G + j * G + i] = y;
                        }
                    group_sum<2 * U * G>(s, P.tl);
#pragma unroll
                    for (int j = 0; j < U; ++j)
#pragma unroll
                        for (int i = 0; i < G; ++i) {
                            float q[E], go[E];
                            qp[j][i].get(q);
                            gp[j][i].get(go);
                            const float p = on[j] ? fast_exp2(fmaf(s[j * G + i], c2, -st[j][i].x)) : 0.f;
                            const float ds = on[j] ? p * (s[U * G + j * G + i] - st[j][i].y) : 0.f;
                            if (decltype(look)::value && p == 0.f) continue;
#pragma unroll
                            for (int c = 0; c < E; ++c) {
                                dv[c] = fmaf(p, go[c], dv[c]);
                                dk[c] = fmaf(ds, q[c], dk[c]);
                            }
                        }
                }
            }
        };
        walk(std::false_type{});
        bool finite = true;
#pragma unroll
        for (int c = 0; c < E; ++c) finite = finite && dk[c] * 0.f == 0.f && dv[c] * 0.f == 0.f;
        if (!__all_sync(FULL, finite)) {                              // once more, without the edges of probability zero
#pragma unroll
            for (int c = 0; c < E; ++c) dk[c] = dv[c] = 0.f;
            walk(std::true_type{});
        }
        for (int o = P.tl; o < width; o <<= 1) {
#pragma unroll
            for (int c = 0; c < E; ++c) {
                dk[c] += __shfl_xor_sync(FULL, dk[c], o);
                dv[c] += __shfl_xor_sync(FULL, dv[c], o);
            }
        }
        if (!w.live || slot) continue;
        if (P.chunk_mode) {
            float* part = P.partial + ((int64_t)w.item * P.a.kv_heads + g) * 2 * D;
            store_partial<VE, NV>(part, t, P.tl, D, dk);
            store_partial<VE, NV>(part + D, t, P.tl, D, dv);
        } else {
#pragma unroll
            for (int c = 0; c < E; ++c) dk[c] *= P.a.scale;
            store_piece<T, VE, NV>((T*)P.a.dk.data + (int64_t)w.row * P.a.dk.row_stride + (int64_t)g * P.a.dk.head_stride, t, P.tl, D, dk);
            store_piece<T, VE, NV>((T*)P.a.dv.data + (int64_t)w.row * P.a.dv.row_stride + (int64_t)g * P.a.dv.head_stride, t, P.tl, D, dv);
        }
    }
}

// The ring kernels have no second walk over a row's edges.  Their dq pass says whether there may be edges of probability
// zero to leave out, in a sum that is not finite or a row without weights; the elements that came out not finite are then
// taken again behind the source-order pass, from p and ds, without those edges and else in the same order.
struct Again {
    const Attend& P;
    // The sum over the edges [b, e), in chunks as the passes take them; part(b, e): over some of them in a row.
    template <typename F> __device__ float sum(int b, int e, bool split, F part) const {
        constexpr int W = AT_THREADS / 32;
        if (!split || e - b <= AT_CHUNK) return part(b, e);
        const int nc = (e - b + AT_CHUNK - 1) / AT_CHUNK, per = (nc + W - 1) / W;
        float all = 0.f;
        for (int c0 = 0; c0 < nc && all == all; c0 += per) {
            float share = 0.f;
            for (int c = c0; c < c0 + per && c < nc && share == share; ++c) share += part(b + c * AT_CHUNK, b + (c + 1) * AT_CHUNK < e ? b + (c + 1) * AT_CHUNK : e);
            all += share;
        }
        return all;
    }
    template <typename T> __device__ float dq(int row, int b, int e, int h, int col) const {
        const HeadView& k = P.a.k;
        const T* from = (const T*)k.data + (int64_t)(h / (P.a.q_heads / P.a.kv_heads)) * k.head_stride + col;
        const int cols = length_of(P.a.src);
        auto over = [&](bool pk) {                                   // sum p (dp - delta) k, or sum p k
            return sum(b, e, P.dst_split, [&](int b, int e) {
                float acc = 0.f;
                for (int i = b; i < e && acc == acc; ++i) {          // NaN stays
                    const int j = __ldg(P.a.indices + i);
                    if ((uint32_t)j >= (uint32_t)cols) continue;
                    const float2 pd = __ldg(P.pd + (int64_t)i * P.a.q_heads + h);
                    if (pd.x != 0.f) acc = fmaf(pk ? pd.x : pd.y, to_f32(from[(int64_t)j * k.row_stride]), acc);
                }
                return acc;
            });
        };
        const float acc = over(false), pk = rounded_out<T> ? over(true) : 0.f;
        return (pk != 0.f ? fmaf(-__ldg(P.shift + (int64_t)row * P.a.q_heads + h), pk, acc) : acc) * P.a.scale;
    }
    template <typename T> __device__ float kv(int b, int e, int g, int col, bool dv) const {
        const HeadView& x = dv ? P.a.dout : P.a.q;
        const int group = P.a.q_heads / P.a.kv_heads, walk = group % 4 == 0 ? 4 : (group % 2 == 0 ? 2 : 1), cols = length_of(P.a.dst);
        const float s = sum(b, e, P.split, [&](int b, int e) {
            float acc = 0.f;
            for (int h0 = g * group; h0 < (g + 1) * group; h0 += walk)
                for (int i = b; i < e && acc == acc; ++i) {
                    const int row = __ldg(P.cols + i), edge = __ldg(P.edges + i);
                    if ((uint32_t)row >= (uint32_t)cols || (uint32_t)edge >= (uint32_t)P.edge_bound) continue;
                    for (int h = h0; h < h0 + walk; ++h) {
                        const float2 pd = __ldg(P.pd + (int64_t)edge * P.a.q_heads + h);
                        if (pd.x == 0.f) continue;
                        const float ds = rounded_out<T> ? fmaf(-pd.x, __ldg(P.shift + (int64_t)row * P.a.q_heads + h), pd.y) : pd.y;
                        acc = fmaf(dv ? pd.x : ds, to_f32(((const T*)x.data)[(int64_t)row * x.row_stride + (int64_t)h * x.head_stride + col]), acc);
                    }
                }
            return acc;
        });
        return dv ? s : s * P.a.scale;
    }
    // Offsets of a row within the edges.
    __device__ int2 range(const int32_t* starts, int row) const {
        const int b = __ldg(starts + row), e = __ldg(starts + row + 1), b1 = b < 0 ? 0 : b, e1 = e > P.edge_bound ? P.edge_bound : e;
        return make_int2(b1, e1 < b1 ? b1 : e1);
    }
    // The rows of a gradient, a warp per (row, head); without `longs`, those of chunks are looked at where they are joined.
    template <typename T, typename F> __device__ void rows(const HeadView& v, const int32_t* starts, int n, int heads, bool longs, F again) const {
        const int lane = threadIdx.x & 31;
        for (int64_t u = ((int64_t)blockIdx.x * AT_THREADS + threadIdx.x) / 32; u < (int64_t)n * heads; u += (int64_t)gridDim.x * AT_THREADS / 32) {
            const int row = (int)(u / heads), h = (int)(u - (int64_t)row * heads);
            const int2 r = range(starts, row);
            if (!longs && r.y - r.x > AT_CHUNK) continue;
            T* x = (T*)v.data + (int64_t)row * v.row_stride + (int64_t)h * v.head_stride;
            for (int col = lane; col < P.a.head_dim; col += 32)
                if (to_f32(x[col]) * 0.f != 0.f) x[col] = from_f32<T>(again(row, r.x, r.y, h, col));
        }
    }
    template <typename T> __device__ void all() const {
        const int n = length_of(P.a.dst), src = length_of(P.a.src);
        rows<T>(P.a.dq, P.a.indptr, n, P.a.q_heads, true, [&](int row, int b, int e, int h, int col) { return dq<T>(row, b, e, h, col); });
        rows<T>(P.a.dk, P.starts, src, P.a.kv_heads, !P.split, [&](int, int b, int e, int h, int col) { return kv<T>(b, e, h, col, false); });
        rows<T>(P.a.dv, P.starts, src, P.a.kv_heads, !P.split, [&](int, int b, int e, int h, int col) { return kv<T>(b, e, h, col, true); });
    }
};

// Chunk sums of long rows added in order: one block per (row, head), its warps over shares of the chunks.  dq: one operand
// of width D; dk and dv: width 2 D, the second half for dv.
template <typename T, bool KV> __global__ void __launch_bounds__(AT_THREADS) k_attend_sum_join(const __grid_constant__ Attend P) {
    constexpr int W = AT_THREADS / 32;
    __shared__ float s_acc[W][513];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, D = P.a.head_dim;
    const int heads = KV ? P.a.kv_heads : P.a.q_heads, width = KV ? 2 * D : dq_part<T>(D);
    const int64_t units = (int64_t)__ldcg(P.words + 1) * heads, stride = (int64_t)heads * width;
    const Again again{P};
    const bool look = KV && __ldcg(P.look) != 0;
    if (look) again.all<T>();
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int4 row = P.longs[u / heads];
        const int h = (int)(u % heads);
        const float* part = P.partial + (int64_t)row.y * stride + (int64_t)h * width;
        const int per = (row.z + W - 1) / W, c0 = warp * per, c1 = c0 + per < row.z ? c0 + per : row.z;
        __syncthreads();                                       // the previous unit's sums are read
        for (int col = lane; col < width; col += 32) {
            float acc = 0.f;
#pragma unroll 4
            for (int c = c0; c < c1; ++c) acc += part[c * stride + col];
            s_acc[warp][col] = acc;
        }
        __syncthreads();
        if constexpr (!KV && rounded_out<T>) {
            float miss = 0.f;
            for (int w = 0; w < W; ++w) miss += s_acc[w][2 * D];
            for (int col = threadIdx.x; col < D; col += AT_THREADS) {
                float acc = 0.f, pk = 0.f;
                for (int w = 0; w < W; ++w) {
                    acc += s_acc[w][col];
                    pk += s_acc[w][D + col];
                }
                ((T*)P.a.dq.data)[(int64_t)row.x * P.a.dq.row_stride + (int64_t)h * P.a.dq.head_stride + col] = from_f32<T>(fmaf(-miss, pk, acc) * P.a.scale);
            }
            if (threadIdx.x == 0) {
                const int64_t at = (int64_t)row.x * P.a.q_heads + h;
                if (P.shift) P.shift[at] = miss;
                else P.stat[at].y += miss;
            }
            continue;
        }
        for (int col = threadIdx.x; col < width; col += AT_THREADS) {
            float acc = 0.f;
            for (int w = 0; w < W; ++w) acc += s_acc[w][col];
            const HeadView& to = !KV ? P.a.dq : (col < D ? P.a.dk : P.a.dv);
            if (!KV || col < D) acc *= P.a.scale;
            if (look && acc * 0.f != 0.f) {
                const int2 r = again.range(P.starts, row.x);
                acc = again.kv<T>(r.x, r.y, h, col < D ? col : col - D, col >= D);
            }
            ((T*)to.data)[(int64_t)row.x * to.row_stride + (int64_t)h * to.head_stride + (col < D ? col : col - D)] = from_f32<T>(acc);
        }
    }
}

}  // namespace gs

#include "gs_attend_ring.cuh"

namespace gs {

// The destination of every edge, in edge order: 8 lanes per row.
__global__ void __launch_bounds__(AT_THREADS) k_edge_rows(const int32_t* __restrict__ indptr, Count dst, int edge_bound, int32_t* __restrict__ rows) {
    chain_wait();
    const int n = length_of(dst), t = threadIdx.x & 7;
    for (int64_t r = (int64_t)blockIdx.x * (AT_THREADS / 8) + threadIdx.x / 8; r < n; r += (int64_t)gridDim.x * (AT_THREADS / 8)) {
        const int b = __ldg(indptr + r), end = __ldg(indptr + r + 1), e = end < edge_bound ? end : edge_bound;
        for (int i = (b < 0 ? 0 : b) + t; i < e; i += 8) rows[i] = (int32_t)r;
    }
}

// The destinations in the order of the sorted edges; with STARTS also the sources' offsets, from the places where the
// key changes (4.36 M edges, 2.03 M sources: 48 us, 59 as two kernels with a search per source): short gaps of sources without edges by the thread that sees them, long ones by the block.
template <bool STARTS>
__global__ void __launch_bounds__(AT_THREADS) k_edge_finish(Count edges, Count src, const uint32_t* __restrict__ keys, const int32_t* __restrict__ edge,
                                                            const int32_t* __restrict__ rows, int32_t* __restrict__ out, int32_t* __restrict__ starts) {
    constexpr int U = 4, TILE = AT_THREADS * U, SHORT = 8;
    __shared__ int gaps[TILE][3], s_gaps;
    chain_wait();
    const int n = length_of(edges);
    const int64_t num_src = STARTS ? length_of(src) : 0;
    for (int64_t base = (int64_t)blockIdx.x * TILE; base <= n; base += (int64_t)gridDim.x * TILE) {      // n itself: the end of the last row
        if (STARTS) {
            __syncthreads();
            if (threadIdx.x == 0) s_gaps = 0;
            __syncthreads();
        }
        int e[U];
        int64_t k0[U], k1[U];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int64_t i = base + j * AT_THREADS + threadIdx.x;
            e[j] = i < n ? __ldcg(edge + i) : -1;
            if (STARTS && i <= n) {
                k0[j] = i > 0 ? (int64_t)__ldcg(keys + i - 1) : -1;
                k1[j] = i < n ? (int64_t)__ldcg(keys + i) : num_src;
                if (k1[j] > num_src) k1[j] = num_src;
            }
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int64_t i = base + j * AT_THREADS + threadIdx.x;
            if (i < n) out[i] = __ldcg(rows + e[j]);
            if (STARTS && i <= n && k1[j] > k0[j]) {
                if (k1[j] - k0[j] <= SHORT) {
                    for (int64_t r = k0[j] + 1; r <= k1[j]; ++r) starts[r] = (int32_t)i;
                } else {
                    const int at = atomicAdd(&s_gaps, 1);
                    gaps[at][0] = (int)(k0[j] + 1);
                    gaps[at][1] = (int)k1[j];
                    gaps[at][2] = (int)i;
                }
            }
        }
        if (STARTS) {
            __syncthreads();
            for (int g = 0; g < s_gaps; ++g)
                for (int64_t r = (int64_t)gaps[g][0] + threadIdx.x; r <= gaps[g][1]; r += AT_THREADS) starts[r] = gaps[g][2];
        }
    }
}

// ---------------------------------------------------------------- launches
struct AttendLayout {
    size_t words, items, longs, stat, pd, partial, total;
};

static AttendLayout attend_layout(int64_t dst, int64_t edges, int32_t q_heads, int32_t head_dim) {
    AttendLayout l{};
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t o = off; off = align_up(off + bytes, 256); return o; };
    const int64_t chunks = 2 * (edges / AT_CHUNK) + 2;
    l.words = take(256);
    l.items = take((size_t)chunks * 8);
    l.longs = take((size_t)(edges / AT_CHUNK + 1) * 16);
    l.stat = take((size_t)dst * q_heads * 8);
    l.pd = take((size_t)edges * q_heads * 8);
    l.partial = take((size_t)chunks * q_heads * (2 * (size_t)head_dim + 2) * 4);
    l.total = off;
    return l;
}

size_t reverse_workspace(int64_t edges) { return 2 * align_up((size_t)edges * 4, 256) + key_sort_bytes(edges); }

size_t attention_workspace(int64_t dst, int64_t edges, int32_t q_heads, int32_t head_dim) {
    const size_t a = attend_layout(dst, edges, q_heads, head_dim).total, b = reverse_workspace(edges);
    return a > b ? a : b;
}

// Elements per access that the head dimension and all operands allow.
static int wide_elems(const BlockAttention& a, std::initializer_list<const HeadView*> views) {
    const int size = a.dtype == GS_BF16 ? 2 : 4;
    for (int ve = 16 / size; ve >= 4; ve /= 2) {
        bool ok = a.head_dim % ve == 0;
        for (const HeadView* v : views)
            ok = ok && ((uintptr_t)v->data % (ve * size)) == 0 && (v->row_stride * size) % (ve * size) == 0 && (v->head_stride * size) % (ve * size) == 0 &&
                 v->row_stride * size < ((int64_t)1 << 32) && v->head_stride * size * a.q_heads < ((int64_t)1 << 31);
        if (ok) return ve;
    }
    return 1;
}

static void shape_groups(Attend& P, int ve, int nv, int64_t rows, int units_per_row, int64_t row_hint) {
    const int pieces = (P.a.head_dim + ve * nv - 1) / (ve * nv);
    P.tl = 1;
    while (P.tl < pieces) P.tl *= 2;
    P.units_per_row = units_per_row;
    P.slots = 1;
    // several groups share a row while the rows alone do not give every SM sixteen warps and each group keeps four edges
    while (P.tl * P.slots * 2 <= 32 && rows * units_per_row * P.tl * P.slots * 2 <= sm_count() * 16 * 32 && (row_hint == 0 || row_hint >= 8 * P.slots)) P.slots *= 2;
}

template <AttendKind K, typename T, int VE, int NV, int G> static void run_attend(Attend P, int64_t rows, int64_t row_hint, cudaStream_t s) {
    constexpr int U = VE * NV * G >= 32 ? 2 : 4;
    const int units_per_row = K == AT_DKV ? P.a.kv_heads : P.a.q_heads / G;
    P.shift = nullptr;                                        // goes to stat
    for (int pass = 0; pass < (P.split ? 2 : 1); ++pass) {
        P.chunk_mode = pass;
        const int64_t n = pass ? 2 * ((int64_t)P.edge_bound / AT_CHUNK) + 2 : rows;
        shape_groups(P, VE, NV, n, units_per_row, pass ? AT_CHUNK : row_hint);
        const int per_block = AT_THREADS / (P.tl * P.slots);
        int64_t blocks = (n * units_per_row + per_block - 1) / per_block;
        const int64_t cap = sm_count() * (pass ? 16 : 64);
        if (blocks > cap) blocks = cap;
        const int grid = (int)limit_grid(blocks);
        if constexpr (K == AT_FORWARD) k_attend_forward<T, VE, NV, G, U><<<grid, AT_THREADS, 0, s>>>(P);
        else if constexpr (K == AT_DQ) k_attend_dq<T, VE, NV, G, U><<<grid, AT_THREADS, 0, s>>>(P);
        else k_attend_dkv<T, VE, NV, G, (G > 1 ? (U > 2 ? 2 : 1) : U)><<<grid, AT_THREADS, 0, s>>>(P);
        count_launches(1);
    }
    if (P.split) {
        const int grid = (int)limit_grid(sm_count() * 8);
        if constexpr (K == AT_FORWARD) k_attend_forward_join<T><<<grid, AT_THREADS, 0, s>>>(P);
        else k_attend_sum_join<T, K == AT_DKV><<<grid, AT_THREADS, 0, s>>>(P);
        count_launches(1);
    }
}

// The ring kernels: edge batches through shared memory.
template <AttendKind K, typename T, int VE, int NV, int G> static cudaError_t run_ring(Attend P, int64_t rows, cudaStream_t s) {
    constexpr int U = K == AT_DKV ? 2 : 4;       // edges per batch: sampled rows have tens, sources two or three (4 there: 8 % slower)
    constexpr int smem = RING_WARPS * RingShape<K, T, VE, NV, G, U>::WARP;
    auto kernel = k_attend_ring<K, T, VE, NV, G, U>;
    static std::atomic<uint64_t> allowed{0};
    cudaError_t e = allow_smem(kernel, smem, allowed);
    if (e != cudaSuccess) return e;
    P.units_per_row = K == AT_DKV ? P.a.kv_heads : P.a.q_heads / G;
    const int pieces = (P.a.head_dim + VE * NV - 1) / (VE * NV);
    P.tl = 1;
    while (P.tl < pieces) P.tl *= 2;
    const int gpw = 32 / P.tl;
    const int64_t resident = sm_count() * RING_WARPS * ((220 << 10) / smem);
    for (int pass = 0; pass < (P.split ? 2 : 1); ++pass) {
        P.chunk_mode = pass;
        const int64_t n = pass ? 2 * ((int64_t)P.edge_bound / AT_CHUNK) + 2 : rows;
        const int64_t tiles = (n * P.units_per_row + gpw - 1) / gpw;
        // rows: four rounds of all resident warps (2 and 8: 3 to 10 % slower), as far as a warp's row offsets go; chunks are long enough alone
        int64_t per = pass ? 1 : tiles / (resident * 4);
        const int64_t most = (int64_t)(RING_ROWS - 2) * P.units_per_row / gpw;
        per = per > most ? most : per;
        P.tiles = (int)(per < 1 ? 1 : per);
        int64_t blocks = (tiles + (int64_t)P.tiles * RING_WARPS - 1) / ((int64_t)P.tiles * RING_WARPS);
        const int64_t cap = pass ? resident / RING_WARPS * 2 : (int64_t)1 << 30;
        kernel<<<(int)limit_grid(blocks > cap ? cap : blocks), RING_WARPS * 32, smem, s>>>(P);
        count_launches(1);
    }
    if (P.split || K == AT_DKV) {                             // behind the source-order pass also what has to be taken again
        const int grid = (int)limit_grid(sm_count() * (K == AT_DKV ? 4 : 8));
        if constexpr (K == AT_FORWARD) k_attend_forward_join<T><<<grid, AT_THREADS, 0, s>>>(P);
        else k_attend_sum_join<T, K == AT_DKV><<<grid, AT_THREADS, 0, s>>>(P);
        count_launches(1);
    }
    return cudaGetLastError();
}

// Query heads of one key/value head that a group takes together (they share the loads of k and v).
template <AttendKind K, typename T, int VE, int NV> static cudaError_t ring_group(const Attend& P, int64_t rows, cudaStream_t s) {
    const int group = P.a.q_heads / P.a.kv_heads;
    if (group % 4 == 0) return run_ring<K, T, VE, NV, 4>(P, rows, s);
    if (group % 2 == 0) return run_ring<K, T, VE, NV, 2>(P, rows, s);
    return run_ring<K, T, VE, NV, 1>(P, rows, s);
}

template <AttendKind K> static cudaError_t run_kind(Attend& P, int ve, int64_t rows, int64_t row_hint, cudaStream_t s) {
    const int D = P.a.head_dim;
    // pieces of 16 or 8 bytes: the ring kernels; else one element at a time
    if (P.a.dtype == GS_BF16) {
        if (ve == 8) return ring_group<K, bf16, 8, 1>(P, rows, s);
        if (ve == 4 && D <= 128) return ring_group<K, bf16, 4, 1>(P, rows, s);
        if (ve == 4) return ring_group<K, bf16, 4, 2>(P, rows, s);
        if (D <= 32) run_attend<K, bf16, 1, 1, 1>(P, rows, row_hint, s);
        else if (D <= 64) run_attend<K, bf16, 1, 2, 1>(P, rows, row_hint, s);
        else if (D <= 128) run_attend<K, bf16, 1, 4, 1>(P, rows, row_hint, s);
        else run_attend<K, bf16, 1, 8, 1>(P, rows, row_hint, s);
    } else {
        if (ve == 4 && D <= 128) return ring_group<K, float, 4, 1>(P, rows, s);
        if (ve == 4) return ring_group<K, float, 4, 2>(P, rows, s);
        if (D <= 32) run_attend<K, float, 1, 1, 1>(P, rows, row_hint, s);
        else if (D <= 64) run_attend<K, float, 1, 2, 1>(P, rows, row_hint, s);
        else if (D <= 128) run_attend<K, float, 1, 4, 1>(P, rows, row_hint, s);
        else run_attend<K, float, 1, 8, 1>(P, rows, row_hint, s);
    }
    return cudaGetLastError();
}

static Attend attend_params(const BlockAttention& a, void* workspace) {
    Attend P{};
    P.a = a;
    P.edge_bound = a.edge_bound;
    const AttendLayout l = attend_layout(a.dst.bound, a.edge_bound, a.q_heads, a.head_dim);
    char* ws = (char*)workspace;
    P.words = (int32_t*)(ws + l.words);
    P.items = (int2*)(ws + l.items);
    P.longs = (int4*)(ws + l.longs);
    P.partial = (float*)(ws + l.partial);
    P.stat = (float2*)(ws + l.stat);
    P.pd = (float2*)(ws + l.pd);
    P.shift = (float*)(ws + l.stat);                         // the ring kernels keep no stat
    return P;
}

cudaError_t launch_attention_forward(const BlockAttention& a, void* workspace, cudaStream_t s) {
    Attend P = attend_params(a, workspace);
    P.starts = a.indptr;
    P.cols = a.indices;
    P.rows = a.dst;
    P.columns = a.src;
    P.split = (a.max_row == 0 || a.max_row > AT_CHUNK) && a.edge_bound > AT_CHUNK;
    const cudaError_t e = P.split ? cudaMemsetAsync(P.words, 0, 8, s) : cudaSuccess;
    if (e != cudaSuccess) return e;
    return run_kind<AT_FORWARD>(P, wide_elems(a, {&a.q, &a.k, &a.v, &a.out}), a.dst.bound, a.max_row, s);
}

cudaError_t launch_attention_backward(const BlockAttention& a, const int32_t* rev_indptr, const int32_t* rev_dst, const int32_t* rev_edge,
                                      void* workspace, cudaStream_t s) {
    Attend P = attend_params(a, workspace);
    const int ve = wide_elems(a, {&a.q, &a.k, &a.v, &a.out, &a.dout, &a.dq, &a.dk, &a.dv});
    P.starts = a.indptr;
    P.cols = a.indices;
    P.rows = a.dst;
    P.columns = a.src;
    P.split = (a.max_row == 0 || a.max_row > AT_CHUNK) && a.edge_bound > AT_CHUNK;
    // the words of both passes, cleared at once
    int32_t* kv_words = P.words + 2;
    P.look = P.words + 4;
    cudaError_t e = cudaMemsetAsync(P.words, 0, 5 * 4, s);
    if (e == cudaSuccess) e = run_kind<AT_DQ>(P, ve, a.dst.bound, a.max_row, s);
    if (e != cudaSuccess) return e;
    P.words = kv_words;
    P.dst_split = P.split;
    P.starts = rev_indptr;
    P.cols = rev_dst;
    P.edges = rev_edge;
    P.rows = a.src;
    P.columns = a.dst;
    P.split = a.edge_bound > AT_CHUNK;
    return run_kind<AT_DKV>(P, ve, a.src.bound, 0, s);
}

cudaError_t launch_block_reverse(const int32_t* indptr, const int32_t* indices, Count dst, Count src, Count edges, int32_t* rev_indptr,
                                 int32_t* rev_dst, int32_t* rev_edge, void* workspace, cudaStream_t s) {
    const size_t list = align_up((size_t)edges.bound * 4, 256);
    int32_t* rows = (int32_t*)workspace;
    uint32_t* keys = (uint32_t*)((char*)workspace + list);
    int64_t blocks = ((int64_t)dst.bound + AT_THREADS / 8 - 1) / (AT_THREADS / 8);
    if (blocks > sm_count() * 32) blocks = sm_count() * 32;
    cudaError_t e = launch_train(k_edge_rows, blocks, AT_THREADS, 0, s, indptr, dst, (int)edges.bound, rows);
    // edges before the first row's offset or behind the last row belong to no destination
    if (e == cudaSuccess) e = launch_key_sort(indices, nullptr, edges, Rows{indptr, dst}, src.bound, (char*)workspace + 2 * list, keys, rev_edge, nullptr, 0, Fill{}, s);
    if (e != cudaSuccess) return e;
    blocks = ((int64_t)edges.bound + AT_THREADS * 4) / (AT_THREADS * 4);
    if (blocks > sm_count() * 16) blocks = sm_count() * 16;
    // More than two sources to an edge (no sampled block has that): the gaps between keys are long, and a search per source
    // is the shorter way.  Whole call, offsets from the gaps | by searches: 4.2 M edges, as many sources 219 | 244 us, twice
    // as many 242 | 270, four times 381 | 326, sixteen times 955 | 536; 65,536 edges: 44 | 51, 50 | 51, 79 | 55, 167 | 54.
    if ((int64_t)src.bound > 2 * (int64_t)edges.bound) {
        e = launch_row_starts(keys, edges, src, rev_indptr, s);
        if (e == cudaSuccess) e = launch_train(k_edge_finish<false>, blocks, AT_THREADS, 0, s, edges, src, keys, rev_edge, rows, rev_dst, rev_indptr);
    } else {
        e = launch_train(k_edge_finish<true>, blocks, AT_THREADS, 0, s, edges, src, keys, rev_edge, rows, rev_dst, rev_indptr);
    }
    return e;
}

}  // namespace gs
