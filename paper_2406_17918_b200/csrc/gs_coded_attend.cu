// Softmax attention of a block's destinations over key and value rows held in 8 bits.
//
// For destination i, query head h, its key/value head g and the edges j of row i, with codes k, v and scales of their blocks:
//   s = scale (q_ih . k_jg) 2^ek,  lse_ih = log sum_j exp s,  o_ih = sum_j exp(s - lse_ih) 2^ev v_jg.
// The scales multiply sums and weights, never single elements.  Statistics and sums are in 32 bits.
//
// A group of tl lanes holds one (row, G query heads of one key/value head); a lane has one piece of VE codes of the key and one of
// the value per edge, U edges in flight, and the next edges' rows are looked up while these are worked on.  Groups of one row's
// heads are neighbours, so that an edge's codes are read in one piece.  Where rows are few, `slots` groups share one and are joined
// at its end; rows of more than LONG edges are cut into chunks of a warp each, whose results are joined in order by a second
// kernel: no atomics on values, the result does not depend on the schedule.
#include "gs_codes.cuh"
#include "gs_device.cuh"
#include "gs_train.h"

namespace gs {

constexpr int CA_THREADS = 128;
constexpr int CA_LONG = 64;          // rows of more edges go to the chunk list
constexpr int CA_CHUNK = 256;        // edges of a chunk
constexpr float CA_LOG2E = 1.4426950408889634f, CA_LN2 = 0.6931471805599453f;

struct CodedAttend {
    CodedAttention a;
    int tl, slots, units_per_row;
    int wide;                        // q and out in whole pieces
    int split, chunk_mode;
    int32_t* words;                  // [0] chunks, [1] long rows
    int2* items;                     // chunk -> (row, chunk of the row)
    int4* longs;                     // long row -> (row, first chunk, chunks, -)
    float* partial;                  // [chunk][q head][head_dim + 2]: sum, maximum, weight
};

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ int list_length(const Count& c) {
    if (!c.d_n) return c.bound;
    const int n = __ldcg(c.d_n);
    return n < 0 ? 0 : (n > c.bound ? c.bound : n);
}

// VE codes as VE / 2 pairs.
template <int VE> struct Codes {
    uint32_t w[VE / 4];
    __device__ __forceinline__ void load(const uint8_t* p, bool on) {
        if constexpr (VE == 16) {
            const uint4 x = on ? __ldg(reinterpret_cast<const uint4*>(p)) : make_uint4(0, 0, 0, 0);
            w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
        } else {
            const uint2 x = on ? __ldg(reinterpret_cast<const uint2*>(p)) : make_uint2(0, 0);
            w[0] = x.x; w[1] = x.y;
        }
    }
    __device__ __forceinline__ void get(f32x2 (&x)[VE / 2]) const {
#pragma unroll
        for (int i = 0; i < VE / 4; ++i) {
            float a, b;
            decode2(w[i], a, b);
            x[2 * i] = pair(a, b);
            decode2(w[i] >> 16, a, b);
            x[2 * i + 1] = pair(a, b);
        }
    }
};

template <typename T, int VE> __device__ __forceinline__ void load_piece(const T* row, int c, int dim, bool wide, bool on, f32x2 (&x)[VE / 2]) {
    constexpr int P = 16 / (int)sizeof(T) < VE ? 16 / (int)sizeof(T) : VE;
    float y[VE];
#pragma unroll
    for (int i = 0; i < VE; ++i) y[i] = 0.f;
    if (on && wide) {
#pragma unroll
        for (int i = 0; i < VE; i += P) {
            if (c + i >= dim) break;
            float z[P];
            unpack<T, P>(load_raw<T, P>(row + c + i), z);
#pragma unroll
            for (int j = 0; j < P; ++j) y[i + j] = z[j];
        }
    } else if (on) {
#pragma unroll
        for (int i = 0; i < VE; ++i)
            if (c + i < dim) y[i] = to_f32(row[c + i]);
    }
#pragma unroll
    for (int i = 0; i < VE / 2; ++i) x[i] = pair(y[2 * i], y[2 * i + 1]);
}

template <typename T, int VE> __device__ __forceinline__ void store_out(T* row, int c, int dim, bool wide, const float (&y)[VE]) {
    constexpr int P = 16 / (int)sizeof(T) < VE ? 16 / (int)sizeof(T) : VE;
    if (wide) {
#pragma unroll
        for (int i = 0; i < VE; i += P) {
            if (c + i >= dim) break;
            float z[P];
#pragma unroll
            for (int j = 0; j < P; ++j) z[j] = y[i + j];
            store_vec<T, P>(row + c + i, z);
        }
    } else {
#pragma unroll
        for (int i = 0; i < VE; ++i)
            if (c + i < dim) row[c + i] = from_f32<T>(y[i]);
    }
}

template <typename T, int VE, int G, int U> __global__ void __launch_bounds__(CA_THREADS) k_coded_attend(const __grid_constant__ CodedAttend P) {
    constexpr int N2 = VE / 2;
    chain_wait();
    const int lane = threadIdx.x & 31, tl = P.tl, t = lane & (tl - 1), slot = (lane / tl) & (P.slots - 1);
    const int width = tl * P.slots, per_block = CA_THREADS / width;
    const int rows = P.chunk_mode ? __ldcg(P.words) : list_length(P.a.dst), cols = list_length(P.a.src);
    const int64_t units = (int64_t)rows * P.units_per_row;
    const float c2 = P.a.scale * CA_LOG2E;
    const int D = P.a.head_dim, c0 = t * VE;
    const bool held = c0 < P.a.k.pitch;                      // this lane has a piece of the codes
    for (int64_t base = (int64_t)blockIdx.x * per_block; base < units; base += (int64_t)gridDim.x * per_block) {
        const int64_t u = base + threadIdx.x / width;
        bool live = u < units;
        const int r = live ? (int)(u / P.units_per_row) : 0, unit = live ? (int)(u - (int64_t)r * P.units_per_row) : 0;
        int row = r, begin = 0, end = 0;
        if (live) {
            int skip = 0;
            if (P.chunk_mode) {
                const int2 it = P.items[r];
                row = it.x;
                skip = it.y * CA_CHUNK;
            }
            int b = __ldg(P.a.indptr + row), e = __ldg(P.a.indptr + row + 1);
            b = b < 0 ? 0 : b;
            e = e > P.a.edge_bound ? P.a.edge_bound : e;
            if (e < b) e = b;
            if (P.chunk_mode) {
                begin = b + skip;
                end = begin + CA_CHUNK < e ? begin + CA_CHUNK : e;
            } else if (P.split && e - b > CA_LONG) {
                if (unit == 0 && t == 0 && slot == 0) {      // listed once, from the row's first unit
                    const int nc = (e - b + CA_CHUNK - 1) / CA_CHUNK, first = atomicAdd(P.words, nc);
                    P.longs[atomicAdd(P.words + 1, 1)] = make_int4(row, first, nc, 0);
                    for (int c = 0; c < nc; ++c) P.items[first + c] = make_int2(row, c);
                }
                live = false;
            } else {
                begin = b;
                end = e;
            }
        }
        const int h0 = unit * G, g = h0 / (P.a.q_heads / P.a.kv_heads);
        const uint8_t* kbase = P.a.k.codes + (int64_t)g * P.a.k.pitch + c0;
        const uint8_t* vbase = P.a.v.codes + (int64_t)g * P.a.v.pitch + c0;
        f32x2 q[G][N2], acc[G][N2];
        float m[G], l[G];
#pragma unroll
        for (int i = 0; i < G; ++i) {
            load_piece<T, VE>((const T*)P.a.q.data + (int64_t)row * P.a.q.row_stride + (int64_t)(h0 + i) * P.a.q.head_stride, c0, D, P.wide, live, q[i]);
            m[i] = -INFINITY;
            l[i] = 0.f;
#pragma unroll
            for (int c = 0; c < N2; ++c) acc[i][c] = 0;
        }
        const int step = P.slots * U;
        const int trips = __reduce_max_sync(FULL, (end - begin + step - 1) / step);
        // the cache rows of a batch's edges, -1 where there is none
        auto look = [&](int it, int (&at)[U]) {
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const int e = begin + (it * U + j) * P.slots + slot;
                int col = e < end ? __ldg(P.a.indices + e) : -1;
                if ((uint32_t)col >= (uint32_t)cols) col = -1;
                if (P.a.row_of && col >= 0) col = __ldg(P.a.row_of + col);
                at[j] = (uint32_t)col < (uint64_t)P.a.k.rows ? col : -1;
            }
        };
        int next[U];
        look(0, next);
        for (int it = 0; it < trips; ++it) {
            int at[U];
            Codes<VE> kc[U], vc[U];
            uint32_t ks[U], vs[U];
#pragma unroll
            for (int j = 0; j < U; ++j) {
                at[j] = next[j];
                const bool on = at[j] >= 0;
                const int64_t b = at[j] >> P.a.k.shift;
                kc[j].load(kbase + (int64_t)at[j] * P.a.k.row_stride, on && held);
                vc[j].load(vbase + (int64_t)at[j] * P.a.v.row_stride, on && held);
                ks[j] = on ? __ldg(P.a.k.scales + b * P.a.k.scale_stride + g) : 0u;
                vs[j] = on ? __ldg(P.a.v.scales + b * P.a.v.scale_stride + g) : 0u;
            }
            look(it + 1, next);
            float s[U * G];
#pragma unroll
            for (int j = 0; j < U; ++j) {
                f32x2 k[N2];
                kc[j].get(k);
#pragma unroll
                for (int i = 0; i < G; ++i) {
                    f32x2 x = mul2(q[i][0], k[0]);
#pragma unroll
                    for (int c = 1; c < N2; ++c) x = fma2(q[i][c], k[c], x);
                    float lo, hi;
                    split(x, lo, hi);
                    s[j * G + i] = lo + hi;
                }
            }
            for (int o = 1; o < tl; o <<= 1) {
#pragma unroll
                for (int x = 0; x < U * G; ++x) s[x] += __shfl_xor_sync(FULL, s[x], o);
            }
            float p[U * G];
#pragma unroll
            for (int i = 0; i < G; ++i) {
                float top = m[i];
#pragma unroll
                for (int j = 0; j < U; ++j) {
                    s[j * G + i] = at[j] >= 0 ? s[j * G + i] * scale_of(ks[j]) * c2 : -INFINITY;
                    top = fmaxf(top, s[j * G + i]);
                }
                const float ref = top == -INFINITY ? 0.f : top;     // nothing seen yet: all weights are zero
                const float corr = exp2_fast(m[i] - ref);
                m[i] = top;
                l[i] *= corr;
#pragma unroll
                for (int j = 0; j < U; ++j) {
                    p[j * G + i] = exp2_fast(s[j * G + i] - ref);
                    l[i] += p[j * G + i];
                }
                const f32x2 cc = pair(corr, corr);
#pragma unroll
                for (int c = 0; c < N2; ++c) acc[i][c] = mul2(cc, acc[i][c]);
            }
#pragma unroll
            for (int j = 0; j < U; ++j) {
                f32x2 v[N2];
                vc[j].get(v);
                const float sv = scale_of(vs[j]);
#pragma unroll
                for (int i = 0; i < G; ++i) {
                    const float w = p[j * G + i] * sv;
                    const f32x2 ww = pair(w, w);
#pragma unroll
                    for (int c = 0; c < N2; ++c) acc[i][c] = fma2(ww, v[c], acc[i][c]);
                }
            }
        }
        for (int o = tl; o < width; o <<= 1) {                        // join the slots of a row
#pragma unroll
            for (int i = 0; i < G; ++i) {
                const float mo = __shfl_xor_sync(FULL, m[i], o), lo = __shfl_xor_sync(FULL, l[i], o);
                const float top = fmaxf(m[i], mo), ref = top == -INFINITY ? 0.f : top;
                const float ca = exp2_fast(m[i] - ref), cb = exp2_fast(mo - ref);
                m[i] = top;
                l[i] = l[i] * ca + lo * cb;
                const f32x2 aa = pair(ca, ca), bb = pair(cb, cb);
#pragma unroll
                for (int c = 0; c < N2; ++c) acc[i][c] = fma2(aa, acc[i][c], mul2(bb, __shfl_xor_sync(FULL, acc[i][c], o)));
            }
        }
        if (!live || slot) continue;
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const int h = h0 + i;
            float y[VE];
#pragma unroll
            for (int c = 0; c < N2; ++c) split(acc[i][c], y[2 * c], y[2 * c + 1]);
            if (P.chunk_mode) {
                float* part = P.partial + ((int64_t)r * P.a.q_heads + h) * (D + 2);
#pragma unroll
                for (int c = 0; c < VE; ++c)
                    if (c0 + c < D) part[c0 + c] = y[c];
                if (t == 0) {
                    part[D] = m[i];
                    part[D + 1] = l[i];
                }
            } else {
                const bool none = l[i] == 0.f;                        // no edge left by the mask: zero row, log of an empty sum
                const float inv = none ? 0.f : 1.f / l[i];
#pragma unroll
                for (int c = 0; c < VE; ++c) y[c] = none ? 0.f : y[c] * inv;
                store_out<T, VE>((T*)P.a.out.data + (int64_t)row * P.a.out.row_stride + (int64_t)h * P.a.out.head_stride, c0, D, P.wide, y);
                if (t == 0) P.a.lse[(int64_t)row * P.a.q_heads + h] = none ? -INFINITY : m[i] * CA_LN2 + logf(l[i]);
            }
        }
    }
}

// One block per (long row, query head): the chunks' sums rescaled to the common maximum; each warp adds a contiguous share of the
// chunks, the shares are added in order.
template <typename T> __global__ void __launch_bounds__(256) k_coded_attend_join(const __grid_constant__ CodedAttend P) {
    constexpr int W = 8;
    __shared__ float s_m[W], s_l[W], s_acc[W][256];
    chain_wait();
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
        for (int c = c0 + lane; c < c1; c += 32) l += part[c * stride + D + 1] * exp2_fast(part[c * stride + D] - ref);
        for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(FULL, l, o);
        if (lane == 0) s_l[warp] = l;
        for (int col = lane; col < D; col += 32) {
            float acc = 0.f;
#pragma unroll 4
            for (int c = c0; c < c1; ++c) acc = fmaf(part[c * stride + col], exp2_fast(part[c * stride + D] - ref), acc);
            s_acc[warp][col] = acc;
        }
        __syncthreads();
        l = 0.f;
        for (int w = 0; w < W; ++w) l += s_l[w];
        const bool none = l == 0.f;
        const float inv = none ? 0.f : 1.f / l;
        T* out = (T*)P.a.out.data + (int64_t)row.x * P.a.out.row_stride + (int64_t)h * P.a.out.head_stride;
        for (int col = threadIdx.x; col < D; col += 256) {
            float acc = 0.f;
            for (int w = 0; w < W; ++w) acc += s_acc[w][col];
            out[col] = from_f32<T>(none ? 0.f : acc * inv);
        }
        if (threadIdx.x == 0) P.a.lse[(int64_t)row.x * P.a.q_heads + h] = none ? -INFINITY : m * CA_LN2 + logf(l);
    }
}

// ---------------------------------------------------------------- launches
struct CodedAttendLayout {
    size_t words, items, longs, partial, total;
};
static CodedAttendLayout coded_attend_layout(int64_t edges, int32_t q_heads, int32_t head_dim) {
    CodedAttendLayout l{};
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t o = off; off = align_up(off + bytes, 256); return o; };
    const int64_t most = edges / CA_LONG + 1;                // chunks, and long rows: each has more than LONG edges
    l.words = take(256);
    l.items = take((size_t)most * 8);
    l.longs = take((size_t)most * 16);
    l.partial = take((size_t)most * q_heads * (head_dim + 2) * 4);
    l.total = off;
    return l;
}
size_t coded_attention_workspace(int64_t edges, int32_t q_heads, int32_t head_dim) { return coded_attend_layout(edges, q_heads, head_dim).total; }

template <typename T, int VE, int G, int U> static cudaError_t run_coded(CodedAttend P, cudaStream_t s) {
    const int pieces = P.a.k.pitch / VE;
    P.tl = 1;
    while (P.tl < pieces) P.tl *= 2;
    P.units_per_row = P.a.q_heads / G;
    cudaError_t e = cudaSuccess;
    for (int pass = 0; pass < (P.split ? 2 : 1) && e == cudaSuccess; ++pass) {
        P.chunk_mode = pass;
        const int64_t n = pass ? (int64_t)P.a.edge_bound / CA_LONG + 1 : P.a.dst.bound;
        P.slots = pass ? 32 / P.tl : 1;
        // groups share a row while the rows alone do not give every SM sixteen warps and each keeps U edges
        const int longest = P.a.max_row == 0 || P.a.max_row > CA_LONG ? CA_LONG : P.a.max_row;
        while (!pass && P.tl * P.slots * 2 <= 32 && n * P.units_per_row * P.tl * P.slots * 2 <= sm_count() * 16 * 32 && P.slots * U < longest) P.slots *= 2;
        const int per_block = CA_THREADS / (P.tl * P.slots);
        int64_t grid = (n * P.units_per_row + per_block - 1) / per_block;
        const int64_t cap = sm_count() * (pass ? 16 : 64);
        if (grid > cap) grid = cap;
        e = launch_train(k_coded_attend<T, VE, G, U>, grid, CA_THREADS, 0, s, P);
    }
    if (P.split && e == cudaSuccess) e = launch_train(k_coded_attend_join<T>, sm_count() * 8, 256, 0, s, P);
    return e;
}

template <typename T> static cudaError_t coded_group(const CodedAttend& P, cudaStream_t s) {
    const int group = P.a.q_heads / P.a.kv_heads;
    // query heads that share a key/value head are taken together; what a lane holds of them stays within its registers
    if (group % 4 == 0) return run_coded<T, 8, 4, 4>(P, s);
    if (group % 2 == 0) return run_coded<T, 8, 2, 4>(P, s);
    return run_coded<T, 16, 1, 4>(P, s);
}

cudaError_t launch_coded_attention(const CodedAttention& a, void* workspace, cudaStream_t s) {
    CodedAttend P{};
    P.a = a;
    const CodedAttendLayout l = coded_attend_layout(a.edge_bound, a.q_heads, a.head_dim);
    char* ws = (char*)workspace;
    P.words = (int32_t*)(ws + l.words);
    P.items = (int2*)(ws + l.items);
    P.longs = (int4*)(ws + l.longs);
    P.partial = (float*)(ws + l.partial);
    P.split = (a.max_row == 0 || a.max_row > CA_LONG) && a.edge_bound > CA_LONG;
    const int size = a.dtype == GS_BF16 ? 2 : 4, ve = 16 / size;
    auto on16 = [&](const HeadView& v) { return (uintptr_t)v.data % 16 == 0 && (v.row_stride * size) % 16 == 0 && (v.head_stride * size) % 16 == 0; };
    P.wide = a.head_dim % ve == 0 && on16(a.q) && on16(a.out);
    if (P.split) {
        const cudaError_t e = cudaMemsetAsync(P.words, 0, 8, s);
        if (e != cudaSuccess) return e;
    }
    return a.dtype == GS_BF16 ? coded_group<bf16>(P, s) : coded_group<float>(P, s);
}

}  // namespace gs
