// Root-mean-square norm of rows, with the addition of a residual before it, forward and backward.
//
//   h = x + r, rounded to its type (what is kept is what is normalised);  v = 1 / sqrt(mean h^2 + eps);  y = w h v
//   g = w dy;  dx = dr = dh + v g - h v^3 mean(g h);  dw = sum over rows of dy h v
// Sums in 32 bits, one rounding per result.  v is recomputed by the backward pass, which has the row in hand anyway.
//
// Every element is read and written once, and that is the time: a row is held in registers by a group of lanes (rows of up to 32
// pieces) or by a block, in pieces of 16 bytes.  Rows of odd widths begin anywhere within a piece: a block then takes the rows that
// begin at one place of it (every 4th f32 row of 1,433, say), so that its threads keep their columns, and only the pieces at a
// row's ends go one element at a time.  Arrays whose rows do not begin alike go one element at a time altogether.
// Measured with a residual (reads and writes of both sides, of a copy's 6.56 TB/s): 2.03 M x 64 bf16 forward 164 us = 0.97, backward 184 = 0.86;
// 30,000 x 2,000 f32 161 and 161 = 0.91; 100,000 x 513 f32 (rows that begin anywhere) 170 and 239 = 0.74 and 0.52; 4,096 x 1,433 13 and 23 cold: the
// latency of a row's sums in a block (two rows of a block in flight: 15 and 31).  300,000 x 33 bf16 76 and 115 = 0.16 and 0.10: a
// row is five pieces on eight lanes, and one or two of them are ends, eight elements one at a time: issue slots 81 % and 66 %.
// Forms of the backward pass that spill (bytes loaded): f32 rows of more than 4,096 columns 108 to 152, odd widths of up to 512 columns 32 to
// 80, one element at a time 56 to 192; the others 0 to 40.
// dw: a group keeps its columns' sums over NM_SUMMED rows and joins them to those before in 64 bits (2.03 M x 128: 3.8e-7 off without
// that, 1.2e-7 with it, for 353 -> 355 us); a block with a row to itself keeps them over all of its rows.  Blocks leave theirs in the
// workspace, and a second kernel adds them in order, in 64 bits.
// Results in 8 bits: the largest magnitude of a group of columns is found among the lanes that hold it, by shuffles where the
// group's pieces are a power of two and by integer maxima in shared memory otherwise.
#include <type_traits>

#include "gs_codes.cuh"
#include "gs_device.cuh"
#include "gs_train.h"

namespace gs {

constexpr int NM_SUMMED = 32;        // rows that a lane adds dw of in 32 bits before the sum is joined to the others in 64
constexpr int NM_THREADS = 256;      // of the kernels whose rows are held by lanes of a warp

__device__ __forceinline__ int norm_rows(const Count& c) {
    if (!c.d_n) return c.bound;
    const int n = __ldg(c.d_n);
    return n < 0 ? 0 : (n > c.bound ? c.bound : n);
}

// Elements in pairs for the packed 32-bit operations; rows that go one element at a time use plain floats.
template <int VE> using El = std::conditional_t<VE == 1, float, f32x2>;
template <int VE> constexpr int EL = VE == 1 ? 1 : VE / 2;
__device__ __forceinline__ float v_mul(float a, float b) { return a * b; }
__device__ __forceinline__ f32x2 v_mul(f32x2 a, f32x2 b) { return mul2(a, b); }
__device__ __forceinline__ float v_fma(float a, float b, float c) { return fmaf(a, b, c); }
__device__ __forceinline__ f32x2 v_fma(f32x2 a, f32x2 b, f32x2 c) { return fma2(a, b, c); }
__device__ __forceinline__ float v_add(float a, float b) { return a + b; }
__device__ __forceinline__ f32x2 v_add(f32x2 a, f32x2 b) { return add2(a, b); }
__device__ __forceinline__ float v_sum(float a) { return a; }
__device__ __forceinline__ float v_sum(f32x2 a) {
    float x, y;
    split(a, x, y);
    return x + y;
}
template <int VE> __device__ __forceinline__ El<VE> v_all(float x) {
    if constexpr (VE == 1) return x;
    else return pair(x, x);
}
template <int VE> __device__ __forceinline__ void v_pack(const float (&x)[VE], El<VE> (&y)[EL<VE>]) {
    if constexpr (VE == 1) {
        y[0] = x[0];
    } else {
#pragma unroll
        for (int i = 0; i < VE / 2; ++i) y[i] = pair(x[2 * i], x[2 * i + 1]);
    }
}
template <int VE> __device__ __forceinline__ void v_unpack(const El<VE> (&y)[EL<VE>], float (&x)[VE]) {
    if constexpr (VE == 1) {
        x[0] = y[0];
    } else {
#pragma unroll
        for (int i = 0; i < VE / 2; ++i) split(y[i], x[2 * i], x[2 * i + 1]);
    }
}

// Where a block's rows begin: row v of its class is row v * period + cls, its first element `phase` elements behind the begin of a
// piece (0 without EDGE).
struct RowClass {
    int cls, phase, n;               // n: rows of the class
    int64_t blk, blks;
};
template <int VE, bool EDGE> __device__ __forceinline__ RowClass row_class(const RmsNorm& P, int n) {
    if constexpr (!EDGE) return RowClass{0, 0, n, (int64_t)blockIdx.x, (int64_t)gridDim.x};
    const int cls = (int)(blockIdx.x % P.period);
    return RowClass{cls, (int)((P.phase + (int64_t)cls * P.x_ld) & (VE - 1)), n > cls ? (n - cls + P.period - 1) / P.period : 0, (int64_t)(blockIdx.x / P.period),
                    (int64_t)(gridDim.x / P.period)};
}

template <typename T, int VE, int NV, bool EDGE> struct RowPart {
    Raw<T, VE> r[NV];
    __device__ __forceinline__ void load(const T* row, int t, int width, int phase, int dim, bool on) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (t + j * width) * VE - phase;
            if (EDGE && on && c < dim && (c < 0 || c + VE > dim)) {
                float x[VE];
#pragma unroll
                for (int i = 0; i < VE; ++i) x[i] = c + i >= 0 && c + i < dim ? to_f32(row[c + i]) : 0.f;
                set(j, x);
            } else {
                r[j] = on && c < dim ? load_raw_stream<T, VE>(row + c) : zero_raw<T, VE>();
            }
        }
    }
    __device__ __forceinline__ void get(int j, float (&x)[VE]) const { unpack<T, VE>(r[j], x); }
    __device__ __forceinline__ void pairs(int j, El<VE> (&y)[EL<VE>]) const {
        float x[VE];
        get(j, x);
        v_pack<VE>(x, y);
    }
    __device__ __forceinline__ void set_pairs(int j, const El<VE> (&y)[EL<VE>]) {
        float x[VE];
        v_unpack<VE>(y, x);
        set(j, x);
    }
    __device__ __forceinline__ void set(int j, const float (&x)[VE]) {
        if constexpr (sizeof(T) == 4) {
            if constexpr (VE == 4) r[j].w = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
            else r[j].w = __float_as_uint(x[0]);
        } else if constexpr (VE == 8) {
            r[j].w = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
        } else {
            r[j].w = (uint16_t)pack_bf16(x[0], 0.f);
        }
    }
    __device__ __forceinline__ void store(T* row, int t, int width, int phase, int dim) const {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (t + j * width) * VE - phase;
            if (EDGE && c < dim && (c < 0 || c + VE > dim)) {
                float x[VE];
                get(j, x);
#pragma unroll
                for (int i = 0; i < VE; ++i)
                    if (c + i >= 0 && c + i < dim) row[c + i] = from_f32<T>(x[i]);
            } else if (c < dim) {
                *reinterpret_cast<typename Raw<T, VE>::word*>(row + c) = r[j].w;
            }
        }
    }
};

template <int VE, int NV> __device__ __forceinline__ void load_weight(const RmsNorm& P, int t, int width, int phase, El<VE> (&w)[NV][EL<VE>]) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        float x[VE];
#pragma unroll
        for (int i = 0; i < VE; ++i) {
            const int c = (t + j * width) * VE + i - phase;
            x[i] = 1.f;
            if (P.weight && c >= 0 && c < P.dim) x[i] = P.weight_dtype == GS_BF16 ? to_f32(static_cast<const bf16*>(P.weight)[c]) : static_cast<const float*>(P.weight)[c];
        }
        v_pack<VE>(x, w[j]);
    }
}

// Sums over the threads of a row: a group of `width` lanes, or (BLOCK) all of the block.
template <bool BLOCK, int N> __device__ __forceinline__ void row_sum(float (&x)[N], int width) {
    for (int o = 1; o < (BLOCK ? 32 : width); o <<= 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] += __shfl_xor_sync(FULL, x[i], o);
    }
    if constexpr (BLOCK) {
        __shared__ float s[N][32];
        const int warp = threadIdx.x >> 5, warps = (blockDim.x + 31) >> 5;
        __syncthreads();
        if ((threadIdx.x & 31) == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) s[i][warp] = x[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            x[i] = 0.f;
            for (int w = 0; w < warps; ++w) x[i] += s[i][w];
        }
    }
}

// The row's result in 8 bits.  y: this thread's pieces.
template <int VE, int NV, bool BLOCK>
__device__ __forceinline__ void store_codes(const RmsNorm& P, int64_t row, bool on, int t, int width, const float (&y)[NV * VE], uint32_t* tops) {
    const CodedView& C = P.coded;
    const int hd = C.head_dim;
    uint32_t top[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        float m = 0.f;                                       // NaN is passed over
#pragma unroll
        for (int i = 0; i < VE; ++i) m = fmaxf(m, fabsf(y[j * VE + i]));
        top[j] = __float_as_uint(m);
        if (m == INFINITY) {
            top[j] = 0;
#pragma unroll
            for (int i = 0; i < VE; ++i) top[j] = max(top[j], finite_magnitude(y[j * VE + i]));
        }
    }
    const int per = hd / VE;                                 // pieces of a group of columns (VE > 1: whole ones)
    const bool shuffled = !BLOCK && per <= width && (per & (per - 1)) == 0;
    if (shuffled) {
        for (int o = 1; o < per; o <<= 1) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                top[j] = max(top[j], __shfl_xor_sync(FULL, top[j], o));
            }
        }
    } else {
        if constexpr (BLOCK) {
            __syncthreads();
            for (int h = threadIdx.x; h < C.heads; h += blockDim.x) tops[h] = 0;
            __syncthreads();
        } else {
            __syncwarp();
            for (int h = t; h < C.heads; h += width) tops[h] = 0;
            __syncwarp();
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (t + j * width) * VE;
            if (on && c < P.dim && top[j]) atomicMax(tops + c / hd, top[j]);
        }
        if constexpr (BLOCK) __syncthreads();
        else __syncwarp();
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (t + j * width) * VE;
            top[j] = c < P.dim ? tops[c / hd] : 0u;
        }
    }
    if (!on) return;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = (t + j * width) * VE;
        if (c >= P.dim) continue;
        const int h = c / hd, in = c - h * hd;
        const uint32_t b = scale_byte(top[j]);
        float x[VE];
#pragma unroll
        for (int i = 0; i < VE; ++i) x[i] = y[j * VE + i];
        uint8_t* to = C.codes + row * C.row_stride + (int64_t)h * C.pitch + in;
        *reinterpret_cast<typename CodeWord<VE>::type*>(to) = encode<VE>(x, unscale_of(b));
        if (in == 0) C.scales[row * C.scale_stride + h] = (uint8_t)b;
        if (in + VE == hd)
            for (int i = VE; in + i < C.pitch; ++i) to[i] = 0;
    }
}

// U rows of each group are in flight.
template <typename T, int VE, int NV, int U, bool BLOCK, bool EDGE, bool CODED>
__global__ void __launch_bounds__(BLOCK ? 512 : NM_THREADS) k_norm_forward(const __grid_constant__ RmsNorm P) {
    constexpr int E = VE * NV;
    extern __shared__ uint32_t norm_tops[];                  // CODED: per row held
    chain_wait();
    const int n = norm_rows(P.n), D = P.dim;
    const int width = BLOCK ? (int)blockDim.x : P.tl, t = BLOCK ? (int)threadIdx.x : (int)threadIdx.x & (P.tl - 1), own = BLOCK ? 0 : threadIdx.x / width;
    const int per_block = BLOCK ? 1 : NM_THREADS / width;
    uint32_t* tops = CODED ? norm_tops + own * P.coded.heads : nullptr;
    const RowClass C = row_class<VE, EDGE>(P, n);
    El<VE> w[NV][EL<VE>];
    RowPart<T, VE, NV, EDGE> x[U], r[U], xn[BLOCK ? U : 1], rn[BLOCK ? U : 1];
    const int64_t step = C.blks * per_block * U;
    int64_t base = C.blk * per_block * U;
    auto row_at = [&](int64_t base, int u) { return EDGE ? (base + u * per_block + own) * P.period + C.cls : base + u * per_block + own; };
    auto load = [&](int64_t base, auto& x, auto& r) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = row_at(base, u);
            const bool on = base < C.n && row < n;
            x[u].load((const T*)P.x + row * P.x_ld, t, width, C.phase, D, on);
            if (P.residual) r[u].load((const T*)P.residual + row * P.residual_ld, t, width, C.phase, D, on);
        }
    };
    load(base, x, r);
    load_weight<VE, NV>(P, t, width, C.phase, w);
    for (; base < C.n; base += step) {
        if constexpr (BLOCK) load(base + step, xn, rn);      // few rows are held at a time: the next is on its way
        float sum[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            El<VE> q = v_all<VE>(0.f);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                El<VE> a[EL<VE>];
                x[u].pairs(j, a);
                if (P.residual) {
                    El<VE> b[EL<VE>];
                    r[u].pairs(j, b);
#pragma unroll
                    for (int i = 0; i < EL<VE>; ++i) a[i] = v_add(a[i], b[i]);
                    x[u].set_pairs(j, a);                    // rounded: what is normalised is what is kept
                    x[u].pairs(j, a);
                }
#pragma unroll
                for (int i = 0; i < EL<VE>; ++i) q = v_fma(a[i], a[i], q);
            }
            sum[u] = v_sum(q);
        }
        row_sum<BLOCK, U>(sum, width);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = row_at(base, u);
            const bool on = row < n;
            const El<VE> inv = v_all<VE>(__frsqrt_rn(fmaf(sum[u], P.inv_dim, P.eps)));
            if (on && P.hidden) x[u].store((T*)P.hidden + row * P.hidden_ld, t, width, C.phase, D);
            float y[E];
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                El<VE> a[EL<VE>];
                x[u].pairs(j, a);
#pragma unroll
                for (int i = 0; i < EL<VE>; ++i) a[i] = v_mul(v_mul(a[i], inv), w[j][i]);
                if constexpr (CODED) {
                    float z[VE];
                    v_unpack<VE>(a, z);
#pragma unroll
                    for (int i = 0; i < VE; ++i) y[j * VE + i] = z[i];
                } else {
                    r[u].set_pairs(j, a);
                }
            }
            if constexpr (CODED) store_codes<VE, NV, BLOCK>(P, row, on, t, width, y, tops);
            else if (on) r[u].store((T*)P.out + row * P.out_ld, t, width, C.phase, D);
        }
        if constexpr (BLOCK) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                x[u] = xn[u];
                r[u] = rn[u];
            }
        } else {
            load(base + step, x, r);
        }
    }
}

// dw_part: [blocks][dim] sums of the rows a block took.
template <typename T, int VE, int NV, int U, bool BLOCK, bool EDGE>
__global__ void __launch_bounds__(BLOCK ? 512 : NM_THREADS, BLOCK ? 1 : (VE * NV <= 8 ? 3 : 2)) k_norm_backward(const __grid_constant__ RmsNorm P, float* dw_part) {
    extern __shared__ double norm_dw[];                      // groups: [warps][dim], each lane its columns
    chain_wait();
    const int n = norm_rows(P.n), D = P.dim;
    const int width = BLOCK ? (int)blockDim.x : P.tl, t = BLOCK ? (int)threadIdx.x : (int)threadIdx.x & (P.tl - 1), own = BLOCK ? 0 : threadIdx.x / width;
    const int per_block = BLOCK ? 1 : NM_THREADS / width;
    const RowClass C = row_class<VE, EDGE>(P, n);
    El<VE> w[NV][EL<VE>], dw[NV][EL<VE>];
    RowPart<T, VE, NV, EDGE> h[U], dy[U], dh[U];             // the rows that are worked on next
    const int64_t step = C.blks * per_block * U;
    auto row_at = [&](int64_t base, int u) { return EDGE ? (base + u * per_block + own) * P.period + C.cls : base + u * per_block + own; };
    auto load = [&](int64_t base) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = row_at(base, u);
            const bool on = base < C.n && row < n;
            h[u].load((const T*)P.x + row * P.x_ld, t, width, C.phase, D, on);
            dy[u].load((const T*)P.dout + row * P.dout_ld, t, width, C.phase, D, on);
            if (P.residual) dh[u].load((const T*)P.residual + row * P.residual_ld, t, width, C.phase, D, on);
        }
    };
    load(C.blk * per_block * U);
    load_weight<VE, NV>(P, t, width, C.phase, w);
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < EL<VE>; ++i) dw[j][i] = v_all<VE>(0.f);
    bool left = false;
    // adds the columns' sums to what is kept of them: those of a warp's groups, in 64 bits, to its lanes' own in shared memory; a block's
    // rows are few, and its threads put their sums into the workspace once
    auto leave = [&]() {
        int at = t;
        asm volatile("" : "+r"(at));                         // addresses are made here, not kept over the rows
        float* part = dw_part + (int64_t)blockIdx.x * D;
        double* mine = norm_dw + (threadIdx.x >> 5) * D;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float x[VE];
            v_unpack<VE>(dw[j], x);
#pragma unroll
            for (int i = 0; i < EL<VE>; ++i) dw[j][i] = v_all<VE>(0.f);
            if constexpr (!BLOCK) {
                for (int o = width; o < 32; o <<= 1) {       // the groups of a warp
#pragma unroll
                    for (int i = 0; i < VE; ++i) x[i] += __shfl_xor_sync(FULL, x[i], o);
                }
                if ((int)(threadIdx.x & 31) >= width) continue;
            }
            const int c0 = (at + j * width) * VE - C.phase;
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                const int c = c0 + i;
                if (c < 0 || c >= D) continue;
                if constexpr (BLOCK) part[c] = x[i];
                else mine[c] = (left ? mine[c] : 0.0) + x[i];
            }
        }
        left = true;
    };
    int64_t base = C.blk * per_block * U;
    auto rows = [&]() {
        RowPart<T, VE, NV, EDGE> hc[U], dyc[U], dhc[U];
        float sum[2 * U];                                    // sum h^2, sum g h
#pragma unroll
        for (int u = 0; u < U; ++u) {
            hc[u] = h[u];
            dyc[u] = dy[u];
            dhc[u] = dh[u];
            El<VE> hh = v_all<VE>(0.f), gh = v_all<VE>(0.f);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                El<VE> a[EL<VE>], b[EL<VE>];
                hc[u].pairs(j, a);
                dyc[u].pairs(j, b);
#pragma unroll
                for (int i = 0; i < EL<VE>; ++i) {
                    hh = v_fma(a[i], a[i], hh);
                    gh = v_fma(v_mul(b[i], w[j][i]), a[i], gh);
                }
            }
            sum[2 * u] = v_sum(hh);
            sum[2 * u + 1] = v_sum(gh);
        }
        load(base + step);                                   // on their way while these are summed and written
        row_sum<BLOCK, 2 * U>(sum, width);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = row_at(base, u);
            if (row >= n) continue;
            const float v = __frsqrt_rn(fmaf(sum[2 * u], P.inv_dim, P.eps));
            const El<VE> inv = v_all<VE>(v), mean = v_all<VE>(-(sum[2 * u + 1] * P.inv_dim * v * v * v));
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                El<VE> a[EL<VE>], b[EL<VE>], x[EL<VE>];
                hc[u].pairs(j, a);
                dyc[u].pairs(j, b);
                if (P.residual) {
                    dhc[u].pairs(j, x);
                } else {
#pragma unroll
                    for (int i = 0; i < EL<VE>; ++i) x[i] = v_all<VE>(0.f);
                }
#pragma unroll
                for (int i = 0; i < EL<VE>; ++i) {
                    dw[j][i] = v_fma(b[i], v_mul(a[i], inv), dw[j][i]);
                    // the two terms of the norm's own gradient, which may cancel, before what arrives beside it
                    x[i] = v_add(v_fma(a[i], mean, v_mul(v_mul(b[i], w[j][i]), inv)), x[i]);
                }
                hc[u].set_pairs(j, x);
            }
            hc[u].store((T*)P.out + row * P.out_ld, t, width, C.phase, D);
        }
    };
    if constexpr (BLOCK) {
        for (; base < C.n; base += step) rows();
    } else {
        while (base < C.n) {
            for (int i = 0; i < NM_SUMMED / U && base < C.n; ++i, base += step) rows();
            if (base < C.n && P.dweight) leave();
        }
    }
    if (!P.dweight) return;
    leave();
    if constexpr (!BLOCK) {
        __syncthreads();
        for (int c = threadIdx.x; c < D; c += NM_THREADS) {
            double s = 0.0;
            for (int i = 0; i < NM_THREADS / 32; ++i) s += norm_dw[i * D + c];
            dw_part[(int64_t)blockIdx.x * D + c] = (float)s;
        }
    }
}

// dw = the blocks' sums, added in order: 32 columns per block, its warps over contiguous shares of the blocks, U on their way together, then
// a column to a warp.
__global__ void __launch_bounds__(1024) k_norm_dweight(const float* __restrict__ part, int parts, int dim, void* dweight, gs_dtype dtype) {
    constexpr int U = 16;
    __shared__ double s[32][33];
    chain_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per = (parts + 31) / 32;
    for (int c0 = blockIdx.x * 32; c0 < dim; c0 += gridDim.x * 32) {
        const int c = c0 + lane, p1 = (warp + 1) * per < parts ? (warp + 1) * per : parts;
        double sum = 0.0;
        for (int p = warp * per; p < p1; p += U) {
            float x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = c < dim && p + u < p1 ? __ldcg(part + (int64_t)(p + u) * dim + c) : 0.f;
            double y[U / 2];
#pragma unroll
            for (int u = 0; u < U / 2; ++u) y[u] = (double)x[2 * u] + (double)x[2 * u + 1];
#pragma unroll
            for (int n = U / 4; n; n /= 2)
#pragma unroll
                for (int u = 0; u < n; ++u) y[u] += y[u + n];
            sum += y[0];
        }
        __syncthreads();
        s[warp][lane] = sum;
        __syncthreads();
        sum = s[lane][warp];
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(FULL, sum, o);
        if (lane == 0 && c0 + warp < dim) {
            if (dtype == GS_BF16) static_cast<bf16*>(dweight)[c0 + warp] = __float2bfloat16_rn((float)sum);
            else static_cast<float*>(dweight)[c0 + warp] = (float)sum;
        }
    }
}

// ---------------------------------------------------------------- launches
// Blocks of the backward pass, at most: what the workspace holds sums for.
static int64_t norm_parts(int64_t rows) {
    const int64_t most = sm_count() * 8;
    return rows < most ? (rows < 1 ? 1 : rows) : most;
}
size_t norm_workspace(int64_t rows, int32_t dim) { return align_up((size_t)norm_parts(rows) * dim * 4, 256); }

// How the rows of several arrays lie in memory: the elements of an access (whole pieces, or one), and, for whole pieces, after how
// many rows they begin at the same place of a piece again.
struct RowLayout {
    int ve, period, phase;
    bool edge;
    void add(const void* p, int64_t ld, int size, int64_t rows) {
        if (!p || ve == 1) return;
        const int at = (int)((uintptr_t)p / size % ve), step = rows > 1 ? (int)(ld % ve) : 0;
        if (phase < 0) {
            phase = at;
            turn = step;
        } else if (at != phase || step != turn) {
            ve = 1;
        }
    }
    int turn;
    void finish(int dim) {
        period = 1;
        if (ve > 1)
            while (period * turn % ve) period *= 2;
        edge = ve > 1 && (phase || turn || dim % ve);
        if (edge && (dim + 2 * ve - 2) / ve > NORM_MAX_DIM / ve) single();   // a piece more than a block holds
    }
    void single() {
        ve = period = 1;
        phase = turn = 0;
        edge = false;
    }
};

// A row's elements per thread: one or two pieces by lanes of a warp, 8 or 16 elements by a block.
template <typename T, int V, bool EDGE, typename F> static cudaError_t norm_width(const RmsNorm& P, F run) {
    constexpr int FEW = 1, MORE = V > 1 ? 2 : 4, HALF = 8 / V, MOST = 16 / V;
    const int pieces = (P.dim + (EDGE ? V - 1 : 0) + V - 1) / V;
    auto with = [&](auto num, auto block) {
        const int threads = (pieces + (int)num - 1) / (int)num;
        int tl = 1;
        if (block) tl = (threads + 31) / 32 * 32;
        else while (tl < threads) tl *= 2;
        return run(T(), std::integral_constant<int, V>(), num, block, std::integral_constant<bool, EDGE>(), tl);
    };
    if (pieces <= 32 * FEW) return with(std::integral_constant<int, FEW>(), std::false_type());
    if (pieces <= 32 * MORE) return with(std::integral_constant<int, MORE>(), std::false_type());
    if (pieces <= 512 * HALF) return with(std::integral_constant<int, HALF>(), std::true_type());
    return with(std::integral_constant<int, MOST>(), std::true_type());
}
template <typename F> static cudaError_t norm_shape(const RmsNorm& P, const RowLayout& l, F run) {
    if (P.dtype == GS_BF16) {
        if (l.ve == 1) return norm_width<bf16, 1, false>(P, run);
        return l.edge ? norm_width<bf16, 8, true>(P, run) : norm_width<bf16, 8, false>(P, run);
    }
    if (l.ve == 1) return norm_width<float, 1, false>(P, run);
    return l.edge ? norm_width<float, 4, true>(P, run) : norm_width<float, 4, false>(P, run);
}

cudaError_t launch_norm_forward(const RmsNorm& p, bool coded, cudaStream_t s) {
    const int size = p.dtype == GS_BF16 ? 2 : 4;
    RowLayout l{16 / size, 1, -1, false, 0};
    const int64_t rows = p.n.bound;
    l.add(p.x, p.x_ld, size, rows);
    l.add(p.residual, p.residual_ld, size, rows);
    l.add(p.hidden, p.hidden_ld, size, rows);
    if (!coded) l.add(p.out, p.out_ld, size, rows);
    l.finish(p.dim);
    // columns of a piece share a scale; fewer blocks than places where rows begin (a capped grid): one element at a time
    if ((coded && (l.edge || p.coded.head_dim % l.ve)) || limit_grid(l.period) < l.period) l.single();
    return norm_shape(p, l, [&](auto type, auto vec, auto num, auto block, auto edge, int tl) {
        using T = decltype(type);
        constexpr int VE = vec, NV = num;
        constexpr bool B = block, EDGE = edge;
        constexpr int U = B ? 1 : 2;
        RmsNorm P = p;
        P.tl = tl;
        P.period = l.period;
        P.inv_dim = 1.f / (float)p.dim;
        P.phase = l.phase;
        const int threads = B ? tl : NM_THREADS, held = B ? 1 : NM_THREADS / tl;
        auto run = [&](auto kernel, size_t smem, std::atomic<uint64_t>& known) {
            int64_t grid = (rows + held * U - 1) / (held * U);
            const int64_t cap = B ? sm_count() * resident_blocks(kernel, threads, smem, known) : sm_count() * 64;
            grid = (grid + l.period - 1) / l.period * l.period;
            grid = limit_grid(grid > cap ? cap : grid) / l.period * l.period;
            return launch_train(kernel, grid, threads, smem, s, P);
        };
        static std::atomic<uint64_t> known{0}, known_coded{0};
        if constexpr (!EDGE) {
            if (coded) return run(k_norm_forward<T, VE, NV, U, B, false, true>, (size_t)held * p.coded.heads * 4, known_coded);
        }
        return run(k_norm_forward<T, VE, NV, U, B, EDGE, false>, 0, known);
    });
}

cudaError_t launch_norm_backward(const RmsNorm& p, void* workspace, cudaStream_t s) {
    const int size = p.dtype == GS_BF16 ? 2 : 4;
    RowLayout l{16 / size, 1, -1, false, 0};
    const int64_t rows = p.n.bound, most = norm_parts(rows);
    l.add(p.x, p.x_ld, size, rows);
    l.add(p.residual, p.residual_ld, size, rows);
    l.add(p.dout, p.dout_ld, size, rows);
    l.add(p.out, p.out_ld, size, rows);
    l.finish(p.dim);
    if (limit_grid(l.period) < l.period || most < l.period) l.single();
    return norm_shape(p, l, [&](auto type, auto vec, auto num, auto block, auto edge, int tl) {
        using T = decltype(type);
        constexpr int VE = vec, NV = num;
        constexpr bool B = block, EDGE = edge;
        constexpr int U = B || VE * NV > 4 ? 1 : 2;
        RmsNorm P = p;
        P.tl = tl;
        P.period = l.period;
        P.inv_dim = 1.f / (float)p.dim;
        P.phase = l.phase;
        const int threads = B ? tl : NM_THREADS, held = (B ? 1 : NM_THREADS / tl) * U;
        const size_t smem = B ? 0 : (size_t)(NM_THREADS / 32) * p.dim * sizeof(double);
        // as many blocks as are resident: each leaves its columns' sums once
        static std::atomic<uint64_t> known{0};
        auto kernel = k_norm_backward<T, VE, NV, U, B, EDGE>;
        int64_t grid = (rows + held - 1) / held, cap = sm_count() * resident_blocks(kernel, threads, smem, known);
        cap = cap < most ? cap : most;
        grid = (grid + l.period - 1) / l.period * l.period;
        grid = limit_grid(grid > cap ? cap : grid) / l.period * l.period;
        float* part = (float*)workspace;
        cudaError_t e = launch_train(kernel, grid, threads, smem, s, P, part);
        if (e == cudaSuccess && p.dweight) e = launch_train(k_norm_dweight, (p.dim + 31) / 32, 1024, 0, s, (const float*)part, (int)grid, (int)p.dim, p.dweight, p.weight_dtype);
        return e;
    });
}

}  // namespace gs
