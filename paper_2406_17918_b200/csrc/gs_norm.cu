// Root-mean-square norm of rows, with the addition of a residual before it, forward and backward.
//
//   h = x + r, rounded to its type (what is kept is what is normalised);  v = 1 / sqrt(mean h^2 + eps);  y = w h v
//   g = w dy;  dx = dr = dh + v g - h v^3 mean(g h);  dw = sum over rows of dy h v
// Sums in 32 bits, one rounding per result.  v is recomputed by the backward pass, which has the row in hand anyway.
//
// Every element is read and written once, and that is the time: a row is held in registers by a group of lanes (rows of up to 32
// pieces) or by a block, in pieces of 16 bytes where bases, pitches and the width allow, one element at a time otherwise.  dw: a
// group keeps its columns' sums over all of its rows; blocks leave theirs in the workspace and a second kernel adds them in order.
// Results in 8 bits: the largest magnitude of a group of columns is found among the lanes that hold it, by shuffles where the
// group's pieces are a power of two and by integer maxima in shared memory otherwise.
#include "gs_codes.cuh"
#include "gs_device.cuh"
#include "gs_train.h"

namespace gs {

constexpr int NM_THREADS = 256;      // of the kernels whose rows are held by lanes of a warp

__device__ __forceinline__ int norm_rows(const Count& c) {
    if (!c.d_n) return c.bound;
    const int n = __ldg(c.d_n);
    return n < 0 ? 0 : (n > c.bound ? c.bound : n);
}

template <typename T, int VE, int NV> struct RowPart {
    Raw<T, VE> r[NV];
    __device__ __forceinline__ void load(const T* row, int t, int width, int dim, bool on) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (t + j * width) * VE;
            r[j] = on && c < dim ? load_raw_stream<T, VE>(row + c) : zero_raw<T, VE>();
        }
    }
    __device__ __forceinline__ void get(int j, float (&x)[VE]) const { unpack<T, VE>(r[j], x); }
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
    __device__ __forceinline__ void store(T* row, int t, int width, int dim) const {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (t + j * width) * VE;
            if (c < dim) *reinterpret_cast<typename Raw<T, VE>::word*>(row + c) = r[j].w;
        }
    }
};

template <int VE, int NV> __device__ __forceinline__ void load_weight(const RmsNorm& P, int t, int width, float (&w)[NV * VE]) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < VE; ++i) {
            const int c = (t + j * width) * VE + i;
            float x = 1.f;
            if (P.weight && c < P.dim) x = P.weight_dtype == GS_BF16 ? to_f32(static_cast<const bf16*>(P.weight)[c]) : static_cast<const float*>(P.weight)[c];
            w[j * VE + i] = x;
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
        top[j] = 0;
#pragma unroll
        for (int i = 0; i < VE; ++i) {
            const uint32_t m = finite_magnitude(y[j * VE + i]);
            top[j] = m > top[j] ? m : top[j];
        }
    }
    const int per = hd / VE;                                 // pieces of a group of columns (VE > 1: whole ones)
    const bool shuffled = !BLOCK && per <= width && (per & (per - 1)) == 0;
    if (shuffled) {
        for (int o = 1; o < per; o <<= 1) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const uint32_t m = __shfl_xor_sync(FULL, top[j], o);
                top[j] = m > top[j] ? m : top[j];
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
template <typename T, int VE, int NV, int U, bool BLOCK, bool CODED>
__global__ void __launch_bounds__(BLOCK ? 512 : NM_THREADS) k_norm_forward(const __grid_constant__ RmsNorm P) {
    constexpr int E = VE * NV;
    extern __shared__ uint32_t norm_tops[];                  // CODED: per row held
    chain_wait();
    const int n = norm_rows(P.n), D = P.dim;
    const int width = BLOCK ? (int)blockDim.x : P.tl, t = BLOCK ? (int)threadIdx.x : (int)threadIdx.x & (P.tl - 1), own = BLOCK ? 0 : threadIdx.x / width;
    const int per_block = BLOCK ? 1 : NM_THREADS / width;
    uint32_t* tops = CODED ? norm_tops + own * P.coded.heads : nullptr;
    float w[E];
    load_weight<VE, NV>(P, t, width, w);
    for (int64_t base = (int64_t)blockIdx.x * per_block * U; base < n; base += (int64_t)gridDim.x * per_block * U) {
        RowPart<T, VE, NV> x[U], r[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = base + u * per_block + own;
            x[u].load((const T*)P.x + row * P.x_ld, t, width, D, row < n);
            if (P.residual) r[u].load((const T*)P.residual + row * P.residual_ld, t, width, D, row < n);
        }
        float sum[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            sum[u] = 0.f;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float a[VE];
                x[u].get(j, a);
                if (P.residual) {
                    float b[VE];
                    r[u].get(j, b);
#pragma unroll
                    for (int i = 0; i < VE; ++i) a[i] += b[i];
                    x[u].set(j, a);                          // rounded: what is normalised is what is kept
                    x[u].get(j, a);
                }
#pragma unroll
                for (int i = 0; i < VE; ++i) sum[u] = fmaf(a[i], a[i], sum[u]);
            }
        }
        row_sum<BLOCK, U>(sum, width);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = base + u * per_block + own;
            const bool on = row < n;
            const float inv = __frsqrt_rn(sum[u] / (float)D + P.eps);
            if (on && P.hidden) x[u].store((T*)P.hidden + row * P.hidden_ld, t, width, D);
            float y[E];
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float a[VE];
                x[u].get(j, a);
#pragma unroll
                for (int i = 0; i < VE; ++i) y[j * VE + i] = a[i] * inv * w[j * VE + i];
            }
            if constexpr (CODED) {
                store_codes<VE, NV, BLOCK>(P, row, on, t, width, y, tops);
            } else if (on) {
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    float a[VE];
#pragma unroll
                    for (int i = 0; i < VE; ++i) a[i] = y[j * VE + i];
                    r[u].set(j, a);
                }
                r[u].store((T*)P.out + row * P.out_ld, t, width, D);
            }
        }
    }
}

// dw_part: [blocks][dim] sums of the rows a block took.
template <typename T, int VE, int NV, int U, bool BLOCK>
__global__ void __launch_bounds__(BLOCK ? 512 : NM_THREADS) k_norm_backward(const __grid_constant__ RmsNorm P, float* dw_part) {
    constexpr int E = VE * NV;
    extern __shared__ float norm_dw[];                       // groups: [warps][dim]
    chain_wait();
    const int n = norm_rows(P.n), D = P.dim;
    const int width = BLOCK ? (int)blockDim.x : P.tl, t = BLOCK ? (int)threadIdx.x : (int)threadIdx.x & (P.tl - 1), own = BLOCK ? 0 : threadIdx.x / width;
    const int per_block = BLOCK ? 1 : NM_THREADS / width;
    float w[E], dw[E];
    load_weight<VE, NV>(P, t, width, w);
#pragma unroll
    for (int i = 0; i < E; ++i) dw[i] = 0.f;
    for (int64_t base = (int64_t)blockIdx.x * per_block * U; base < n; base += (int64_t)gridDim.x * per_block * U) {
        RowPart<T, VE, NV> h[U], dy[U], dh[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = base + u * per_block + own;
            h[u].load((const T*)P.x + row * P.x_ld, t, width, D, row < n);
            dy[u].load((const T*)P.dout + row * P.dout_ld, t, width, D, row < n);
            if (P.residual) dh[u].load((const T*)P.residual + row * P.residual_ld, t, width, D, row < n);
        }
        float sum[2 * U];                                    // sum h^2, sum g h
#pragma unroll
        for (int u = 0; u < U; ++u) {
            sum[2 * u] = sum[2 * u + 1] = 0.f;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float a[VE], b[VE];
                h[u].get(j, a);
                dy[u].get(j, b);
#pragma unroll
                for (int i = 0; i < VE; ++i) {
                    sum[2 * u] = fmaf(a[i], a[i], sum[2 * u]);
                    sum[2 * u + 1] = fmaf(b[i] * w[j * VE + i], a[i], sum[2 * u + 1]);
                }
            }
        }
        row_sum<BLOCK, 2 * U>(sum, width);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = base + u * per_block + own;
            if (row >= n) continue;
            const float inv = __frsqrt_rn(sum[2 * u] / (float)D + P.eps), mean = sum[2 * u + 1] / (float)D * inv * inv * inv;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float a[VE], b[VE], x[VE];
                h[u].get(j, a);
                dy[u].get(j, b);
#pragma unroll
                for (int i = 0; i < VE; ++i) {
                    dw[j * VE + i] = fmaf(b[i], a[i] * inv, dw[j * VE + i]);
                    x[i] = fmaf(-a[i], mean, b[i] * w[j * VE + i] * inv);
                }
                if (P.residual) {
                    dh[u].get(j, b);
#pragma unroll
                    for (int i = 0; i < VE; ++i) x[i] += b[i];
                }
                h[u].set(j, x);
            }
            h[u].store((T*)P.out + row * P.out_ld, t, width, D);
        }
    }
    if (!P.dweight) return;
    float* part = dw_part + (int64_t)blockIdx.x * D;
    if constexpr (BLOCK) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                const int c = (t + j * width) * VE + i;
                if (c < D) part[c] = dw[j * VE + i];
            }
    } else {
        for (int o = width; o < 32; o <<= 1) {               // the groups of a warp
#pragma unroll
            for (int i = 0; i < E; ++i) dw[i] += __shfl_xor_sync(FULL, dw[i], o);
        }
        if ((threadIdx.x & 31) < width) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < VE; ++i) {
                    const int c = (t + j * width) * VE + i;
                    if (c < D) norm_dw[(threadIdx.x >> 5) * D + c] = dw[j * VE + i];
                }
        }
        __syncthreads();
        for (int c = threadIdx.x; c < D; c += NM_THREADS) {
            float s = 0.f;
            for (int i = 0; i < NM_THREADS / 32; ++i) s += norm_dw[i * D + c];
            part[c] = s;
        }
    }
}

// dw = the blocks' sums, added in order: 32 columns per block, its warps over contiguous shares of the blocks.
__global__ void __launch_bounds__(1024) k_norm_dweight(const float* __restrict__ part, int parts, int dim, void* dweight, gs_dtype dtype) {
    __shared__ float s[32][33];
    chain_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per = (parts + 31) / 32;
    for (int c0 = blockIdx.x * 32; c0 < dim; c0 += gridDim.x * 32) {
        const int c = c0 + lane, p1 = (warp + 1) * per < parts ? (warp + 1) * per : parts;
        float x = 0.f;
        if (c < dim) {
#pragma unroll 8
            for (int p = warp * per; p < p1; ++p) x += __ldcg(part + (int64_t)p * dim + c);
        }
        __syncthreads();
        s[warp][lane] = x;
        __syncthreads();
        if (warp == 0 && c < dim) {
            x = 0.f;
            for (int i = 0; i < 32; ++i) x += s[i][lane];
            if (dtype == GS_BF16) static_cast<bf16*>(dweight)[c] = __float2bfloat16_rn(x);
            else static_cast<float*>(dweight)[c] = x;
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

// A row's elements per thread: one to four pieces by lanes of a warp, up to 16 elements by a block.
template <typename F> static cudaError_t norm_shape(const RmsNorm& P, int ve, F run) {
    const int pieces = (P.dim + ve - 1) / ve;
    if (P.dtype == GS_BF16) {
        if (ve == 8) {
            if (pieces <= 32) return run(bf16(), std::integral_constant<int, 8>(), std::integral_constant<int, 1>(), std::false_type());
            if (pieces <= 64) return run(bf16(), std::integral_constant<int, 8>(), std::integral_constant<int, 2>(), std::false_type());
            return run(bf16(), std::integral_constant<int, 8>(), std::integral_constant<int, 2>(), std::true_type());
        }
        if (pieces <= 32) return run(bf16(), std::integral_constant<int, 1>(), std::integral_constant<int, 1>(), std::false_type());
        if (pieces <= 128) return run(bf16(), std::integral_constant<int, 1>(), std::integral_constant<int, 4>(), std::false_type());
        return run(bf16(), std::integral_constant<int, 1>(), std::integral_constant<int, 16>(), std::true_type());
    }
    if (ve == 4) {
        if (pieces <= 32) return run(float(), std::integral_constant<int, 4>(), std::integral_constant<int, 1>(), std::false_type());
        if (pieces <= 64) return run(float(), std::integral_constant<int, 4>(), std::integral_constant<int, 2>(), std::false_type());
        return run(float(), std::integral_constant<int, 4>(), std::integral_constant<int, 4>(), std::true_type());
    }
    if (pieces <= 32) return run(float(), std::integral_constant<int, 1>(), std::integral_constant<int, 1>(), std::false_type());
    if (pieces <= 128) return run(float(), std::integral_constant<int, 1>(), std::integral_constant<int, 4>(), std::false_type());
    return run(float(), std::integral_constant<int, 1>(), std::integral_constant<int, 16>(), std::true_type());
}

static bool whole_pieces(const RmsNorm& P, const void* p, int64_t ld, int size) { return !p || ((uintptr_t)p % 16 == 0 && (ld * size) % 16 == 0); }

static int norm_width(const RmsNorm& P, int ve, int nv, bool block) {
    const int threads = (P.dim + ve * nv - 1) / (ve * nv);
    if (block) return (threads + 31) / 32 * 32;
    int tl = 1;
    while (tl < threads) tl *= 2;
    return tl;
}

cudaError_t launch_norm_forward(const RmsNorm& p, bool coded, cudaStream_t s) {
    const int size = p.dtype == GS_BF16 ? 2 : 4;
    int ve = 16 / size;
    if (p.dim % ve || !whole_pieces(p, p.x, p.x_ld, size) || !whole_pieces(p, p.residual, p.residual_ld, size) || !whole_pieces(p, p.hidden, p.hidden_ld, size) ||
        !whole_pieces(p, p.out, p.out_ld, size) || (coded && p.coded.head_dim % ve))
        ve = 1;
    return norm_shape(p, ve, [&](auto type, auto vec, auto num, auto block) {
        using T = decltype(type);
        constexpr int VE = vec, NV = num, U = 2;
        constexpr bool B = block;
        RmsNorm P = p;
        P.tl = norm_width(p, VE, NV, B);
        const int threads = B ? P.tl : NM_THREADS, per = (B ? 1 : NM_THREADS / P.tl) * (coded || B ? 1 : U);
        int64_t grid = ((int64_t)p.n.bound + per - 1) / per;
        if (grid > sm_count() * 64) grid = sm_count() * 64;
        const size_t smem = coded ? (size_t)(B ? 1 : NM_THREADS / P.tl) * p.coded.heads * 4 : 0;
        if (coded) return launch_train(k_norm_forward<T, VE, NV, 1, B, true>, grid, threads, smem, s, P);
        return launch_train(k_norm_forward<T, VE, NV, (B ? 1 : U), B, false>, grid, threads, smem, s, P);
    });
}

cudaError_t launch_norm_backward(const RmsNorm& p, void* workspace, cudaStream_t s) {
    const int size = p.dtype == GS_BF16 ? 2 : 4;
    int ve = 16 / size;
    if (p.dim % ve || !whole_pieces(p, p.x, p.x_ld, size) || !whole_pieces(p, p.residual, p.residual_ld, size) || !whole_pieces(p, p.dout, p.dout_ld, size) ||
        !whole_pieces(p, p.out, p.out_ld, size))
        ve = 1;
    return norm_shape(p, ve, [&](auto type, auto vec, auto num, auto block) {
        using T = decltype(type);
        constexpr int VE = vec, NV = num;
        constexpr bool B = block;
        constexpr int U = B ? 1 : 2;
        RmsNorm P = p;
        P.tl = norm_width(p, VE, NV, B);
        const int threads = B ? P.tl : NM_THREADS, per = (B ? 1 : NM_THREADS / P.tl) * U;
        int64_t grid = ((int64_t)p.n.bound + per - 1) / per;
        const int64_t most = norm_parts(p.n.bound);
        grid = limit_grid(grid > most ? most : grid);
        float* part = (float*)workspace;
        cudaError_t e = launch_train(k_norm_backward<T, VE, NV, U, B>, grid, threads, B ? 0 : (size_t)(NM_THREADS / 32) * p.dim * 4, s, P, part);
        if (e == cudaSuccess && p.dweight) e = launch_train(k_norm_dweight, (p.dim + 31) / 32, 1024, 0, s, (const float*)part, (int)grid, (int)p.dim, p.dweight, p.weight_dtype);
        return e;
    });
}

}  // namespace gs
