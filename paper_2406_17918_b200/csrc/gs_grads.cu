// The norm over all gradients of a step, and their scaling to a largest norm.
//
//   norm = sqrt(sum over all tensors of g^2);  g <- g min(1, max_norm / (norm + 1e-6))
//
// Two passes over the bytes, because no element may be scaled before the last has been counted; what L2 still holds of the first
// pass is met first by the second, which walks the tiles backwards: the first pass asks L2 to keep only its last GN_KEPT bytes, the
// second's results are not kept (on one device 174 MB of f32: 85 -> 81 us, 708 MB 322 -> 308; 40 MB instead of 80: 84 and 313, all of them: 83
// and 318).  Of the 522 MB that two passes over 174 ask for DRAM moves 447: 0.85 to 0.87 of a plain copy's rate in 78 to 80 us.  The tensors'
// addresses travel as a kernel argument: nothing is copied to the device, and a captured call can be replayed.  Squares are added eight or four at a time in 32 bits, then in 64, each
// block its tiles in order and the blocks' sums in order: the result does not depend on the schedule.  Squares that leave the range
// of 32 bits are taken in 64.
#include "gs_device.cuh"
#include "gs_train.cuh"
#include "gs_train.h"

namespace gs {

constexpr int GN_THREADS = 256;
constexpr int GN_TILE = 8192;        // elements of a tile
constexpr int64_t GN_KEPT = 80 << 20;
constexpr int GN_FEW = 32, GN_MANY = 512;   // tensors that travel with one launch

template <int N> struct GradList {
    GradTensor t[N];
    int n, tiles, kept;              // kept: the first tile that the second pass finds in L2
};

template <int N> __device__ __forceinline__ int tensor_of(const GradList<N>& L, int tile) {
    int lo = 0, hi = L.n;                                    // the last tensor that starts at or before the tile
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (L.t[mid].first_tile <= tile) lo = mid;
        else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ int64_t elems_of(const GradTensor& t) {
    if (!t.d_rows) return t.elems;
    const int64_t n = (int64_t)__ldg(t.d_rows) * t.row_elems;
    return n < 0 ? 0 : (n > t.elems ? t.elems : n);
}

template <typename T, int VE> __device__ __forceinline__ double square_sum(const Raw<T, VE>& r) {
    float x[VE];
    unpack<T, VE>(r, x);
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < VE; ++i) s = fmaf(x[i], x[i], s);
    if (s >= 1e-25f && s < 1e37f) return (double)s;
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < VE; ++i) top = fmaxf(top, fabsf(x[i]));
    if (top == 0.f && s == 0.f) return 0.0;                  // zeros: a table's rows that no batch touched
    double d = 0.0;                                          // squares too small or too large for 32 bits
#pragma unroll
    for (int i = 0; i < VE; ++i) d += (double)x[i] * (double)x[i];
    return d;
}

template <typename T> __device__ __forceinline__ double tile_squares(const T* g, int64_t n, bool kept) {
    constexpr int VE = 16 / (int)sizeof(T), U = 4;
    double sum = 0.0;
    const int m = (int)(n < GN_TILE ? n : GN_TILE);
    if ((uintptr_t)g % 16 == 0) {
        const int whole = m / VE * VE;
        for (int i = threadIdx.x * VE; i < whole; i += GN_THREADS * VE * U) {
            Raw<T, VE> r[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int at = i + u * GN_THREADS * VE;
                r[u] = at >= whole ? zero_raw<T, VE>() : (kept ? load_raw<T, VE>(g + at) : load_raw_stream<T, VE>(g + at));
            }
#pragma unroll
            for (int u = 0; u < U; ++u) sum += square_sum<T, VE>(r[u]);
        }
        if ((int)threadIdx.x < m - whole) sum += square_sum<T, 1>(load_raw<T, 1>(g + whole + threadIdx.x));
    } else {
        for (int i = threadIdx.x; i < m; i += GN_THREADS) sum += square_sum<T, 1>(load_raw<T, 1>(g + i));
    }
    return sum;
}

// In every thread: the block's sum, warps in order.
__device__ __forceinline__ double block_sum(double x) {
    __shared__ double s[GN_THREADS / 32];
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(FULL, x, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = x;
    __syncthreads();
    x = 0.0;
    for (int w = 0; w < GN_THREADS / 32; ++w) x += s[w];
    return x;
}

template <int N> __global__ void __launch_bounds__(GN_THREADS) k_grad_squares(const __grid_constant__ GradList<N> L, double* __restrict__ sums) {
    chain_wait();
    double sum = 0.0;
    for (int tile = blockIdx.x; tile < L.tiles; tile += gridDim.x) {
        const GradTensor& t = L.t[tensor_of(L, tile)];
        const int64_t at = (int64_t)(tile - t.first_tile) * GN_TILE, n = elems_of(t) - at;
        if (n <= 0) continue;
        const bool kept = tile >= L.kept;
        sum += t.dtype == GS_BF16 ? tile_squares((const bf16*)t.grad + at, n, kept) : tile_squares((const float*)t.grad + at, n, kept);
    }
    sum = block_sum(sum);
    if (threadIdx.x == 0) sums[blockIdx.x] = sum;
}

__device__ __forceinline__ double total_norm(const double* sums, int n) {
    double x = 0.0;
    for (int i = threadIdx.x; i < n; i += GN_THREADS) x += __ldcg(sums + i);
    return sqrt(block_sum(x));
}

__global__ void __launch_bounds__(GN_THREADS) k_grad_total(const double* sums, int n, float* norm) {
    chain_wait();
    const double x = total_norm(sums, n);
    if (threadIdx.x == 0) *norm = (float)x;
}

template <typename T> __device__ __forceinline__ void tile_scale(const T* g, T* out, int64_t n, float c) {
    constexpr int VE = 16 / (int)sizeof(T), U = 4;
    const int m = (int)(n < GN_TILE ? n : GN_TILE);
    int whole = 0;
    if (((uintptr_t)g | (uintptr_t)out) % 16 == 0) {
        whole = m / VE * VE;
        for (int i = threadIdx.x * VE; i < whole; i += GN_THREADS * VE * U) {
            Raw<T, VE> r[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int at = i + u * GN_THREADS * VE;
                if (at < whole) r[u] = load_raw_stream<T, VE>(g + at);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int at = i + u * GN_THREADS * VE;
                if (at >= whole) continue;
                float x[VE];
                unpack<T, VE>(r[u], x);
#pragma unroll
                for (int j = 0; j < VE; ++j) x[j] *= c;
                store_vec<T, VE, true>(out + at, x);
            }
        }
    }
    for (int i = whole + threadIdx.x; i < m; i += GN_THREADS) out[i] = from_f32<T>(to_f32(g[i]) * c);
}

template <int N> __global__ void __launch_bounds__(GN_THREADS) k_grad_scale(const __grid_constant__ GradList<N> L, const double* sums, int n_sums, float max_norm, float* norm) {
    chain_wait();
    const double total = total_norm(sums, n_sums);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)total;
    const double ratio = (double)max_norm / (total + 1e-6);
    const float c = ratio >= 1.0 ? 1.f : (float)ratio;       // NaN stays NaN
    for (int i = blockIdx.x; i < L.tiles; i += gridDim.x) {
        const int tile = L.tiles - 1 - i;
        const GradTensor& t = L.t[tensor_of(L, tile)];
        const int64_t at = (int64_t)(tile - t.first_tile) * GN_TILE, n = elems_of(t) - at;
        if (n <= 0 || (c == 1.f && t.out == t.grad)) continue;
        if (t.dtype == GS_BF16) tile_scale((const bf16*)t.grad + at, (bf16*)t.out + at, n, c);
        else tile_scale((const float*)t.grad + at, (float*)t.out + at, n, c);
    }
}

// ---------------------------------------------------------------- launches
static int64_t grad_blocks() { return sm_count() * 8; }
size_t grad_workspace(int32_t tensors) { return align_up((size_t)((tensors + GN_MANY - 1) / GN_MANY + 1) * grad_blocks() * 8, 256); }

template <int N> static cudaError_t run_grads(const GradTensor* tensors, int32_t n, bool clip, float max_norm, float* norm, double* sums, cudaStream_t s) {
    int used = 0;
    const int lists = n > 0 ? (n + N - 1) / N : 1;           // none at all: a norm of zero
    for (int pass = 0; pass < (clip ? 2 : 1); ++pass)
        for (int i = 0; i < lists; ++i) {
            // the second pass begins with the tensors that the first ended with
            const int at = (pass ? lists - 1 - i : i) * N;
            GradList<N> L;
            L.n = n - at < N ? n - at : N;
            L.tiles = 0;
            for (int k = 0; k < L.n; ++k) {
                L.t[k] = tensors[at + k];
                L.t[k].first_tile = L.tiles;
                L.tiles += (int)((L.t[k].elems + GN_TILE - 1) / GN_TILE);
            }
            L.kept = L.tiles;
            int64_t room = GN_KEPT;
            for (int k = L.n - 1; k >= 0 && room > 0 && i == lists - 1; --k) {
                const int64_t bytes = GN_TILE * (L.t[k].dtype == GS_BF16 ? 2 : 4), have = L.kept - L.t[k].first_tile;
                const int64_t tiles = have < room / bytes ? have : room / bytes;
                L.kept -= (int)tiles;
                room = tiles < have ? 0 : room - tiles * bytes;
            }
            const int64_t grid = limit_grid(L.tiles > grad_blocks() ? grad_blocks() : L.tiles);
            const cudaError_t e = pass ? launch_train(k_grad_scale<N>, grid, GN_THREADS, 0, s, L, (const double*)sums, used, max_norm, i ? (float*)nullptr : norm)
                                       : launch_train(k_grad_squares<N>, grid, GN_THREADS, 0, s, L, sums + used);
            if (e != cudaSuccess) return e;
            if (!pass) used += (int)grid;
        }
    return clip ? cudaSuccess : launch_train(k_grad_total, 1, GN_THREADS, 0, s, (const double*)sums, used, norm);
}

cudaError_t launch_grad_norm(const GradTensor* tensors, int32_t n, bool clip, float max_norm, float* norm, void* workspace, cudaStream_t s) {
    return n <= GN_FEW ? run_grads<GN_FEW>(tensors, n, clip, max_norm, norm, (double*)workspace, s)
                       : run_grads<GN_MANY>(tensors, n, clip, max_norm, norm, (double*)workspace, s);
}

}  // namespace gs
