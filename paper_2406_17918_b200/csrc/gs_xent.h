// How the softmax-over-a-table kernels divide their work.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace gs {

// A grid of tiles_x by tiles_y output tiles, walked with y fastest, cut into `parts` equal runs: run c covers the
// tiles [start(c), start(c + 1)) of the flattened grid.  A run that does not hold a whole row of tiles leaves a
// partial result for that row: the run that starts inside row i in slot 2c, a run that starts at or before row i
// and ends inside it in slot 2c + 1.
struct Runs {
    int64_t tiles_x, tiles_y, parts, quot, rem;    // quot, rem: of total() / parts
    double per_tile;                                // parts / total()
    __host__ __device__ int64_t total() const { return tiles_x * tiles_y; }
    // total() * c / parts with a 32-bit division (parts is a small multiple of the SMs)
    __host__ __device__ int64_t start(int64_t c) const { return quot * c + (uint32_t)((uint32_t)c * (uint32_t)rem) / (uint32_t)parts; }
    // The run that holds flattened tile t.
    __host__ __device__ int64_t run_of(int64_t t) const {
        int64_t c = (int64_t)((double)t * per_tile);
        if (c > parts - 1) c = parts - 1;
        while (c + 1 < parts && start(c + 1) <= t) ++c;
        while (c > 0 && start(c) > t) --c;
        return c;
    }
    __host__ __device__ int64_t slot(int64_t c, int64_t row) const { return start(c) > row * tiles_y ? 2 * c : 2 * c + 1; }
};

inline Runs make_runs(int64_t x, int64_t tile_x, int64_t y, int64_t tile_y, int64_t parts) {
    Runs r{};
    r.tiles_x = (x + tile_x - 1) / tile_x;
    r.tiles_y = (y + tile_y - 1) / tile_y;
    r.parts = parts > r.total() ? r.total() : parts;
    if (r.parts < 1) r.parts = 1;
    r.quot = r.total() / r.parts;
    r.rem = r.total() % r.parts;
    r.per_tile = (double)r.parts / (double)r.total();
    return r;
}

// The rows of tiles that several runs share: row, the first run that starts inside it, the number of runs that do.
constexpr int MAX_JOINS = 320;
struct JoinList {
    struct Entry {
        int32_t row, first, runs;
    } e[MAX_JOINS];
};
inline int list_joins(const Runs& r, JoinList* l) {
    int n = 0;
    for (int64_t c = 1; c < r.parts && n < MAX_JOINS; ++c) {
        const int64_t t = r.start(c), i = t / r.tiles_y;
        if (t == i * r.tiles_y || r.start(c - 1) > i * r.tiles_y) continue;
        int64_t last = c;
        while (last + 1 < r.parts && r.start(last + 1) < (i + 1) * r.tiles_y) ++last;
        l->e[n++] = {(int32_t)i, (int32_t)c, (int32_t)(last - c + 1)};
    }
    return n;
}

constexpr int XENT_TC_TILE = 128;       // rows of either operand per tile of the tensor-core kernels
constexpr int XENT_TC_STATS = 4;        // entries of forward statistics per run and row of tiles
constexpr int XENT_TC_MAX_DIM = 256;    // a gradient tile of 128 rows and S of two units fill the 512 columns of tensor memory

struct Xent;
bool xent_tc_takes(const Xent& a);
size_t xent_tc_workspace(const Xent& a);
cudaError_t launch_xent_tc_forward(const Xent& a, void* workspace, Runs* runs, const float2** stats, const float** picked, cudaStream_t s);
cudaError_t launch_xent_tc_backward(const Xent& a, void* workspace, cudaStream_t s);
cudaError_t launch_xent_join(const Xent& a, bool hidden, const Runs& runs, int tile, int pitch, const float* partial, cudaStream_t s);
cudaError_t xent_gave_up(cudaStream_t s, int* h_flag);

}  // namespace gs
