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
// What bounds it is instructions (issue slots 67 %, 41 % of the DRAM rate): 677 per warp and batch of 4 edges x 16 columns, 256 of them the
// codes' conversion and the products.  262,144 rows, 4.36 M edges, 4 x 32 bf16: 281 to 299 us from device to device (1.1 GB gathered, 3.8 TB/s),
// f32 8 more.  Timed on one device against 285: 2 or 3 edges a batch 370, 5 292, 8 328; 8 columns a lane 467, 32 404 (fewer warps).  Spills, bytes
// loaded: heads by fours 46 to 58 at 168 registers, the join 144 at 64.
#include "gs_codes.cuh"
#include "gs_device.cuh"
#include "gs_train.h"

namespace gs {

constexpr int CA_THREADS = 128;
constexpr int CA_LONG = 64;          // rows of more edges go to the chunk list
constexpr int CA_CHUNK = 128, CA_CHUNK_MOST = 512;   // edges of a chunk (at least 2 CA_LONG: the workspace's bound)
constexpr float CA_LOG2E = 1.4426950408889634f, CA_LN2 = 0.6931471805599453f;

// Lengths of the lists.  The chunks that rows ask for are counted in 64 bits: offsets that do not ascend can name the same edges from
// every row, 2^31 times 2^23 chunks, and a count that wraps would hand places out twice.
struct ListWords {
    unsigned long long chunks;
    int longs;
};

struct CodedAttend {
    CodedAttention a;
    int tl, slots, units_per_row, unit_shift;
    int wide;                        // q and out in whole pieces
    int split, chunk_mode, chunk;    // chunk: edges of one
    int most;                        // places in the lists
    ListWords* words;
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
    __device__ __forceinline__ void take(const unsigned char* p) {
        if constexpr (VE == 16) {
            const uint4 x = *reinterpret_cast<const uint4*>(p);
            w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
        } else {
            const uint2 x = *reinterpret_cast<const uint2*>(p);
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

// What a warp works on at a time: a set of units, one to each group of lanes (or to `slots` groups), over the same number of batches.
struct CodedUnits {
    int r, row, unit, begin, end;    // r: the row, or the chunk
    bool live;
};

// The chunks of a row from `first` on that the lists have places for: all, where the offsets ascend.
__device__ __forceinline__ int list_room(const CodedAttend& P, int first, int nc) {
    const int room = P.most - first;
    return nc < room ? nc : room;
}
// Puts a row of nc chunks on the list of long rows, by one thread; the first of its places among the chunks.
__device__ __forceinline__ int list_row(const CodedAttend& P, int row, int nc) {
    const unsigned long long at = atomicAdd(&P.words->chunks, (unsigned long long)nc);
    const int first = at < (unsigned long long)P.most ? (int)at : P.most;
    if (list_room(P, first, nc) > 0) P.longs[atomicAdd(&P.words->longs, 1)] = make_int4(row, first, list_room(P, first, nc), 0);
    return first;
}
__device__ __forceinline__ int listed_chunks(const CodedAttend& P) {
    const unsigned long long n = __ldcg(&P.words->chunks);
    return n < (unsigned long long)P.most ? (int)n : P.most;
}

// What a launch does with rows of more than CA_LONG edges: there are none (or they are no matter), they are listed, or their chunks are
// its rows.
enum { CA_ALL, CA_LIST, CA_CHUNKS };

template <int MODE> __device__ __forceinline__ CodedUnits find_units(const CodedAttend& P, int64_t u, int64_t units, int part, int parts) {
    CodedUnits w;
    w.live = u < units;
    w.r = w.row = w.unit = w.begin = w.end = 0;
    if (!w.live) return w;
    if (P.unit_shift >= 0) w.r = (int)(u >> P.unit_shift);
    else w.r = units >> 31 ? (int)(u / P.units_per_row) : (int)((uint32_t)u / (uint32_t)P.units_per_row);
    w.unit = (int)(u - (int64_t)w.r * P.units_per_row);
    w.row = w.r;
    int skip = 0;
    if constexpr (MODE == CA_CHUNKS) {
        const int2 it = P.items[w.r];
        w.row = it.x;
        skip = it.y * P.chunk;
    }
    int b = __ldg(P.a.indptr + w.row), e = __ldg(P.a.indptr + w.row + 1);
    b = b < 0 ? 0 : b;
    e = e > P.a.edge_bound ? P.a.edge_bound : e;
    if (e < b) e = b;
    if constexpr (MODE == CA_CHUNKS) {
        w.begin = b + skip;
        w.end = w.begin + P.chunk < e ? w.begin + P.chunk : e;
    } else if (MODE == CA_LIST && e - b > CA_LONG) {
        if (w.unit == 0) {                                   // listed once, by the lanes of the row's first unit
            const int lanes = parts - 1;
            int nc = (e - b + P.chunk - 1) / P.chunk;
            const uint32_t mask = parts == 32 ? FULL : ((1u << parts) - 1u) << (threadIdx.x & 31 & ~lanes);
            int first = 0;
            if (part == 0) first = list_row(P, w.row, nc);
            first = __shfl_sync(mask, first, threadIdx.x & 31 & ~lanes);
            nc = list_room(P, first, nc);
            for (int c = part; c < nc; c += parts) P.items[first + c] = make_int2(w.row, c);
        }
        w.live = false;
    } else {
        w.begin = b;
        w.end = e;
    }
    return w;
}

// The batches of a warp's sets are one stream: the codes of a batch are on their way to slots of the lane's own in shared memory
// (zeros where there is no edge) while the batch before is worked on, the rows of the next one are looked up, and the next set's
// offsets and query rows are fetched when its first batch is.  No lane reads what another has copied: no barriers.
template <typename T, int VE, int G, int U, int MODE> __global__ void __launch_bounds__(CA_THREADS, G == 1 ? 4 : 3) k_coded_attend(const __grid_constant__ CodedAttend P) {
    constexpr int N2 = VE / 2;
    constexpr int SLOT = U * 2 * VE * 32;                    // bytes of a batch's copies, per warp
    extern __shared__ __align__(16) unsigned char ca_smem[];
    chain_wait();
    const int lane = threadIdx.x & 31, tl = P.tl, t = lane & (tl - 1), slot = (lane / tl) & (P.slots - 1);
    const int width = tl * P.slots, per_warp = 32 / width;
    const int rows = MODE == CA_CHUNKS ? listed_chunks(P) : list_length(P.a.dst), cols = list_length(P.a.src);
    const int64_t units = (int64_t)rows * P.units_per_row;
    const int64_t step = (int64_t)gridDim.x * (CA_THREADS / 32) * per_warp;
    const float c2 = P.a.scale * CA_LOG2E;
    const int D = P.a.head_dim, c0 = t * VE, group = P.a.q_heads / P.a.kv_heads;
    const int held = min(VE, max(D - c0, 0));                // this lane's codes; what lies behind head_dim is not read
    const uint32_t kstep = (uint32_t)P.a.k.row_stride, vstep = (uint32_t)P.a.v.row_stride, ksstep = (uint32_t)P.a.k.scale_stride, vsstep = (uint32_t)P.a.v.scale_stride;
    unsigned char* mine = ca_smem + (threadIdx.x >> 5) * 2 * SLOT + lane * VE;
    const uint32_t mine_a = (uint32_t)__cvta_generic_to_shared(mine);

    // ---- ahead: the set whose batches are being fetched
    int64_t base = ((int64_t)blockIdx.x * (CA_THREADS / 32) + (threadIdx.x >> 5)) * per_warp;
    CodedUnits w = find_units<MODE>(P, base + lane / width, units, lane & (width - 1), width);
    const uint8_t* kbase = nullptr;
    const uint8_t* vbase = nullptr;
    const uint8_t* ksbase = nullptr;
    const uint8_t* vsbase = nullptr;
    f32x2 qn[G][N2];
    int trips = 0, it = 0;
    int next[U];                                             // the rows of the batch that is fetched next, -1 where there is none
    auto begin_set = [&]() {
        const int h0 = w.unit * G, g = h0 / group;
        kbase = P.a.k.codes + (int64_t)g * P.a.k.pitch + (held ? c0 : 0);
        vbase = P.a.v.codes + (int64_t)g * P.a.v.pitch + (held ? c0 : 0);
        ksbase = P.a.k.scales + g;
        vsbase = P.a.v.scales + g;
        const int n = (w.end - w.begin + P.slots * U - 1) / (P.slots * U);
        trips = __reduce_max_sync(FULL, n < 1 ? 1 : n);
        it = 0;
#pragma unroll
        for (int i = 0; i < G; ++i)
            load_piece<T, VE>((const T*)P.a.q.data + (int64_t)w.row * P.a.q.row_stride + (int64_t)(h0 + i) * P.a.q.head_stride, c0, D, P.wide, w.live, qn[i]);
    };
    auto look = [&]() {
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int e = w.begin + (it * U + j) * P.slots + slot;
            int col = e < w.end ? __ldg(P.a.indices + e) : -1;
            if ((uint32_t)col >= (uint32_t)cols) col = -1;
            if (P.a.row_of && col >= 0) col = __ldg(P.a.row_of + col);
            next[j] = (uint32_t)col < (uint32_t)P.a.k.rows ? col : -1;
        }
    };
    uint32_t ks[U], vs[U], on = 0;                           // of the batch on its way
    auto issue = [&](int s) {
        on = 0;
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const bool is = next[j] >= 0;
            const uint32_t at = is ? (uint32_t)next[j] : 0u, b = at >> P.a.k.shift;
            const int bytes = is ? held : 0;
            copy_async<VE>(mine_a + s * SLOT + j * 2 * VE * 32, kbase + (uint64_t)at * kstep, bytes);
            copy_async<VE>(mine_a + s * SLOT + (j * 2 + 1) * VE * 32, vbase + (uint64_t)at * vstep, bytes);
            ks[j] = is ? __ldg(ksbase + (uint64_t)b * ksstep) : 0u;
            vs[j] = is ? __ldg(vsbase + (uint64_t)b * vsstep) : 0u;
            on |= is ? 1u << j : 0u;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    bool more = base < units;
    if (!more) return;
    begin_set();
    look();
    issue(0);

    f32x2 q[G][N2], acc[G][N2];
    float m[G], l[G];
    int s = 0;
    while (more) {
        const bool first = it == 0, last = it + 1 == trips;
        const CodedUnits cur = w;
        const uint32_t my_on = on;
        uint32_t my_ks[U], my_vs[U];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            my_ks[j] = ks[j];
            my_vs[j] = vs[j];
        }
        if (first) {
#pragma unroll
            for (int i = 0; i < G; ++i) {
                m[i] = -INFINITY;
                l[i] = 0.f;
#pragma unroll
                for (int c = 0; c < N2; ++c) {
                    q[i][c] = qn[i][c];
                    acc[i][c] = 0;
                }
            }
        }
        // what comes next: this set's next batch, or the next set's first
        ++it;
        if (last) {
            base += step;
            more = base < units;
            if (more) {
                w = find_units<MODE>(P, base + lane / width, units, lane & (width - 1), width);
                begin_set();
            }
        }
        if (more) {
            look();
            issue(s ^ 1);
            asm volatile("cp.async.wait_group 1;" ::: "memory");
        } else {
            asm volatile("cp.async.wait_group 0;" ::: "memory");
        }
        const unsigned char* from = mine + s * SLOT;
        s ^= 1;
        float sc[U * G];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            Codes<VE> kc;
            f32x2 k[N2];
            kc.take(from + j * 2 * VE * 32);
            kc.get(k);
#pragma unroll
            for (int i = 0; i < G; ++i) {
                f32x2 x = mul2(q[i][0], k[0]);
#pragma unroll
                for (int c = 1; c < N2; ++c) x = fma2(q[i][c], k[c], x);
                float lo, hi;
                split(x, lo, hi);
                sc[j * G + i] = lo + hi;
            }
        }
        for (int o = 1; o < tl; o <<= 1) {
#pragma unroll
            for (int x = 0; x < U * G; ++x) sc[x] += __shfl_xor_sync(FULL, sc[x], o);
        }
        float p[U * G];
#pragma unroll
        for (int i = 0; i < G; ++i) {
            float top = m[i];
#pragma unroll
            for (int j = 0; j < U; ++j) {
                sc[j * G + i] = my_on >> j & 1 ? sc[j * G + i] * scale_of(my_ks[j]) * c2 : -INFINITY;
                top = fmaxf(top, sc[j * G + i]);
            }
            const float ref = top == -INFINITY ? 0.f : top;         // nothing seen yet: all weights are zero
            const float corr = exp2_fast(m[i] - ref);
            m[i] = top;
            l[i] *= corr;
#pragma unroll
            for (int j = 0; j < U; ++j) {
                p[j * G + i] = exp2_fast(sc[j * G + i] - ref);
                l[i] += p[j * G + i];
            }
            const f32x2 cc = pair(corr, corr);
#pragma unroll
            for (int c = 0; c < N2; ++c) acc[i][c] = mul2(cc, acc[i][c]);
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
            Codes<VE> vc;
            f32x2 v[N2];
            vc.take(from + (j * 2 + 1) * VE * 32);
            vc.get(v);
            const float sv = scale_of(my_vs[j]);
#pragma unroll
            for (int i = 0; i < G; ++i) {
                const float x = p[j * G + i] * sv;
                const f32x2 xx = pair(x, x);
#pragma unroll
                for (int c = 0; c < N2; ++c) acc[i][c] = fma2(xx, v[c], acc[i][c]);
            }
        }
        if (!last) continue;
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
        if (!cur.live || slot) continue;
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const int h = cur.unit * G + i;
            float y[VE];
#pragma unroll
            for (int c = 0; c < N2; ++c) split(acc[i][c], y[2 * c], y[2 * c + 1]);
            if constexpr (MODE == CA_CHUNKS) {
                float* part = P.partial + ((int64_t)cur.r * P.a.q_heads + h) * (D + 2);
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
                store_out<T, VE>((T*)P.a.out.data + (int64_t)cur.row * P.a.out.row_stride + (int64_t)h * P.a.out.head_stride, c0, D, P.wide, y);
                if (t == 0) P.a.lse[(int64_t)cur.row * P.a.q_heads + h] = none ? -INFINITY : m[i] * CA_LN2 + logf(l[i]);
            }
        }
    }
}

// The sums of chunks [c0, c1) of one head and 32 columns (x: of this lane's column of the first), relative to their largest maximum m;
// 32 chunks at a time, all on their way together.
__device__ __forceinline__ void join_chunks(const float* part, int64_t stride, int D, int col, int c0, int c1, float& m, float& l, float& acc) {
    const int lane = threadIdx.x & 31;
    m = -INFINITY;
    l = acc = 0.f;
    for (int c = c0; c < c1; c += 32) {
        const bool is = c + lane < c1;
        const float* mine = part + (int64_t)(is ? c + lane : c) * stride + D;
        const float mc = is ? mine[0] : -INFINITY, lc = is ? mine[1] : 0.f;
        float x[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) x[i] = c + i < c1 && col < D ? part[(int64_t)(c + i) * stride + col] : 0.f;
        float top = fmaxf(m, mc);
        for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(FULL, top, o));
        const float ref = top == -INFINITY ? 0.f : top, corr = exp2_fast(m - ref), scale = exp2_fast(mc - ref);
        m = top;
        l = fmaf(lc, scale, l * corr);                        // of this lane's chunks
        acc *= corr;
#pragma unroll
        for (int i = 0; i < 32; ++i) acc = fmaf(x[i], __shfl_sync(FULL, scale, i), acc);
    }
    for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(FULL, l, o);
}

// Joins the chunks of a long row, for one query head and 32 columns: by a warp if there are at most 32 of them, else each of a
// block's warps takes a contiguous share and the shares are joined in order.
template <typename T> __global__ void __launch_bounds__(1024) k_coded_attend_join(const __grid_constant__ CodedAttend P) {
    constexpr int W = 32;
    __shared__ float s_m[W], s_l[W], s_acc[W][32];
    chain_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, D = P.a.head_dim, parts = (D + 31) / 32, per_row = P.a.q_heads * parts;
    const int64_t units = (int64_t)__ldcg(&P.words->longs) * per_row, stride = (int64_t)P.a.q_heads * (D + 2);
    auto put = [&](const int4& row, int h, int col, float m, float l, float sum) {
        const bool none = l == 0.f;
        T* out = (T*)P.a.out.data + (int64_t)row.x * P.a.out.row_stride + (int64_t)h * P.a.out.head_stride;
        if (col < D) out[col] = from_f32<T>(none ? 0.f : sum / l);
        if (col == 0) P.a.lse[(int64_t)row.x * P.a.q_heads + h] = none ? -INFINITY : m * CA_LN2 + logf(l);
    };
    for (int64_t base = blockIdx.x; base < units; base += (int64_t)gridDim.x * W) {
        float m, l, acc;
        int64_t u = base + (int64_t)warp * gridDim.x;
        if (u < units) {
            const int4 row = P.longs[u / per_row];
            const int h = (int)(u % per_row) / parts, col = (int)(u % parts) * 32 + lane;
            if (row.z <= 32) {
                join_chunks(P.partial + (int64_t)row.y * stride + (int64_t)h * (D + 2), stride, D, col, 0, row.z, m, l, acc);
                put(row, h, col, m, l, acc);
            }
        }
        u = base;
        for (int i = 0; i < W && u < units; ++i, u += gridDim.x) {
            const int4 row = P.longs[u / per_row];
            if (row.z <= 32) continue;
            const int h = (int)(u % per_row) / parts, col = (int)(u % parts) * 32 + lane;
            const int per = (row.z + W - 1) / W, c0 = warp * per, c1 = c0 + per < row.z ? c0 + per : row.z;
            join_chunks(P.partial + (int64_t)row.y * stride + (int64_t)h * (D + 2), stride, D, col, c0, c1, m, l, acc);
            __syncthreads();                                   // the previous unit's sums are read
            if (lane == 0) {
                s_m[warp] = m;
                s_l[warp] = l;
            }
            s_acc[warp][lane] = acc;
            __syncthreads();
            if (warp != 0) continue;
            const float mw = s_m[lane];
            m = mw;
            for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(FULL, m, o));
            const float scale = exp2_fast(mw - (m == -INFINITY ? 0.f : m));
            l = s_l[lane] * scale;
            for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(FULL, l, o);
            acc = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) acc = fmaf(s_acc[w][lane], __shfl_sync(FULL, scale, w), acc);
            put(row, h, col, m, l, acc);
        }
    }
}

}  // namespace gs

#include "gs_coded_attend_tc.cuh"

namespace gs {

// ---------------------------------------------------------------- launches
struct CodedAttendLayout {
    size_t words, items, longs, partial, total;
};
// Chunks, and long rows: each has more than LONG edges.
static int64_t coded_attend_most(int64_t edges) { return edges / CA_LONG + 1; }
static CodedAttendLayout coded_attend_layout(int64_t edges, int32_t q_heads, int32_t head_dim) {
    CodedAttendLayout l{};
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t o = off; off = align_up(off + bytes, 256); return o; };
    const int64_t most = coded_attend_most(edges);
    l.words = take(256);
    l.items = take((size_t)most * 8);
    l.longs = take((size_t)most * 16);
    l.partial = take((size_t)most * q_heads * (head_dim + 2) * 4);
    l.total = off;
    return l;
}
size_t coded_attention_workspace(int64_t edges, int32_t q_heads, int32_t head_dim) { return coded_attend_layout(edges, q_heads, head_dim).total; }

static void set_units(CodedAttend& P, int heads) {
    P.units_per_row = P.a.q_heads / heads;
    P.unit_shift = -1;
    for (int i = 0; i < 8; ++i)
        if (P.units_per_row == 1 << i) P.unit_shift = i;
}
static int64_t chunk_bound(const CodedAttend& P) { return P.most; }
// Chunks that keep the warps that are resident busy once, so that no warp has a second one while others have none, and the join little
// to do (one row of 200,011 edges, 2 x 4 heads of 64: 38 us, with chunks of 128 46).
static int chunk_length(const CodedAttend& P, int heads, int64_t warps) {
    const int64_t n = ((int64_t)P.a.edge_bound * (P.a.q_heads / heads) / warps + 31) / 32 * 32;
    return n < CA_CHUNK ? CA_CHUNK : (n > CA_CHUNK_MOST ? CA_CHUNK_MOST : (int)n);
}

// Edges by groups of lanes: rows of up to CA_LONG edges, or chunks.
template <typename T, int VE, int G> static cudaError_t run_coded(CodedAttend P, int chunk_mode, cudaStream_t s) {
    constexpr int U = 4;
    const int pieces = P.a.k.pitch / VE;
    P.tl = 1;
    while (P.tl < pieces) P.tl *= 2;
    set_units(P, G);
    constexpr int smem = CA_THREADS / 32 * 2 * U * 2 * VE * 32;
    P.chunk_mode = chunk_mode;
    const int64_t n = chunk_mode ? chunk_bound(P) : P.a.dst.bound;
    P.slots = chunk_mode ? 32 / P.tl : 1;
    // groups share a row while the rows alone do not give every SM sixteen warps and each keeps U edges
    const int longest = P.a.max_row == 0 || P.a.max_row > CA_LONG ? CA_LONG : P.a.max_row;
    while (!chunk_mode && P.tl * P.slots * 2 <= 32 && n * P.units_per_row * P.tl * P.slots * 2 <= sm_count() * 16 * 32 && P.slots * U < longest) P.slots *= 2;
    const int per_block = CA_THREADS / (P.tl * P.slots);
    int64_t grid = (n * P.units_per_row + per_block - 1) / per_block;
    const int64_t cap = sm_count() * 16;
    if (grid > cap) grid = cap;
    if constexpr (!(std::is_same<T, bf16>::value && G == 4))       // those chunks go to the tensor cores
        if (chunk_mode) return launch_train(k_coded_attend<T, VE, G, U, CA_CHUNKS>, grid, CA_THREADS, smem, s, P);
    return P.split ? launch_train(k_coded_attend<T, VE, G, U, CA_LIST>, grid, CA_THREADS, smem, s, P)
                   : launch_train(k_coded_attend<T, VE, G, U, CA_ALL>, grid, CA_THREADS, smem, s, P);
}
// Query heads that share a key/value head are taken together; what a lane holds of them stays within its registers.
static int lane_heads(const CodedAttend& P) {
    const int group = P.a.q_heads / P.a.kv_heads;
    return group % 4 == 0 ? 4 : (group % 2 == 0 ? 2 : 1);
}
template <typename T> static cudaError_t coded_lanes(const CodedAttend& P, int chunk_mode, cudaStream_t s) {
    const int heads = lane_heads(P);
    if (heads == 4) return run_coded<T, 8, 4>(P, chunk_mode, s);
    if (heads == 2) return run_coded<T, 8, 2>(P, chunk_mode, s);
    return run_coded<T, 16, 1>(P, chunk_mode, s);
}

// On the tensor cores.  warps: what is resident on the device.
template <int SP> static cudaError_t tensor_warps(int64_t& warps) {
    static std::atomic<uint64_t> allowed{0}, known{0};
    const cudaError_t e = allow_smem(k_coded_attend_tc<SP>, TcShape<SP>::SMEM, allowed);
    if (e == cudaSuccess) warps = (int64_t)sm_count() * resident_blocks(k_coded_attend_tc<SP>, TC_WARPS * 32, TcShape<SP>::SMEM, known) * TC_WARPS;
    return e;
}
template <int SP> static cudaError_t run_tc(CodedAttend P, int chunk_mode, int64_t warps, cudaStream_t s) {
    using S = TcShape<SP>;
    set_units(P, S::SLOTS);
    P.chunk_mode = chunk_mode;
    const int64_t n = chunk_mode ? chunk_bound(P) : P.a.dst.bound;
    int64_t grid = (n * P.units_per_row + TC_WARPS - 1) / TC_WARPS;
    if (grid > warps / TC_WARPS) grid = warps / TC_WARPS;
    return launch_train(k_coded_attend_tc<SP>, grid, TC_WARPS * 32, S::SMEM, s, P);
}
// Where the rows of a block go whose heads share by fours (chunks always go to the tensor cores).  A tile costs the same however few
// edges it has, and little less for narrow heads than for wide ones; but two rounds of the resident warps, or one, are sooner done with
// than the lanes' longer work on a row.  Tensor cores : lanes, us, 2 x 4 heads, rows of as many edges on average, by columns:
//          many rows (20,000 to 200,000)                        64 rows of 4    2,000 of 4    2,000 of 15
//   16     3: 426 : 100    24: 229 : 135    48: 184 : 129        8.2 : 10.2      10 : 10       12 : 18
//   32     3: 453 : 201    18: 152 : 139    24: 127 : 141        8.2 : 10.2      12 : 12       14 : 23
//   64     3: 408 : 311     6: 209 : 217     9: 141 : 182        8.2 : 12.3      12 : 20       14 : 29
//   128    3: 461 : 317     6: 236 : 219     9: 162 : 184       10.2 : 12.3      18 : 23       23 : 39
//   256    3: 606 : 324     9: 338 : 307    12: 340 : 367       10.3 : 14.3      45 : 33       53 : 59
static bool rows_to_tensor_cores(const CodedAttend& P, int64_t warps) {
    if ((int64_t)P.a.dst.bound * (P.a.q_heads / 4) <= 2 * warps) return true;
    int64_t edges = P.a.edge_bound / P.a.dst.bound;          // of a row
    if (P.a.max_row > 0 && edges > P.a.max_row) edges = P.a.max_row;
    const int pieces = P.a.k.pitch / 16;
    return pieces > 1 && edges >= (pieces <= 2 ? 20 : (pieces <= 4 ? 5 : (pieces <= 8 ? 7 : 10)));
}
template <int SP> static cudaError_t run_shared(CodedAttend P, cudaStream_t s) {
    int64_t warps = 0;
    cudaError_t e = tensor_warps<SP>(warps);
    if (e != cudaSuccess) return e;
    P.chunk = chunk_length(P, 4, warps);
    e = rows_to_tensor_cores(P, warps) ? run_tc<SP>(P, 0, warps, s) : coded_lanes<bf16>(P, 0, s);
    return P.split && e == cudaSuccess ? run_tc<SP>(P, 1, warps, s) : e;
}
template <typename T> static cudaError_t run_parts(CodedAttend P, cudaStream_t s) {
    if constexpr (std::is_same<T, bf16>::value)
        if (lane_heads(P) == 4) {
            const int pieces = P.a.k.pitch / 16;
            if (pieces <= 1) return run_shared<1>(P, s);
            if (pieces <= 2) return run_shared<2>(P, s);
            if (pieces <= 4) return run_shared<4>(P, s);
            if (pieces <= 8) return run_shared<8>(P, s);
            return run_shared<16>(P, s);
        }
    P.chunk = chunk_length(P, lane_heads(P), sm_count() * 16);
    const cudaError_t e = coded_lanes<T>(P, 0, s);
    return P.split && e == cudaSuccess ? coded_lanes<T>(P, 1, s) : e;
}
template <typename T> static cudaError_t run_attention(const CodedAttend& P, cudaStream_t s) {
    const cudaError_t e = run_parts<T>(P, s);
    return P.split && e == cudaSuccess ? launch_train(k_coded_attend_join<T>, sm_count() * 2, 1024, 0, s, P) : e;
}

cudaError_t launch_coded_attention(const CodedAttention& a, void* workspace, cudaStream_t s) {
    CodedAttend P{};
    P.a = a;
    const CodedAttendLayout l = coded_attend_layout(a.edge_bound, a.q_heads, a.head_dim);
    char* ws = (char*)workspace;
    P.most = (int)coded_attend_most(a.edge_bound);
    P.words = (ListWords*)(ws + l.words);
    P.items = (int2*)(ws + l.items);
    P.longs = (int4*)(ws + l.longs);
    P.partial = (float*)(ws + l.partial);
    if (a.k.rows == 0) P.a.k.codes = P.a.v.codes = P.a.k.scales = P.a.v.scales = (uint8_t*)workspace;   // nothing is read: every edge is masked
    P.split = (a.max_row == 0 || a.max_row > CA_LONG) && a.edge_bound > CA_LONG;
    const int size = a.dtype == GS_BF16 ? 2 : 4, ve = 16 / size;
    auto on16 = [&](const HeadView& v) { return (uintptr_t)v.data % 16 == 0 && (v.row_stride * size) % 16 == 0 && (v.head_stride * size) % 16 == 0; };
    P.wide = a.head_dim % ve == 0 && on16(a.q) && on16(a.out);
    if (P.split) {
        const cudaError_t e = cudaMemsetAsync(P.words, 0, sizeof(ListWords), s);
        if (e != cudaSuccess) return e;
    }
    return a.dtype == GS_BF16 ? run_attention<bf16>(P, s) : run_attention<float>(P, s);
}

}  // namespace gs
