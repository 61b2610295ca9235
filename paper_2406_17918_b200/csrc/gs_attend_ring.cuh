// Attention over a block with operands on 16- or 8-byte pieces: the edges stream through shared memory.
//
// A group of tl lanes owns one (row, head) unit at a time and walks through its units batch by batch (up to U edges of
// one row).  Every lane copies exactly the pieces it will use itself into slots of its own (cp.async, zero-filled where
// an edge is masked), RING_DEPTH batches ahead, and the column indices one batch earlier still: the gathers of the next
// batches are in flight across row boundaries while one is computed, they hold no registers, and no barrier is needed
// because no lane reads another's copies.  Rows' own operands (q; q, dout, out) ride in their first batch.
// Latency is hidden with 16 to 21 warps per SM, so what is left to save is instructions: pairs of values go through
// packed 32-bit operations, addresses are one multiply-add per copy, and masked edges take the same path as others.
#pragma once
#include "gs_train.cuh"

namespace gs {

constexpr int RING_SLOTS = 2;            // batches of copies per lane: 346 us with 2, 390 with 3, 492 with 4 (fewer warps fit)
constexpr int RING_DEPTH = RING_SLOTS - 1;
constexpr int RING_WARPS = 2;            // warps per block
constexpr int RING_ROWS = 64;            // rows whose offsets a warp holds at a time

template <int N> __device__ __forceinline__ float dot2(const f32x2 (&a)[N], const f32x2 (&b)[N]) {
    f32x2 s = mul2(a[0], b[0]);
#pragma unroll
    for (int i = 1; i < N; ++i) s = fma2(a[i], b[i], s);
    float lo, hi;
    split(s, lo, hi);
    return lo + hi;
}
template <int N> __device__ __forceinline__ void axpy2(float p, const f32x2 (&x)[N], f32x2 (&acc)[N]) {
    const f32x2 pp = pair(p, p);
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i] = fma2(pp, x[i], acc[i]);
}
template <int N> __device__ __forceinline__ void scale2(float p, f32x2 (&x)[N]) {
    const f32x2 pp = pair(p, p);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = mul2(pp, x[i]);
}
template <int N> __device__ __forceinline__ void unpair(const f32x2 (&x)[N], float (&y)[2 * N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) split(x[i], y[2 * i], y[2 * i + 1]);
}

// No element is infinite or NaN: a product with zero is zero.
template <int N> __device__ __forceinline__ bool all_finite(const f32x2 (&x)[N]) {
    f32x2 z = mul2(x[0], pair(0.f, 0.f));
#pragma unroll
    for (int i = 1; i < N; ++i) z = fma2(x[i], pair(0.f, 0.f), z);
    float lo, hi;
    split(z, lo, hi);
    return lo + hi == 0.f;
}

// Shifts of G neighbouring heads, zeros where there is no edge.
template <int G> __device__ __forceinline__ void load_shifts(const float* p, bool on, float* x) {
    if constexpr (G == 4) {
        const float4 w = on ? __ldg(reinterpret_cast<const float4*>(p)) : make_float4(0.f, 0.f, 0.f, 0.f);
        x[0] = w.x; x[1] = w.y; x[2] = w.z; x[3] = w.w;
    } else if constexpr (G == 2) {
        const float2 w = on ? __ldg(reinterpret_cast<const float2*>(p)) : make_float2(0.f, 0.f);
        x[0] = w.x; x[1] = w.y;
    } else {
        x[0] = on ? __ldg(p) : 0.f;
    }
}

// The sums over the tl lanes of a group, in every lane; straight code for the usual widths.
template <int N, int TL> __device__ __forceinline__ void group_sum_of(float (&x)[N]) {
#pragma unroll
    for (int o = 1; o < TL; o <<= 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] += __shfl_xor_sync(FULL, x[i], o);
    }
}
template <int N> __device__ __forceinline__ void ring_sum(float (&x)[N], int tl) {
    if (tl == 4) group_sum_of<N, 4>(x);
    else if (tl == 2) group_sum_of<N, 2>(x);
    else if (tl == 8) group_sum_of<N, 8>(x);
    else group_sum<N>(x, tl);
}

template <AttendKind K, typename T, int VE, int NV, int G, int U> struct RingShape {
    static constexpr int PB = (int)sizeof(T) * VE;                                 // bytes of a piece
    static constexpr int EDGE = (K == AT_DKV ? 2 * NV * G : 2 * NV);               // pieces per edge
    static constexpr int ROW = K == AT_FORWARD ? NV * G : (K == AT_DQ ? 3 * NV * G : 0);
    static constexpr int PIECES = (U * EDGE + ROW) * 32 * PB;
    static constexpr int STAT = K == AT_DKV ? U * G * 32 * 8 : (K == AT_DQ ? G * 32 * 4 : 0);
    static constexpr int SLOT = PIECES + STAT;
    static constexpr int WARP = RING_SLOTS * SLOT + RING_ROWS * 16;
};

template <AttendKind K, typename T, int VE, int NV, int G, int U>
__global__ void __launch_bounds__(RING_WARPS * 32) k_attend_ring(const __grid_constant__ Attend P) {
    using S = RingShape<K, T, VE, NV, G, U>;
    constexpr int E = VE * NV, N2 = E / 2, PB = S::PB, SZ = (int)sizeof(T);
    constexpr bool SHIFTED = rounded_out<T>;                                      // delta of the dq pass lacks P.shift
    extern __shared__ __align__(16) unsigned char ring_smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned char* mine = ring_smem + (size_t)warp * S::WARP;
    int4* rows_s = reinterpret_cast<int4*>(mine + RING_SLOTS * S::SLOT);           // begin, end, row, item (or -1: listed as long)
    const uint32_t mine_a = (uint32_t)__cvta_generic_to_shared(mine);
    const int tl = P.tl, t = lane & (tl - 1), gpw = 32 / tl, upr = P.units_per_row;
    const int rows = P.chunk_mode ? __ldcg(P.words) : length_of(P.rows), cols = length_of(P.columns);
    const int64_t units = (int64_t)rows * upr;
    const float c2 = P.a.scale * LOG2E;
    const int D = P.a.head_dim, group = P.a.q_heads / P.a.kv_heads;
    const int passes = K == AT_DKV ? group / G : 1;                                 // walks over a row's edges
    const HeadView& av = K == AT_DKV ? P.a.q : P.a.k;                               // the edges' two operands
    const HeadView& bv = K == AT_DKV ? P.a.dout : P.a.v;
    const uint32_t astep = (uint32_t)av.row_stride * SZ, bstep = (uint32_t)bv.row_stride * SZ;   // below 2^32 by the choice of kernel
    const uint32_t ahead_step = (uint32_t)av.head_stride * SZ, bhead_step = (uint32_t)bv.head_stride * SZ;
    const char* abase = (const char*)av.data + t * PB;
    const char* bbase = (const char*)bv.data + t * PB;
    const int tshift = 31 - __clz(tl), ushift = (upr & (upr - 1)) == 0 ? 31 - __clz(upr) : -1;
    // byte strides of the rows' own operands and of the results
    auto stride32 = [](const HeadView& v) { return (uint32_t)v.row_stride * SZ; };
    const HeadView& r0v = P.a.q;
    const HeadView& r1v = P.a.dout;
    const HeadView& o0v = K == AT_FORWARD ? P.a.out : (K == AT_DQ ? P.a.dq : P.a.dk);
    const HeadView& o1v = P.a.dv;
    const uint32_t r0step = stride32(r0v), r1step = stride32(r1v), o0step = stride32(o0v), o1step = stride32(o1v), outstep = stride32(P.a.out);
    int size[NV];                                                                   // bytes of this lane's pieces: 0 behind the row's end
#pragma unroll
    for (int n = 0; n < NV; ++n) size[n] = (t + n * tl) * VE < D ? PB : 0;
    enum : uint32_t { LIVE = 1, FIRST = 2, LAST = 4, HEAD = 8, EDGES = 15 << 4 };                    // a batch: flags | edges << 4 | local row << 8 | head << 16 | walk << 24

    // a warp takes P.tiles tiles of gpw consecutive units at a time
    const int64_t span = (int64_t)P.tiles * gpw;
    for (int64_t u0 = ((int64_t)blockIdx.x * RING_WARPS + warp) * span; u0 < units; u0 += (int64_t)gridDim.x * RING_WARPS * span) {
        const int r0 = (int)(u0 / upr), off = (int)(u0 - (int64_t)r0 * upr);
        const int left = (int)(units - u0 < span ? units - u0 : span);
        const int nrows = (off + left + upr - 1) / upr;                             // at most RING_ROWS by the choice of P.tiles
        __syncwarp();
        for (int i = lane; i < nrows; i += 32) {
            int row = r0 + i, item = 0, first = 0;
            if (P.chunk_mode) {
                const int2 it = P.items[row];
                item = row;
                row = it.x;
                first = it.y * AT_CHUNK;
            }
            int b = __ldg(P.starts + row), e = __ldg(P.starts + row + 1);
            b = b < 0 ? 0 : b;
            e = e > P.edge_bound ? P.edge_bound : e;
            if (e < b) e = b;
            if (P.chunk_mode) {
                b += first;
                e = b + AT_CHUNK < e ? b + AT_CHUNK : e;
            } else if (P.split && e - b > AT_CHUNK) {
                // listed once: by the warp that holds the row's first unit
                if (i > 0 || off == 0) list_long_row(P, row, e - b);
                e = b;
                item = -1;
            }
            rows_s[i] = make_int4(b, e, row, item);
        }
        __syncwarp();

        // ---- the producer's position: unit, row, walk and next edge of this group.  A group that has finished its unit takes
        // the warp's next one, so that long rows do not hold up the others; the heads of a row stay side by side.
        int next_unit = 0, e_next = 0, e_end = 0, pass = 0, lr = 0, head = -1;
        bool fresh = true, walk = true;
        const char* ap = abase;                              // this lane's first piece in row 0 of the edges' operands
        const char* bp = bbase;
        uint32_t next = 0;
        int idx[U], edge[U];                                 // the batch whose indices are on their way; dkv: its edges, dq: the first
        auto fetch = [&]() {
            next = 0;
#pragma unroll
            for (int j = 0; j < U; ++j) idx[j] = -1;
            for (;;) {
                const uint32_t want = __ballot_sync(FULL, fresh);
                if (!want || next_unit >= left) break;
                const int lu = next_unit + (__popc(want & ((1u << (lane - t)) - 1u)) >> tshift);
                next_unit += __popc(want) >> tshift;
                if (fresh && lu < left) {
                    const int v = off + lu, last = head;
                    lr = ushift >= 0 ? v >> ushift : v / upr;
                    head = v - lr * upr;
                    const int4 r = rows_s[lr];
                    walk = walk || head != last;
                    if (K == AT_DKV && r.y <= r.x) {
                        // a source that no destination lists: zeros at once (a listed long row: nothing)
                        if (r.w >= 0 && !P.chunk_mode) {
                            const float zero[E] = {};
                            store_piece<T, VE, NV>((T*)((char*)o0v.data + (uint64_t)(uint32_t)r.z * o0step) + head * (int)o0v.head_stride, t, tl, D, zero);
                            store_piece<T, VE, NV>((T*)((char*)o1v.data + (uint64_t)(uint32_t)r.z * o1step) + head * (int)o1v.head_stride, t, tl, D, zero);
                        }
                    } else {
                        e_next = r.x;
                        e_end = r.y;
                        pass = 0;
                        next = FIRST;
                        fresh = false;
                    }
                }
            }
            if (fresh) return;                               // nothing left for this group
            if (walk) next |= HEAD;
            walk = false;
            const int32_t* c = P.cols + e_next;
#pragma unroll
            for (int j = 0; j < U; ++j)
                if (e_next + j < e_end) {
                    idx[j] = __ldg(c + j);
                    if (K == AT_DKV) edge[j] = __ldg(P.edges + e_next + j);
                }
            if (K == AT_DQ) edge[0] = e_next;
            next |= LIVE | (uint32_t)lr << 8 | (uint32_t)head << 16 | (uint32_t)pass << 24;
            e_next += U;
            if (e_next >= e_end) {
                if (K == AT_DKV && passes > 1 && ++pass < passes && e_end > rows_s[lr].x) {
                    e_next = rows_s[lr].x;
                    walk = true;
                } else {
                    next |= LAST;
                    walk = passes > 1;
                    fresh = true;
                }
            }
        };
        // the copies of the batch whose indices have arrived; returns its description
        int h0 = 0;
        float shift[U * G];                                  // dkv: what the edges' destinations add to delta
        auto issue = [&](int slot) -> uint32_t {
            uint32_t batch = next;
            const uint32_t base = mine_a + slot * S::SLOT, lp = base + lane * PB;
            const int hd = (batch >> 16) & 255;
            if (batch & HEAD) {
                h0 = K == AT_DKV ? hd * group + (int)(batch >> 24) * G : hd * G;
                const int he = K == AT_DKV ? h0 : (group == G ? hd : h0 / group);
                ap = abase + (uint64_t)he * ahead_step;
                bp = bbase + (uint64_t)he * bhead_step;
            }
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const bool on = (uint32_t)idx[j] < (uint32_t)cols && (K != AT_DKV || (uint32_t)edge[j] < (uint32_t)P.edge_bound);
                const uint32_t col = on ? idx[j] : 0;
                batch |= on ? 16u << j : 0u;
                const char* a = ap + (uint64_t)col * astep;
                const char* b = bp + (uint64_t)col * bstep;
#pragma unroll
                for (int i = 0; i < (K == AT_DKV ? G : 1); ++i)
#pragma unroll
                    for (int n = 0; n < NV; ++n) {
                        const uint32_t to = lp + (uint32_t)(j * S::EDGE + i * 2 * NV + n) * 32 * PB;
                        const int sz = on ? size[n] : 0;
                        const uint32_t off_n = sz ? n * tl * PB : 0;
                        copy_async<PB>(to, a + i * ahead_step + off_n, sz);
                        copy_async<PB>(to + NV * 32 * PB, b + i * bhead_step + off_n, sz);
                    }
                if (K == AT_DKV) {
#pragma unroll
                    for (int i = 0; i < G; ++i)
                        copy_async<8>(base + S::PIECES + ((j * G + i) * 32 + lane) * 8, P.pd + (uint64_t)(on ? edge[j] : 0) * P.a.q_heads + h0 + i, on ? 8 : 0);
                    if (SHIFTED) load_shifts<G>(P.shift + (uint64_t)col * P.a.q_heads + h0, on, &shift[j * G]);
                }
            }
            if (K != AT_DKV && (batch & FIRST)) {
                const int4 r = rows_s[(batch >> 8) & 255];
                auto rowcopy = [&](const HeadView& v, uint32_t step, int h, int piece) {
                    const char* p = (const char*)v.data + (uint64_t)(uint32_t)r.z * step + (uint32_t)(h * (int)v.head_stride * SZ);
#pragma unroll
                    for (int n = 0; n < NV; ++n)
                        copy_async<PB>(lp + (uint32_t)(U * S::EDGE + piece + n) * 32 * PB, size[n] ? p + (t + n * tl) * PB : p, size[n]);
                };
#pragma unroll
                for (int i = 0; i < G; ++i) {
                    rowcopy(r0v, r0step, h0 + i, i * NV);
                    if (K == AT_DQ) {
                        rowcopy(r1v, r1step, h0 + i, (G + i) * NV);
                        rowcopy(P.a.out, outstep, h0 + i, (2 * G + i) * NV);
                        copy_async<4>(base + S::PIECES + (i * 32 + lane) * 4, P.a.lse + (int64_t)r.z * P.a.q_heads + h0 + i, 4);
                    }
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            return batch;
        };
        auto pieces = [&](int slot, int p, f32x2 (&x)[N2]) {
#pragma unroll
            for (int n = 0; n < NV; ++n) {
                Raw<T, VE> r;
                float y[VE];
                r.w = *reinterpret_cast<const typename Raw<T, VE>::word*>(mine + slot * S::SLOT + (size_t)(p + n) * 32 * PB + lane * PB);
                unpack<T, VE>(r, y);
#pragma unroll
                for (int c = 0; c < VE / 2; ++c) x[n * VE / 2 + c] = pair(y[2 * c], y[2 * c + 1]);
            }
        };

        // what a unit keeps from batch to batch
        constexpr int NX = K == AT_DKV ? 1 : G, NA = K == AT_DKV ? 2 : G;
        f32x2 x0[K == AT_DKV ? 1 : NX][K == AT_DKV ? 1 : N2], x1[K == AT_DQ ? NX : 1][K == AT_DQ ? N2 : 1];   // q; q, dout
        f32x2 acc[NA][N2];                                                           // out; dq; dk, dv
        float m[G], l[G];                                                            // running maximum and sum; lse (base 2), delta
        f32x2 kp[K == AT_DQ && SHIFTED ? G : 1][K == AT_DQ && SHIFTED ? N2 : 1];     // dq: sum of p k
        float miss[G];                                                               // and of p (dp - delta): 0 but for delta's rounding
        if constexpr (K != AT_DKV) {
#pragma unroll
            for (int i = 0; i < NX; ++i)
#pragma unroll
                for (int c = 0; c < N2; ++c) {
                    x0[i][c] = 0;
                    if constexpr (K == AT_DQ) x1[i][c] = 0;
                }
        }
#pragma unroll
        for (int i = 0; i < NA; ++i)
#pragma unroll
            for (int c = 0; c < N2; ++c) acc[i][c] = 0;
#pragma unroll
        for (int i = 0; i < G; ++i) m[i] = l[i] = 0.f;

        uint32_t batches[RING_DEPTH];
        int first_edge[K == AT_DQ ? RING_DEPTH : 1];         // dq: where p and ds of a batch's edges go
        constexpr int NS = K == AT_DKV && SHIFTED ? U * G : 1;
        float shifts[RING_DEPTH][NS];
        auto keep_shifts = [&](int s) {
            if constexpr (K == AT_DKV && SHIFTED) {
#pragma unroll
                for (int i = 0; i < NS; ++i) shifts[s][i] = shift[i];
            }
        };
        fetch();
#pragma unroll
        for (int s = 0; s < RING_DEPTH; ++s) {
            batches[s] = issue(s);
            keep_shifts(s);
            if (K == AT_DQ) first_edge[s] = edge[0];
            fetch();
        }
        int slot = 0, ahead = RING_DEPTH;
        while (__any_sync(FULL, batches[0] & LIVE)) {
            const uint32_t batch = batches[0];
            const int my_edge = first_edge[0];
            float my_shift[NS];
#pragma unroll
            for (int i = 0; i < NS; ++i) my_shift[i] = shifts[0][i];
#pragma unroll
            for (int s = 0; s + 1 < RING_DEPTH; ++s) {
                batches[s] = batches[s + 1];
#pragma unroll
                for (int i = 0; i < NS; ++i) shifts[s][i] = shifts[s + 1][i];
                if (K == AT_DQ) first_edge[s] = first_edge[s + 1];
            }
            batches[RING_DEPTH - 1] = issue(ahead);
            keep_shifts(RING_DEPTH - 1);
            if (K == AT_DQ) first_edge[RING_DEPTH - 1] = edge[0];
            fetch();
            asm volatile("cp.async.wait_group %0;" ::"n"(RING_DEPTH) : "memory");
            const int h = (batch >> 16) & 255;
            auto on = [&](int j) { return (batch >> (4 + j)) & 1; };
            if constexpr (K == AT_FORWARD) {
                if (batch & FIRST) {
#pragma unroll
                    for (int i = 0; i < G; ++i) {
                        pieces(slot, U * S::EDGE + i * NV, x0[i]);
                        m[i] = -INFINITY;
                        l[i] = 0.f;
#pragma unroll
                        for (int c = 0; c < N2; ++c) acc[i][c] = 0;
                    }
                }
                float s[U * G];
#pragma unroll
                for (int j = 0; j < U; ++j) {
                    f32x2 k[N2];
                    pieces(slot, j * S::EDGE, k);
#pragma unroll
                    for (int i = 0; i < G; ++i) s[j * G + i] = dot2(x0[i], k);
                }
                ring_sum<U * G>(s, tl);
                float p[U * G];
#pragma unroll
                for (int i = 0; i < G; ++i) {
                    float top = m[i];
#pragma unroll
                    for (int j = 0; j < U; ++j) {
                        s[j * G + i] = on(j) ? s[j * G + i] * c2 : -INFINITY;
                        top = fmaxf(top, s[j * G + i]);
                    }
                    const float ref = top == -INFINITY ? 0.f : top;
                    const float corr = fast_exp2(m[i] - ref);
                    m[i] = top;
                    l[i] *= corr;
#pragma unroll
                    for (int j = 0; j < U; ++j) {
                        p[j * G + i] = fast_exp2(s[j * G + i] - ref);
                        l[i] += p[j * G + i];
                    }
                    scale2(corr, acc[i]);
                }
#pragma unroll
                for (int j = 0; j < U; ++j) {
                    f32x2 v[N2];
                    pieces(slot, j * S::EDGE + NV, v);
#pragma unroll
                    for (int i = 0; i < G; ++i) axpy2(p[j * G + i], v, acc[i]);
                }
                if (batch & LAST) {
                    const int4 rw = rows_s[(batch >> 8) & 255];
                    if (rw.w >= 0) {
#pragma unroll
                        for (int i = 0; i < G; ++i) {
                            const int hh = h * G + i;
                            float o[E];
                            unpair(acc[i], o);
                            if (P.chunk_mode) {
                                float* part = P.partial + ((int64_t)rw.w * P.a.q_heads + hh) * (D + 2);
                                store_partial<VE, NV>(part, t, tl, D, o);
                                if (t == 0) {
                                    part[D] = m[i];
                                    part[D + 1] = l[i];
                                }
                            } else {
                                const bool none = l[i] == 0.f;
                                const float inv = none ? 0.f : 1.f / l[i];
#pragma unroll
                                for (int c = 0; c < E; ++c) o[c] = none ? 0.f : o[c] * inv;
                                store_piece<T, VE, NV>((T*)((char*)o0v.data + (uint64_t)(uint32_t)rw.z * o0step) + hh * (int)o0v.head_stride, t, tl, D, o);
                                if (t == 0) P.a.lse[(int64_t)rw.z * P.a.q_heads + hh] = none ? -INFINITY : m[i] * LN2 + logf(l[i]);
                            }
                        }
                    }
                }
            } else if constexpr (K == AT_DQ) {
                if (__any_sync(FULL, batch & FIRST)) {
                    float delta[G];
#pragma unroll
                    for (int i = 0; i < G; ++i) delta[i] = 0.f;
                    if (batch & FIRST) {
#pragma unroll
                        for (int i = 0; i < G; ++i) {
                            f32x2 o[N2];
                            pieces(slot, U * S::EDGE + i * NV, x0[i]);
                            pieces(slot, U * S::EDGE + (G + i) * NV, x1[i]);
                            pieces(slot, U * S::EDGE + (2 * G + i) * NV, o);
                            m[i] = backward_lse(*reinterpret_cast<const float*>(mine + slot * S::SLOT + S::PIECES + (i * 32 + lane) * 4));
                            delta[i] = dot2(x1[i], o);
#pragma unroll
                            for (int c = 0; c < N2; ++c) acc[i][c] = 0;
                            if constexpr (SHIFTED) {
                                miss[i] = 0.f;
#pragma unroll
                                for (int c = 0; c < N2; ++c) kp[i][c] = 0;
                            }
                        }
                    }
                    __syncwarp();
                    ring_sum<G>(delta, tl);
                    if (batch & FIRST) {
#pragma unroll
                        for (int i = 0; i < G; ++i) l[i] = delta[i];
                    }
                    __syncwarp();
                }
#pragma unroll
                for (int i = 0; i < G; ++i)
                    if (m[i] == INFINITY && (batch & EDGES)) *P.look = 1;       // edges, but no weights
                float s[2 * U * G];
#pragma unroll
                for (int j = 0; j < U; ++j) {
                    f32x2 k[N2], v[N2];
                    pieces(slot, j * S::EDGE, k);
                    pieces(slot, j * S::EDGE + NV, v);
#pragma unroll
                    for (int i = 0; i < G; ++i) {
                        s[j * G + i] = dot2(x0[i], k);
                        s[U * G + j * G + i] = dot2(x1[i], v);
                    }
                }
                ring_sum<2 * U * G>(s, tl);
#pragma unroll
                for (int j = 0; j < U; ++j) {
                    f32x2 k[N2];
                    pieces(slot, j * S::EDGE, k);
#pragma unroll
                    for (int i = 0; i < G; ++i) {
                        const float p = on(j) ? fast_exp2(fmaf(s[j * G + i], c2, -m[i])) : 0.f;
                        const float ds = on(j) ? p * (s[U * G + j * G + i] - l[i]) : 0.f;
                        axpy2(ds, k, acc[i]);
                        if constexpr (SHIFTED) {
                            axpy2(p, k, kp[i]);
                            miss[i] += ds;
                        }
                        if (on(j) && t == 0) P.pd[(int64_t)(my_edge + j) * P.a.q_heads + h * G + i] = make_float2(p, ds);
                    }
                }
                if (batch & LAST) {
                    const int4 rw = rows_s[(batch >> 8) & 255];
                    if (rw.w >= 0) {
#pragma unroll
                        for (int i = 0; i < G; ++i) {
                            const int hh = h * G + i;
                            if (!all_finite(acc[i])) *P.look = 1;
                            float o[E];
                            if (P.chunk_mode) {
                                float* part = P.partial + ((int64_t)rw.w * P.a.q_heads + hh) * dq_part<T>(D);
                                unpair(acc[i], o);
                                store_partial<VE, NV>(part, t, tl, D, o);
                                if constexpr (SHIFTED) {
                                    unpair(kp[i], o);
                                    store_partial<VE, NV>(part + D, t, tl, D, o);
                                    if (t == 0) part[2 * D] = miss[i];
                                }
                                continue;
                            }
                            if constexpr (SHIFTED) {
                                axpy2(-miss[i], kp[i], acc[i]);
                                if (t == 0) P.shift[(int64_t)rw.z * P.a.q_heads + hh] = miss[i];
                            }
                            scale2(P.a.scale, acc[i]);
                            unpair(acc[i], o);
                            store_piece<T, VE, NV>((T*)((char*)o0v.data + (uint64_t)(uint32_t)rw.z * o0step) + hh * (int)o0v.head_stride, t, tl, D, o);
                        }
                    }
                }
            } else {
                if (batch & FIRST) {
#pragma unroll
                    for (int c = 0; c < N2; ++c) acc[0][c] = acc[1][c] = 0;
                }
#pragma unroll
                for (int j = 0; j < U; ++j)
#pragma unroll
                    for (int i = 0; i < G; ++i) {            // what is not an edge was filled with zeros
                        f32x2 q[N2], go[N2];
                        pieces(slot, j * S::EDGE + i * 2 * NV, q);
                        pieces(slot, j * S::EDGE + i * 2 * NV + NV, go);
                        const float2 pd = *reinterpret_cast<const float2*>(mine + slot * S::SLOT + S::PIECES + ((j * G + i) * 32 + lane) * 8);
                        axpy2(pd.x, go, acc[1]);
                        axpy2(SHIFTED ? fmaf(-pd.x, my_shift[SHIFTED ? j * G + i : 0], pd.y) : pd.y, q, acc[0]);
                    }
                if (batch & LAST) {
                    const int4 rw = rows_s[(batch >> 8) & 255];
                    if (rw.w >= 0) {
                        if (!P.chunk_mode) scale2(P.a.scale, acc[0]);
                        float dk[E], dv[E];
                        unpair(acc[0], dk);
                        unpair(acc[1], dv);
                        if (P.chunk_mode) {
                            float* part = P.partial + ((int64_t)rw.w * P.a.kv_heads + h) * 2 * D;
                            store_partial<VE, NV>(part, t, tl, D, dk);
                            store_partial<VE, NV>(part + D, t, tl, D, dv);
                        } else {
                            store_piece<T, VE, NV>((T*)((char*)o0v.data + (uint64_t)(uint32_t)rw.z * o0step) + h * (int)o0v.head_stride, t, tl, D, dk);
                            store_piece<T, VE, NV>((T*)((char*)o1v.data + (uint64_t)(uint32_t)rw.z * o1step) + h * (int)o1v.head_stride, t, tl, D, dv);
                        }
                    }
                }
            }
            __syncwarp();
            slot = slot + 1 == RING_SLOTS ? 0 : slot + 1;
            ahead = ahead + 1 == RING_SLOTS ? 0 : ahead + 1;
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
    }
}

}  // namespace gs
