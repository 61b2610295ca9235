// Attention over rows in 8 bits for bf16 queries, four or more of whose heads share a key head: the products on the tensor cores.
//
// A warp owns one (row, four query heads of one key head: the "slots") at a time and takes its edges 16 at a time.  The codes are
// e4m3 numbers, exact as f16, and so is a bf16 query once it is scaled by a power of two (one that has an element other than zero 2^31
// below its largest is found when it is scaled, and its units are done again at the warp's end, edge by edge in 32 bits):
//   scores:  C[16 edges][slots] += K[16 edges][16 columns] q^T   (m16n8k16, sums in 32 bits; slot t is column 2 t, in lane t of a quad)
//   values:  acc[slots][columns] += P[slots][16 edges] V[16 edges][8 columns]
// P is not rounded to f16: a weight is hi + 2^-11 lo, two rows of the matrix, to 2^-23 of itself.  The weights carry their value block's
// scale; they are held relative to a power of two near the largest weight times scale so far, as 2^14.  f16 ends 2^-38 below that, and
// yet such weights are the result where the heavier edges' values are zero: a tile that has weights below 2^-26 multiplies those
// again by themselves, they and the sums brought up together, down to 2^-98 of the largest.  It takes a score 18 below a row's largest.  A unit
// with lighter weights still (a score 68 below; 32 bits end at 87) and a column next to zero is done again at the warp's end, edge by edge
// in 32 bits.
// What bounds it is instructions around the products (64 columns: ALU 54 %, issue slots 62 %; 513 a row and 427 a tile), not their rate, so
// the legacy matrix instruction serves.  Above 128 columns one block of four warps fits an SM, and latency bounds it (issue slots 23 %).
// Spills, bytes loaded: 88 for 65 to 128 columns, 108 above, none below.  This : the other kernel (2 x 4 heads): one row of 200,011 edges,
// 64 columns 47 : 112 us, 16 columns 42 : 52; 4,096 rows of up to 300, 64 columns 353 : 519.  Rows of few edges do not fill a tile: which go
// where, with both sides' figures, is at the dispatch.  With fewer shared heads the other kernel needs fewer instructions (2 of 32 columns, 20
// edges 314 : 258; 1 of 32, 20 edges 527 : 284; one row of 200,011 edges 44 : 43).
//
// Rows are gathered by cp.async into TC_STAGES buffers of 16 edges a warp, TC_STAGES - 1 tiles ahead; the columns of 32 edges are read
// one unit (a row's first) and the offsets two units ahead of the gathers.  No block barriers.  16-byte pieces are permuted within
// 128 bytes by the edge so that every fragment is read without bank conflicts (up to 128 columns).
#pragma once

namespace gs {

constexpr int TC_STAGES = 3;
constexpr int TC_WARPS = 4;
constexpr int TC_MOST = 72;                   // the largest power that sums are brought up by: those of 2^30 edges stay within 32 bits
constexpr float TC_GONE = 0x1p-120f;          // weights that are not whole in 32 bits
constexpr uint32_t TC_AGAIN = 0x7FC0A6A1u;    // a NaN that no arithmetic gives, in the place of a unit's lse: its weights are too far apart
constexpr float TC_NEAR = 1.f / 4096.f;       // weights (the largest is 2^14) whose two parts hold 2^-23 of them

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Rows 0 to 7 of the product are added to c; a has no others.
__device__ __forceinline__ void mma_f16_half(float (&c)[2], uint32_t a0, uint32_t a2, uint32_t b0, uint32_t b1) {
    float d[4];
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %5}, {%7, %8}, {%9, %10, %11, %11};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a0), "r"(0), "r"(a2), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(0.f));
    c[0] = d[0];
    c[1] = d[1];
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t codes_to_f16(uint32_t two) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)two));
    return h;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float f16_lo(uint32_t x) {
    float y;
    asm("{.reg .f16 a, b;\n\tmov.b32 {a, b}, %1;\n\tcvt.f32.f16 %0, a;}" : "=f"(y) : "r"(x));
    return y;
}
// 2^e; 0 below the range of f32 (and its largest power above: of no number that is not zero).
__device__ __forceinline__ float power_of(int e) { return __uint_as_float((uint32_t)(min(max(e, -127), 127) + 127) << 23); }
// Place of byte `at` of an edge's row in a buffer of 16 edges.
__device__ __forceinline__ int tile_byte(int edge, int at) {
    const int c = (((edge & 1) << 1) | ((edge >> 1) & 1)) ^ ((edge >> 2 & 1) << 1), key = c << 1 | (edge & 1);
    return (at >> 7) * 2048 + edge * 128 + ((((at >> 4) & 7) ^ key) << 4) + (at & 15);
}
template <int WORDS> __device__ __forceinline__ void read_words(const unsigned char* tile, int edge, int at, uint32_t (&w)[WORDS]) {
    if constexpr (WORDS == 1) {
        w[0] = *reinterpret_cast<const uint32_t*>(tile + tile_byte(edge, at));
    } else if constexpr (WORDS == 2) {
        const uint2 x = *reinterpret_cast<const uint2*>(tile + tile_byte(edge, at));
        w[0] = x.x; w[1] = x.y;
    } else {
#pragma unroll
        for (int i = 0; i < WORDS / 4; ++i) {
            const uint4 x = *reinterpret_cast<const uint4*>(tile + tile_byte(edge, at + i * 16));
            w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w;
        }
    }
}

// Two weights of slot t, of the edges g and g + 8, as an operand whose rows 2 slot are f16 and rows 2 slot + 1 the rest times 2^11.
__device__ __forceinline__ uint2 split_weights(float x0, float x1) {
    const float hi0 = f16_lo(pack_f16(x0, 0.f)), hi1 = f16_lo(pack_f16(x1, 0.f));
    return make_uint2(transpose8(pack_f16(x0, (x0 - hi0) * 2048.f)), transpose8(pack_f16(x1, (x1 - hi1) * 2048.f)));
}
// The products of weights and a tile's values: edges 2 t, 2 t + 1, 2 t + 8, 2 t + 9, columns 2 SP g ...; mma(i, weights, values) for column i of them.
template <int SP, typename M> __device__ __forceinline__ void multiply_values(const unsigned char* vt, uint2 a, M mma) {
    const int t = threadIdx.x & 3, byte = ((threadIdx.x & 31) >> 2) * 2 * SP;
    if constexpr (SP == 1) {
        auto two = [&](int edge) { return (uint32_t)*reinterpret_cast<const uint16_t*>(vt + tile_byte(edge, byte)); };
        const uint32_t low = __byte_perm(two(2 * t), two(2 * t + 1), 0x5140), high = __byte_perm(two(2 * t + 8), two(2 * t + 9), 0x5140);
        mma(0, a, codes_to_f16(low), codes_to_f16(high));
        mma(1, a, codes_to_f16(low >> 16), codes_to_f16(high >> 16));
    } else {
        constexpr int VW = SP / 2;
        uint32_t v0[VW], v1[VW], v2[VW], v3[VW];
        read_words<VW>(vt, 2 * t, byte, v0);
        read_words<VW>(vt, 2 * t + 1, byte, v1);
        read_words<VW>(vt, 2 * t + 8, byte, v2);
        read_words<VW>(vt, 2 * t + 9, byte, v3);
#pragma unroll
        for (int i = 0; i < VW; ++i) {
            const uint32_t la = __byte_perm(v0[i], v1[i], 0x5140), lb = __byte_perm(v0[i], v1[i], 0x7362);
            const uint32_t ha = __byte_perm(v2[i], v3[i], 0x5140), hb = __byte_perm(v2[i], v3[i], 0x7362);
            mma(4 * i, a, codes_to_f16(la), codes_to_f16(ha));
            mma(4 * i + 1, a, codes_to_f16(la >> 16), codes_to_f16(ha >> 16));
            mma(4 * i + 2, a, codes_to_f16(lb), codes_to_f16(hb));
            mma(4 * i + 3, a, codes_to_f16(lb >> 16), codes_to_f16(hb >> 16));
        }
    }
}

// SP: 16 columns each (a power of two).
template <int SP> struct TcShape {
    static constexpr int SLOTS = 4, ROWB = SP > 8 ? 256 : 128, TILE = 16 * ROWB, Q = SLOTS * SP * 32;
    static constexpr int STAGE = 2 * TILE + Q, WARP = TC_STAGES * STAGE, SMEM = TC_WARPS * WARP;
};

struct TcUnit {
    int r, row, unit, begin, end;    // r: the row, or the chunk
    bool live;
};

// Whether f16 keeps the 8 bits of all elements, given the bf16 bits of the largest and of the smallest that is not zero, less one: the
// largest is scaled to 2^14 (see up_of), and 2^-17 is the least that f16 has 8 bits of.
__device__ __forceinline__ int up_of(uint32_t top) {         // exponent, with its bias, of the power that does so, within the range of f32
    const int e = (int)(top >> 7);
    return e < 15 ? 253 : (e > 253 ? 15 : 268 - e);
}
__device__ __forceinline__ bool too_wide(uint32_t top, uint32_t least) { return least < 0x7F80u && (int)((least + 1) >> 7) + up_of(top) < 237; }

// The units of a warp whose queries are too wide for f16, or which are marked, in 32 bits throughout: a lane has every 32nd column.  100,000
// rows of 20 edges, 4 x 4 heads of 64: all queries too wide 4,830 us, none 820; scores spread by 8 1,020, by 32 1,660.
template <int SP> __device__ __noinline__ void attend_again(const CodedAttend& P, int64_t units) {
    constexpr int SLOTS = 4, C = (SP + 1) / 2;
    const int lane = threadIdx.x & 31, D = P.a.head_dim, group = P.a.q_heads / P.a.kv_heads, cols = list_length(P.a.src);
    const float c2 = P.a.scale * CA_LOG2E;
    for (int64_t u = (int64_t)blockIdx.x * TC_WARPS + (threadIdx.x >> 5); u < units; u += (int64_t)gridDim.x * TC_WARPS) {
        const int r = (int)(u / P.units_per_row), h0 = (int)(u - (int64_t)r * P.units_per_row) * SLOTS, kv = h0 / group;
        const int2 it = P.chunk_mode ? P.items[r] : make_int2(r, 0);
        float q[SLOTS][C], acc[SLOTS][C], m[SLOTS], l[SLOTS];
        const float* mark = P.chunk_mode ? P.partial + ((int64_t)r * P.a.q_heads + h0) * (D + 2) + D : P.a.lse + (int64_t)it.x * P.a.q_heads + h0;
        bool again = __float_as_uint(*mark) == TC_AGAIN;
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) {
            const bf16* row = (const bf16*)P.a.q.data + (int64_t)it.x * P.a.q.row_stride + (int64_t)(h0 + i) * P.a.q.head_stride;
            uint32_t top = 0, least = 0xFFFFu;
#pragma unroll
            for (int j = 0; j < C; ++j) {
                q[i][j] = lane + 32 * j < D ? to_f32(row[lane + 32 * j]) : 0.f;
                acc[i][j] = 0.f;
                const uint32_t bits = (__float_as_uint(q[i][j]) >> 16) & 0x7FFFu;
                if (bits <= 0x7F80u) top = max(top, bits);
                least = min(least, (bits - 1) & 0xFFFFu);
            }
            again |= too_wide(__reduce_max_sync(FULL, top), __reduce_min_sync(FULL, least));
            m[i] = -INFINITY;
            l[i] = 0.f;
        }
        int begin = max(__ldg(P.a.indptr + it.x), 0), end = min(__ldg(P.a.indptr + it.x + 1), P.a.edge_bound);
        if (!again || (!P.chunk_mode && P.split && end - begin > CA_LONG)) continue;
        if (P.chunk_mode) {
            begin += it.y * P.chunk;
            end = min(end, begin + P.chunk);
        }
        for (int e = begin; e < end; ++e) {
            int at = __ldg(P.a.indices + e);
            if ((uint32_t)at >= (uint32_t)cols) continue;
            if (P.a.row_of) at = __ldg(P.a.row_of + at);
            if ((uint32_t)at >= (uint32_t)P.a.k.rows) continue;
            const uint8_t* k = P.a.k.codes + (uint64_t)(uint32_t)at * (uint32_t)P.a.k.row_stride + (int64_t)kv * P.a.k.pitch;
            const uint8_t* v = P.a.v.codes + (uint64_t)(uint32_t)at * (uint32_t)P.a.v.row_stride + (int64_t)kv * P.a.v.pitch;
            const float ks = scale_of(P.a.k.scales[(uint64_t)((uint32_t)at >> P.a.k.shift) * (uint32_t)P.a.k.scale_stride + kv]);
            const float vs = scale_of(P.a.v.scales[(uint64_t)((uint32_t)at >> P.a.v.shift) * (uint32_t)P.a.v.scale_stride + kv]);
            float x[C], s[SLOTS] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < C; ++j) {
                const bool is = lane + 32 * j < D;
                const float y = is ? decode1(k[lane + 32 * j]) : 0.f;
                x[j] = is ? decode1(v[lane + 32 * j]) : 0.f;
#pragma unroll
                for (int i = 0; i < SLOTS; ++i) s[i] = fmaf(q[i][j], y, s[i]);
            }
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
                for (int o = 16; o; o >>= 1) s[i] += __shfl_xor_sync(FULL, s[i], o);
                s[i] = s[i] * ks * c2;
                const float top = fmaxf(m[i], s[i]), ref = top == -INFINITY ? 0.f : top, corr = exp2_fast(m[i] - ref), p = exp2_fast(s[i] - ref);
                m[i] = top;
                l[i] = fmaf(l[i], corr, p);
#pragma unroll
                for (int j = 0; j < C; ++j) acc[i][j] = fmaf(p * vs, x[j], acc[i][j] * corr);
            }
        }
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) {
            const int h = h0 + i;
            const bool none = l[i] == 0.f;
            float* part = P.partial + ((int64_t)r * P.a.q_heads + h) * (D + 2);
            bf16* to = (bf16*)P.a.out.data + (int64_t)it.x * P.a.out.row_stride + (int64_t)h * P.a.out.head_stride;
#pragma unroll
            for (int j = 0; j < C; ++j) {
                const int c = lane + 32 * j;
                if (c >= D) continue;
                if (P.chunk_mode) part[c] = acc[i][j];
                else to[c] = from_f32<bf16>(none ? 0.f : acc[i][j] / l[i]);
            }
            if (lane) continue;
            if (P.chunk_mode) {
                part[D] = m[i];
                part[D + 1] = l[i];
            } else {
                P.a.lse[(int64_t)it.x * P.a.q_heads + h] = none ? -INFINITY : m[i] * CA_LN2 + logf(l[i]);
            }
        }
    }
}

template <int SP> __global__ void __launch_bounds__(TC_WARPS * 32, SP >= 16 ? 1 : (SP >= 8 ? 3 : 4)) k_coded_attend_tc(const __grid_constant__ CodedAttend P) {
    using S = TcShape<SP>;
    constexpr int SLOTS = S::SLOTS, L = 4 * SP, TILES = 2 * SP, PIECES = SP;
    extern __shared__ __align__(16) unsigned char tc_smem[];
    chain_wait();
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int rows = P.chunk_mode ? listed_chunks(P) : list_length(P.a.dst), cols = list_length(P.a.src);
    const int64_t units = (int64_t)rows * P.units_per_row, step = (int64_t)gridDim.x * TC_WARPS;
    const int D = P.a.head_dim, group = P.a.q_heads / P.a.kv_heads, pitch = P.a.k.pitch;
    const uint32_t kstep = (uint32_t)P.a.k.row_stride, vstep = (uint32_t)P.a.v.row_stride;
    const CodedView& SV = lane < 16 ? P.a.k : P.a.v;         // whose scales this lane fetches
    const uint32_t sstep = (uint32_t)SV.scale_stride;
    unsigned char* mine = tc_smem + (threadIdx.x >> 5) * S::WARP;
    const uint32_t mine_a = (uint32_t)__cvta_generic_to_shared(mine);

    // ---- units: offsets two units ahead, columns one
    int64_t u = (int64_t)blockIdx.x * TC_WARPS + (threadIdx.x >> 5);
    if (u >= units) return;
    auto raw_unit = [&](int64_t u) {
        TcUnit w{0, 0, 0, 0, 0, u < units};
        if (!w.live) return w;
        if (P.unit_shift >= 0) w.r = (int)(u >> P.unit_shift);
        else w.r = units >> 31 ? (int)(u / P.units_per_row) : (int)((uint32_t)u / (uint32_t)P.units_per_row);
        w.unit = (int)(u - (int64_t)w.r * P.units_per_row);
        w.row = w.r;
        if (P.chunk_mode) w.row = P.items[w.r].x;
        w.begin = __ldg(P.a.indptr + w.row);
        w.end = __ldg(P.a.indptr + w.row + 1);
        return w;
    };
    auto finish_unit = [&](TcUnit w) {
        if (!w.live) return w;
        w.begin = w.begin < 0 ? 0 : w.begin;
        w.end = w.end > P.a.edge_bound ? P.a.edge_bound : w.end;
        if (w.end < w.begin) w.end = w.begin;
        if (P.chunk_mode) {
            w.begin += P.items[w.r].y * P.chunk;
            w.end = w.begin + P.chunk < w.end ? w.begin + P.chunk : w.end;
        } else if (P.split && w.end - w.begin > CA_LONG) {
            if (w.unit == 0) {                               // listed once, by the warp of the row's first unit
                int nc = (w.end - w.begin + P.chunk - 1) / P.chunk, first = 0;
                if (lane == 0) first = list_row(P, w.row, nc);
                first = __shfl_sync(FULL, first, 0);
                nc = list_room(P, first, nc);
                for (int c = lane; c < nc; c += 32) P.items[first + c] = make_int2(w.row, c);
            }
            w.live = false;
            w.end = w.begin;
        }
        return w;
    };
    auto window = [&](const TcUnit& w, int pos) { return pos + lane < w.end ? __ldg(P.a.indices + pos + lane) : -1; };
    auto to_row = [&](int col) {
        if ((uint32_t)col >= (uint32_t)cols) col = -1;
        if (P.a.row_of && col >= 0) col = __ldg(P.a.row_of + col);
        return (uint32_t)col < (uint32_t)P.a.k.rows ? col : -1;
    };
    TcUnit W0 = finish_unit(raw_unit(u)), W1 = finish_unit(raw_unit(u + step)), W2 = raw_unit(u + 2 * step);
    int64_t u0 = u;                                          // the unit that is gathered
    int pos = W0.begin, at = to_row(window(W0, pos));        // rows of 32 edges from pos & ~16 (of the unit) on
    int next = window(W0, pos + 32), later = window(W1, W1.begin);
    bool second = false;                                     // the tile is the later half of the window
    bool more = true;

    // ---- a tile on its way
    struct Tile {
        TcUnit w;
        uint32_t on, scales;
        bool first, last;
    };
    const int edges_per = 32 / (PIECES > 8 ? 8 : PIECES), piece0 = lane & (PIECES > 8 ? 7 : PIECES - 1), edge0 = lane / (PIECES > 8 ? 8 : PIECES);
    auto issue = [&](int stage) {
        Tile x;
        x.w = W0;
        x.first = pos == W0.begin;
        const int mine_at = __shfl_sync(FULL, at, (second ? 16 : 0) + (lane & 15));
        const bool is = pos + (lane & 15) < W0.end && mine_at >= 0;
        const int h0 = W0.unit * SLOTS, kv0 = h0 / group;
        x.on = __ballot_sync(FULL, is) & 0xFFFFu;
        x.scales = 0;
        if (is) {
            const uint8_t* p = SV.scales + (uint64_t)((uint32_t)mine_at >> SV.shift) * sstep + kv0;
            x.scales = __ldg(p);
        }
        const uint32_t base = mine_a + stage * S::STAGE;
#pragma unroll
        for (int i = 0; i < (16 * PIECES + 31) / 32; ++i) {
            const int edge = PIECES > 8 ? (i >> 1) * edges_per + edge0 : i * edges_per + edge0, piece = PIECES > 8 ? piece0 + (i & 1) * 8 : piece0;
            const int from = __shfl_sync(FULL, mine_at, edge & 15), sub = piece * 16;
            if (edge >= 16) continue;                        // fewer pieces than lanes
            const bool has = (x.on >> edge & 1) && sub < D;
            const int bytes = has ? min(16, D - sub) : 0;    // what lies behind head_dim is not read
            const uint64_t row = has ? (uint32_t)from : 0u;
            const uint32_t to = base + tile_byte(edge, piece * 16), in = has ? kv0 * pitch + sub : 0;
            copy_async<16>(to, P.a.k.codes + row * kstep + in, bytes);
            copy_async<16>(to + S::TILE, P.a.v.codes + row * vstep + in, bytes);
        }
        if (x.first && P.wide) {
            for (int i = lane; i < SLOTS * SP * 2; i += 32) {
                const int slot = i / (SP * 2), c = (i - slot * SP * 2) * 8;
                const bool has = W0.live && c < D;
                const bf16* q = (const bf16*)P.a.q.data + (has ? (int64_t)W0.row * P.a.q.row_stride + (int64_t)(h0 + slot) * P.a.q.head_stride + c : 0);
                copy_async<16>(base + 2 * S::TILE + i * 16, q, has ? 16 : 0);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        // the next tile: of this window, of the next one, or of the next unit
        pos += 16;
        x.last = pos >= W0.end;
        if (x.last) {
            u0 += step;
            more = u0 < units;
            W0 = W1;
            pos = W0.begin;
            at = to_row(later);
            next = window(W0, pos + 32);
            W1 = finish_unit(W2);
            later = window(W1, W1.begin);
            W2 = raw_unit(u0 + 2 * step);
            second = false;
        } else if (second) {
            at = to_row(next);
            next = window(W0, pos + 32);
            second = false;
        } else {
            second = true;
        }
        return x;
    };

    Tile queue[TC_STAGES - 1];
    int ahead = 0;                                           // tiles on their way
#pragma unroll
    for (int i = 0; i < TC_STAGES - 1; ++i)
        if (more) {
            queue[i] = issue(i);
            ++ahead;
        } else {
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    int stage = 0;

    // what a unit keeps: the queries' fragments (lane g, t: slot g / 2, columns t L ...), sums, maxima (lane g, t: slot t)
    uint32_t q[SP][2];
    float acc[TILES][2], m = 0.f, l = 0.f, qhalf = 0.f, qscale = 0.f;
    bool apart = false, gone = false;                        // queries whose elements are too far apart, weights of the unit
    int unit = 0;                                            // acc is in units of 2^(unit - 254 - 14)
    const float c2 = P.a.scale * CA_LOG2E;
    const int my_slot = g >> 1;
    while (ahead > 0) {
        const Tile x = queue[0];
#pragma unroll
        for (int i = 0; i + 1 < TC_STAGES - 1; ++i) queue[i] = queue[i + 1];
        --ahead;
        if (more) {
            queue[TC_STAGES - 2] = issue(stage == 0 ? TC_STAGES - 1 : stage - 1);
            ++ahead;
        } else {
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(TC_STAGES - 1) : "memory");
        __syncwarp();
        const unsigned char* tile = mine + stage * S::STAGE;
        stage = stage + 1 == TC_STAGES ? 0 : stage + 1;
        const int h0 = x.w.unit * SLOTS;
        if (x.first) {
            m = -INFINITY;
            l = 0.f;
            unit = 0;
            gone = false;
#pragma unroll
            for (int i = 0; i < TILES; ++i) acc[i][0] = acc[i][1] = 0.f;
            const bool has = (g & 1) == 0 && x.w.live;
            uint32_t w[L / 2], least = 0xFFFFFFFFu;
            if (P.wide) {
                const uint32_t* from = reinterpret_cast<const uint32_t*>(tile + 2 * S::TILE + my_slot * SP * 32 + t * L * 2);
#pragma unroll
                for (int i = 0; i < L / 2; ++i) w[i] = has ? from[i] : 0u;
            } else {
                const uint16_t* from = (const uint16_t*)P.a.q.data + (has ? (int64_t)x.w.row * P.a.q.row_stride + (int64_t)(h0 + my_slot) * P.a.q.head_stride : 0);
#pragma unroll
                for (int i = 0; i < L / 2; ++i) {
                    const int c = t * L + 2 * i;
                    w[i] = has && c < D ? from[c] : 0u;
                    w[i] |= has && c + 1 < D ? (uint32_t)from[c + 1] << 16 : 0u;
                }
            }
            float y[L], top = 0.f;
#pragma unroll
            for (int i = 0; i < L / 2; ++i) {
                least = __viaddmin_u16x2(w[i] & 0x7FFF7FFFu, 0xFFFFFFFFu, least);        // zeros become the largest
                y[2 * i] = bf16_lo(w[i]);
                y[2 * i + 1] = bf16_hi(w[i]);
                top = fmaxf(top, fmaxf(fabsf(y[2 * i]), fabsf(y[2 * i + 1])));
            }
            top = fmaxf(top, __shfl_xor_sync(FULL, top, 1));
            top = fmaxf(top, __shfl_xor_sync(FULL, top, 2));
            // 2^(14 - e) for a largest element of 2^e
            const int up = up_of(__float_as_uint(top) >> 16);
            apart |= too_wide(__float_as_uint(top) >> 16, min(least & 0xFFFFu, least >> 16));
            const float scale = __uint_as_float((uint32_t)up << 23);
#pragma unroll
            for (int i = 0; i < SP; ++i) {
                q[i][0] = pack_f16(y[4 * i] * scale, y[4 * i + 1] * scale);
                q[i][1] = pack_f16(y[4 * i + 2] * scale, y[4 * i + 3] * scale);
            }
            // back by two halves, around the key's scale: a large key and a small query do not pass the range of f32 between them
            const int back = 127 - __shfl_sync(FULL, up, 8 * t);
            qhalf = power_of(back >> 1);
            qscale = power_of(back - (back >> 1)) * c2;
        }
        // ---- scores
        uint32_t k0[SP], k1[SP];
        float c[4] = {0.f, 0.f, 0.f, 0.f};
        read_words<SP>(tile, g, t * L, k0);
        read_words<SP>(tile, g + 8, t * L, k1);
#pragma unroll
        for (int i = 0; i < SP; ++i) mma_f16(c, codes_to_f16(k0[i]), codes_to_f16(k1[i]), codes_to_f16(k0[i] >> 16), codes_to_f16(k1[i] >> 16), q[i][0], q[i][1]);
        // ---- weights of slot t and the edges g and g + 8
        const uint32_t kb0 = __shfl_sync(FULL, x.scales, g), kb1 = __shfl_sync(FULL, x.scales, g + 8);
        const uint32_t vb0 = __shfl_sync(FULL, x.scales, g + 16), vb1 = __shfl_sync(FULL, x.scales, g + 24);
        const float s0 = x.on >> g & 1 ? c[0] * qhalf * scale_of(kb0) * qscale : -INFINITY, s1 = x.on >> (g + 8) & 1 ? c[2] * qhalf * scale_of(kb1) * qscale : -INFINITY;
        float top = fmaxf(s0, s1);
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(FULL, top, o));
        top = fmaxf(top, m);
        const float ref = top == -INFINITY ? 0.f : top;      // nothing seen yet: all weights are zero
        const float fall = m - ref;
        float p0 = exp2_fast(s0 - ref), p1 = exp2_fast(s1 - ref);
        m = top;
        l = fmaf(l, exp2_fast(fall), p0 + p1);
        // exponents of weight times scale, both with their bias: the largest, and the one so far after the maximum's rise
        const int e0 = p0 > 0.f ? (int)(__float_as_uint(p0) >> 23) + (int)vb0 : 0, e1 = p1 > 0.f ? (int)(__float_as_uint(p1) >> 23) + (int)vb1 : 0;
        int most = max(e0, e1);
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) most = max(most, __shfl_xor_sync(FULL, most, o));
        most = max(most, unit + (int)ceilf(fmaxf(fall, -1000.f)));
        const float risen = exp2_fast(fall);
        float corr = unit > 0 ? risen * power_of(unit - most) : 1.f;     // nothing yet: nothing to correct
        float x0 = p0 * 16384.f * power_of((int)vb0 - most + 127), x1 = p1 * 16384.f * power_of((int)vb1 - most + 127);
        unit = most;
        // ---- values: the weights near the largest first, then what is left, from the largest of each slot down
        const unsigned char* vt = tile + S::TILE;
        auto rescale = [&](float by) {
            const float mul = __shfl_sync(FULL, by, my_slot);     // lane `slot` of the first quad
#pragma unroll
            for (int i = 0; i < TILES; ++i) {
                acc[i][0] *= mul;
                acc[i][1] *= mul;
            }
        };
        gone |= corr < TC_GONE && risen > 0.f;
        int up = 0;
        while (true) {
            if (__any_sync(FULL, corr != 1.f)) rescale(corr);
            const bool far0 = x0 < TC_NEAR && up < TC_MOST, far1 = x1 < TC_NEAR && up < TC_MOST;
            multiply_values<SP>(vt, split_weights(far0 ? 0.f : x0, far1 ? 0.f : x1), [&](int i, uint2 a, uint32_t b0, uint32_t b1) { mma_f16_half(acc[i], a.x, a.y, b0, b1); });
            if (!__any_sync(FULL, (far0 && p0 > 0.f) || (far1 && p1 > 0.f))) break;      // p: x may have left the range of 32 bits
            x0 = far0 ? x0 : 0.f;
            x1 = far1 ? x1 : 0.f;
            gone |= (far0 && p0 > 0.f && x0 < TC_GONE) || (far1 && p1 > 0.f && x1 < TC_GONE);
            p0 = x0;
            p1 = x1;
            float high = fmaxf(x0, x1);
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) high = fmaxf(high, __shfl_xor_sync(FULL, high, o));
            if (!__any_sync(FULL, high > 0.f)) break;
            const int more_up = high > 0.f ? min(141 - (int)(__float_as_uint(high) >> 23), TC_MOST - up) : 0;
            up += more_up;
            corr = power_of(more_up);
            x0 *= corr;
            x1 *= corr;
            gone |= up == TC_MOST && ((x0 > 0.f && x0 < TC_NEAR) || (x1 > 0.f && x1 < TC_NEAR));
        }
        if (__any_sync(FULL, up != 0)) rescale(power_of(-up));
        __syncwarp();                                        // the buffer is read before it is filled again
        if (!x.last) continue;
        // ---- the unit's end: rows 2 slot (hi) and 2 slot + 1 (lo) of acc; a lane has columns 4 SP t ...
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) l += __shfl_xor_sync(FULL, l, o);
        const float total = __shfl_sync(FULL, l, my_slot), at_m = __shfl_sync(FULL, m, my_slot), in = scale_of((uint32_t)max(__shfl_sync(FULL, unit, my_slot) - 127, 0));
        float out[L];
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
            out[i] = fmaf(__shfl_xor_sync(FULL, acc[i][0], 4), 1.f / 33554432.f, acc[i][0] * (1.f / 16384.f));
            out[TILES + i] = fmaf(__shfl_xor_sync(FULL, acc[i][1], 4), 1.f / 33554432.f, acc[i][1] * (1.f / 16384.f));
        }
        bool mark = __any_sync(FULL, gone);
        if (mark) {
            // what went is below 2^-84 2^9 an edge: nothing beside columns that are not next to zero
            bool small = false;
#pragma unroll
            for (int i = 0; i < L; ++i) small |= (g & 1) == 0 && t * L + i < D && fabsf(out[i]) < 0x1p-44f;
            mark = __any_sync(FULL, small);
            apart |= mark;
        }
        if (!x.w.live || (g & 1)) continue;
        const int h = h0 + my_slot, col = t * L;
        const bool none = total == 0.f;                      // no edge left by the mask: zero row, log of an empty sum
        if (P.chunk_mode) {
            float* part = P.partial + ((int64_t)x.w.r * P.a.q_heads + h) * (D + 2);
#pragma unroll
            for (int i = 0; i < L; ++i)
                if (col + i < D) part[col + i] = none ? 0.f : out[i] * in;
            if (t == 0) {
                part[D] = mark ? __uint_as_float(TC_AGAIN) : at_m;
                part[D + 1] = total;
            }
        } else {
            const float inv = none ? 0.f : 1.f / total;
            bf16* to = (bf16*)P.a.out.data + (int64_t)x.w.row * P.a.out.row_stride + (int64_t)h * P.a.out.head_stride;
            if (P.wide && L >= 8) {
#pragma unroll
                for (int i = 0; i < L / 8; ++i) {
                    float z[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) z[j] = none ? 0.f : out[8 * i + j] * in * inv;
                    if (col + 8 * i < D) store_vec<bf16, 8>(to + col + 8 * i, z);
                }
            } else {
#pragma unroll
                for (int i = 0; i < L; ++i)
                    if (col + i < D) to[col + i] = from_f32<bf16>(none ? 0.f : out[i] * in * inv);
            }
            if (t == 0) P.a.lse[(int64_t)x.w.row * P.a.q_heads + h] = mark ? __uint_as_float(TC_AGAIN) : none ? -INFINITY : at_m * CA_LN2 + logf(total);
        }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncwarp();                                            // what is overwritten has been written
    if (__any_sync(FULL, apart)) attend_again<SP>(P, units);
}

}  // namespace gs
