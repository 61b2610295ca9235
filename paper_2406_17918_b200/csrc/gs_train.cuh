// Device helpers of the training operators: typed vector access and the bound on spin waits.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace gs {

using bf16 = __nv_bfloat16;

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(bf16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ bf16 from_f32<bf16>(float x) { return __float2bfloat16_rn(x); }

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// VE consecutive elements of T held in one register word group of 16, 8, 4 or 2 bytes.
template <int BYTES> struct WordOf;
template <> struct WordOf<16> { using type = uint4; };
template <> struct WordOf<8> { using type = uint2; };
template <> struct WordOf<4> { using type = uint32_t; };
template <> struct WordOf<2> { using type = uint16_t; };
template <typename T, int VE> struct Raw {
    using word = typename WordOf<(int)sizeof(T) * VE>::type;
    word w;
};

template <typename T, int VE> __device__ __forceinline__ Raw<T, VE> zero_raw() {
    Raw<T, VE> r;
    if constexpr (sizeof(T) * VE == 16) r.w = make_uint4(0, 0, 0, 0);
    else if constexpr (sizeof(T) * VE == 8) r.w = make_uint2(0, 0);
    else r.w = 0;
    return r;
}
template <typename T, int VE> __device__ __forceinline__ Raw<T, VE> load_raw(const T* p) {
    Raw<T, VE> r;
    r.w = __ldg(reinterpret_cast<const typename Raw<T, VE>::word*>(p));
    return r;
}
// The same for data that is read once: evicted first.
template <typename T, int VE> __device__ __forceinline__ Raw<T, VE> load_raw_stream(const T* p) {
    Raw<T, VE> r;
    r.w = __ldcs(reinterpret_cast<const typename Raw<T, VE>::word*>(p));
    return r;
}

template <typename T, int VE> __device__ __forceinline__ void unpack(const Raw<T, VE>& r, float (&x)[VE]) {
    constexpr int BYTES = (int)sizeof(T) * VE;
    uint32_t w[BYTES >= 4 ? BYTES / 4 : 1];
    if constexpr (BYTES == 16) { w[0] = r.w.x; w[1] = r.w.y; w[2] = r.w.z; w[3] = r.w.w; }
    else if constexpr (BYTES == 8) { w[0] = r.w.x; w[1] = r.w.y; }
    else w[0] = (uint32_t)r.w;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < VE; ++i) x[i] = __uint_as_float(w[i]);
    } else if constexpr (VE == 1) {
        x[0] = bf16_lo(w[0]);
    } else {
#pragma unroll
        for (int i = 0; i < VE; i += 2) { x[i] = bf16_lo(w[i / 2]); x[i + 1] = bf16_hi(w[i / 2]); }
    }
}

// Stores VE floats as VE elements of T in pieces of at most 16 bytes; the address is aligned to the piece.
template <typename T, int VE> __device__ __forceinline__ void store_vec(T* p, const float (&x)[VE]) {
    constexpr int BYTES = (int)sizeof(T) * VE;
    uint32_t w[BYTES >= 4 ? BYTES / 4 : 1];
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < VE; ++i) w[i] = __float_as_uint(x[i]);
    } else if constexpr (VE > 1) {
#pragma unroll
        for (int i = 0; i < VE; i += 2) w[i / 2] = pack_bf16(x[i], x[i + 1]);
    }
    if constexpr (BYTES == 2) {
        *p = from_f32<T>(x[0]);
    } else if constexpr (BYTES == 4) {
        *reinterpret_cast<uint32_t*>(p) = w[0];
    } else if constexpr (BYTES == 8) {
        *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
        for (int i = 0; i < BYTES / 16; ++i) reinterpret_cast<uint4*>(p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    }
}

// Two 32-bit values in one 64-bit register pair.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair(float lo, float hi) {
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void split(f32x2 x, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(x)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

template <int BYTES> __device__ __forceinline__ void copy_async(uint32_t dst, const void* src, int n) {   // n bytes, the rest zero
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
    else if constexpr (BYTES == 8) asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}

}  // namespace gs
