// Loads and stores shared by the kernels around the pruned products: eight consecutive elements of a lane as binary32.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace mvue {

__device__ __forceinline__ void ld256(const void* p, uint32_t (&w)[8]) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p) : "memory");
}
__device__ __forceinline__ void st256(void* p, const uint32_t (&w)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]),
                 "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Eight elements from p (wide: all eight exist and p is aligned to their size; otherwise `count` of them, the rest zero).
__device__ __forceinline__ void load8(const float* p, bool wide, int count, float (&x)[8]) {
    if (wide) {
        uint32_t w[8];
        ld256(p, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = i < count ? p[i] : 0.0f;
    }
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, bool wide, int count, float (&x)[8]) {
    if (wide) {
        const uint4 w = *reinterpret_cast<const uint4*>(p);
        x[0] = bf16_lo(w.x); x[1] = bf16_hi(w.x); x[2] = bf16_lo(w.y); x[3] = bf16_hi(w.y);
        x[4] = bf16_lo(w.z); x[5] = bf16_hi(w.z); x[6] = bf16_lo(w.w); x[7] = bf16_hi(w.w);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = i < count ? __bfloat162float(p[i]) : 0.0f;
    }
}
__device__ __forceinline__ void store8(float* p, bool wide, int count, const float (&x)[8]) {
    if (wide) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(x[i]);
        st256(p, w);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) p[i] = x[i];
    }
}
// Eight bf16 already packed in words, lower element first.
__device__ __forceinline__ void store8_words(__nv_bfloat16* p, bool wide, int count, const uint32_t (&w)[4]) {
    if (wide) {
        *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
        unsigned short* q = reinterpret_cast<unsigned short*>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) q[i] = (unsigned short)(w[i >> 1] >> (16 * (i & 1)));
    }
}

}  // namespace mvue
