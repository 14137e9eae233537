// Loads and stores shared by the kernels around the pruned products: eight consecutive elements of a lane as binary32.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "mvue_device.cuh"

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

// Two binary32 values in one register pair: sm_100a adds, multiplies and fuses both in one instruction, each rounded as
// the scalar instruction rounds it.
struct f2 {
    unsigned long long v;
};
__device__ __forceinline__ f2 pair(float lo, float hi) {
    f2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ f2 pair(float both) { return pair(both, both); }
__device__ __forceinline__ void unpair(f2 a, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(a.v)); }
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
    f2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
    f2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
    f2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
// 2^x and 1/x to about one unit in the last place, subnormal results as zero.
__device__ __forceinline__ float fast_exp2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float fast_reciprocal(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

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

// Eight elements of a row per thread: consecutive ones where the rows allow wide accesses, else one of every
// `stride` (the team's threads), so that a warp's accesses stay together.
template <bool kWide>
struct Cols {
    int64_t first;
    int step, count;
    __device__ __forceinline__ Cols(int64_t slab0, int64_t cols, int lane, int team) {
        first = slab0 + (kWide ? (int64_t)lane * 8 : lane);
        step = kWide ? 1 : team;
        const int64_t left = cols - first;
        count = left <= 0 ? 0 : (int)min((int64_t)8, kWide ? left : (left + team - 1) / team);
    }
    template <typename T> __device__ __forceinline__ void load(const T* row, float (&x)[8]) const {
        if (kWide) {
            load8(row + first, true, 8, x);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = j < count ? (float)row[first + (int64_t)j * step] : 0.0f;
        }
    }
    __device__ __forceinline__ void store(float* row, const float (&x)[8]) const {
        if (kWide) {
            store8(row + first, true, 8, x);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < count) row[first + (int64_t)j * step] = x[j];
        }
    }
    __device__ __forceinline__ void store(__nv_bfloat16* row, const float (&x)[8]) const {
        if (kWide) {
            const uint32_t w[4] = {pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
            store8_words(row + first, true, 8, w);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < count) row[first + (int64_t)j * step] = __float2bfloat16_rn(x[j]);
        }
    }
};

}  // namespace mvue
