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

// Eight elements of a row per thread in groups of kVec neighbours: 8 where the rows allow wide accesses (then they are
// consecutive), 2 where they allow those, else 1; the groups lie the team's threads apart, so that a warp's accesses stay
// together.
template <typename T> struct Two;
template <> struct Two<float> { using Type = float2; };
template <> struct Two<__nv_bfloat16> { using Type = __nv_bfloat162; };

template <int kVec>
struct Cols {
    int64_t first;
    int step, count;                 // elements from one group to the next; elements that exist
    __device__ __forceinline__ Cols(int64_t slab0, int64_t cols, int lane, int team) {
        first = slab0 + (int64_t)lane * kVec;
        step = team * kVec;
        const int64_t left = cols - first;
        count = left <= 0 ? 0 : (int)min((int64_t)8, kVec == 8 ? left : (left + step - 1) / step * kVec);
    }
    __device__ __forceinline__ int64_t at(int j) const { return first + (int64_t)(j / kVec) * step + j % kVec; }
    template <typename T> __device__ __forceinline__ void load(const T* row, float (&x)[8]) const {
        if constexpr (kVec == 8) {
            load8(row + first, true, 8, x);
        } else if constexpr (kVec == 2) {
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                float2 v = make_float2(0.0f, 0.0f);
                if (j < count) {
                    const typename Two<T>::Type q = *reinterpret_cast<const typename Two<T>::Type*>(row + at(j));
                    v = make_float2((float)q.x, (float)q.y);
                }
                x[j] = v.x;
                x[j + 1] = v.y;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = j < count ? (float)row[at(j)] : 0.0f;
        }
    }
    __device__ __forceinline__ void store(float* row, const float (&x)[8]) const {
        if constexpr (kVec == 8) {
            store8(row + first, true, 8, x);
        } else if constexpr (kVec == 2) {
#pragma unroll
            for (int j = 0; j < 8; j += 2)
                if (j < count) *reinterpret_cast<float2*>(row + at(j)) = make_float2(x[j], x[j + 1]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < count) row[at(j)] = x[j];
        }
    }
    __device__ __forceinline__ void store(__nv_bfloat16* row, const float (&x)[8]) const {
        if constexpr (kVec == 8) {
            const uint32_t w[4] = {pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
            store8_words(row + first, true, 8, w);
        } else if constexpr (kVec == 2) {
#pragma unroll
            for (int j = 0; j < 8; j += 2)
                if (j < count) *reinterpret_cast<uint32_t*>(row + at(j)) = pack_bf16x2(x[j], x[j + 1]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < count) row[at(j)] = __float2bfloat16_rn(x[j]);
        }
    }
};

// ---- host: how many neighbouring elements of a matrix's rows one access may take: eight (16 bytes of bf16, 32 of fp32), two, or
// one, by the alignment of base, leading dimension and columns.  Pairs against single elements, group norm on 16 x 3000 x 90
// bf16: backward 33 us against 38 us, forward 27 us either way. ----
inline bool off(const void* p, int64_t size) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(size - 1)) != 0; }
inline int64_t size_of(int dtype) { return dtype == 1 ? 2 : 4; }                 // MVUE_BF16, MVUE_F32
inline int row_vector(const void* p, int64_t ld, int64_t cols, int dtype) {
    for (int v = 8; v > 1; v /= 4)
        if (!off(p, v * size_of(dtype)) && cols % v == 0 && ld % v == 0) return v;
    return 1;
}

}  // namespace mvue
