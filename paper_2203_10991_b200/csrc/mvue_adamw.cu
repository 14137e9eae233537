// AdamW over many tensors in one launch, states in 32 bits or in 8.
//
// Element-wise: 30 bytes per element with fp32 states, a float copy and fp32 gradients; 10 with 8-bit states, a bf16
// param and a bf16 gradient.  The list of tensors travels in the kernel's parameters (no table in device memory to keep or
// copy); a thread block finds the tensor of its tile by binary search.  A warp owns one block of 256 elements that shares a
// scale, a lane eight consecutive ones: 16 or 32 bytes per load, the block's largest magnitude is one warp-wide integer
// maximum (the bit patterns of non-negative floats are in their order, and a NaN is above all of them), and the lane's
// eight 16-bit random numbers are one generator call.
//
// Measured (B200, HBM copy 6.55 TB/s).  24 matrices of 4 M elements, 32-bit states, bf16 + float copy: 438 us for 3.02 GB,
// 105 % of the copy rate: bound by HBM.  Two matrices of 59 M elements, 8-bit states, bf16: 315 us against 180 us of HBM
// time: bound by instructions, above 60 per element of which 8 are the generator.  What brought it down: the code taken from
// the bit pattern instead of by way of a step and a rounded sum (400 -> 341 us), packed pairs and hardware decoding
// (457 -> 400 us), five blocks an SM (341 -> 315 us, although eight words a thread spill).  Six blocks spill more (368 us); loads of
// the next block ahead of the arithmetic cost more registers than they hide (351 us).  The root is approximate; the correctly
// rounded one for every element would take 374 us, finding the lanes whose code may differ between the two costs what codes below
// 2^-6 in line have saved.  The time depends on the data: lanes with such codes, zeros among them, take longer.  Every second block
// zero 354 us, all zero 408 us, one zero in every lane 441 us.  96 vectors of 2500 elements: 7 to 9 us, the launch.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/mvue_train.h"
#include "mvue_device.cuh"
#include "mvue_internal.h"
#include "mvue_train.cuh"

namespace mvue {
namespace {

constexpr int kTile = 2048, kThreads = 256, kBlock = MVUE_ADAMW_BLOCK;
static_assert(kTile == 8 * kThreads && kBlock == 8 * 32, "a lane owns eight elements, a warp one scale block");

enum : uint32_t { kParamBf16 = 1, kMaster = 2, kGradBf16 = 4, kWide = 8 };

struct Tensor {
    void* param;
    float* master;
    const void* grad;
    void *m, *v;
    float *m_scale, *v_scale;
    int64_t numel;
    int64_t first_block;    // the call's 256-element blocks before this tensor
    uint32_t flags, pad;
};

struct Constants {
    float beta1, one_beta1, beta2, one_beta2, inv_root, eps, decay, step_size, grad_scale, minus_zero;
    const float* dev_grad_scale;
    bool round_up_at_random;   // a bf16 param without master
};

// Kernel parameters may take 32764 bytes: 320 tensors of 84 bytes take 27 KB.  Short lists go in a small block, since the
// parameters of every launch are copied.
template <int kCapacity>
struct Params {
    Constants c;
    RoundKeys keys;
    int count;
    int first_tile[kCapacity];
    Tensor tensor[kCapacity];
};

// Two e4m3 codes (the half-word's low byte first) as binary32; exact by way of binary16.
__device__ __forceinline__ f2 e4m3_values(uint32_t half) {
    uint32_t h;
    asm("{\n\t.reg .b16 c;\n\tcvt.u16.u32 c, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, c;\n\t}" : "=r"(h) : "r"(half));
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    return pair(f.x, f.y);
}

// Code of a magnitude y <= 448 (a few units in its last place above are no matter), any y: steps of 2^-3 of its power of
// two (2^-9 below 2^-6), rounded up where the fraction plus the random number r 2^-16 reaches one.  The product by a power
// of two is exact; adding 2^23 rounded down leaves the whole steps in the low bits.
__device__ __forceinline__ uint32_t e4m3_code(float y, uint32_t r) {
    const uint32_t e = max(__float_as_uint(y) & 0x7F800000u, 121u << 23);
    const float steps = __fmaf_rn(y, __uint_as_float((257u << 23) - e), (float)r * 1.52587890625e-05f);
    return (e >> 20) - (121u << 3) + (__float_as_uint(__fadd_rd(steps, 8388608.0f)) - 0x4B000000u);
}
// The same for four numbers y with magnitudes of at least 2^-6, signs apart, without a step for the power of two: adding
// r to the 16 bits below the three mantissa bits of a binary32 carries into them exactly that often, and the code is the
// low five exponent bits and the three mantissa bits less a constant.  r8: r << 8, which is r's place four bits further up,
// where the code fills the highest byte; the sign is shifted out.
__device__ __forceinline__ uint32_t carried(float y, uint32_t r8) { return __float_as_uint(y) * 16u + r8; }
__device__ __forceinline__ uint32_t e4m3_codes_normal(const uint32_t* t) {
    const uint32_t bytes = __byte_perm(__byte_perm(t[0], t[1], 0x0073), __byte_perm(t[2], t[3], 0x0073), 0x5410);
    return (bytes ^ 0x40404040u) & 0x7F7F7F7Fu;              // less 120 << 3: the top two bits are 11 or 00, to become 00 or 01
}

__device__ __forceinline__ uint32_t min_halves(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("min.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// Square root with a relative error of at most 2^-23; without kSubnormal, arguments below 2^-126 have the root 0 (v' of |g'| below
// 3e-18 on a fresh state).
template <bool kSubnormal>
__device__ __forceinline__ float fast_root(float x) {
    float r;
    if (kSubnormal) asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    else asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// the larger magnitude, NaN if there is one
__device__ __forceinline__ float larger(float a, float b) {
    float r;
    asm("max.NaN.xorsign.abs.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// the warp's largest magnitude (NaN above all: the bit patterns of non-negative floats are in their order)
__device__ __forceinline__ float warp_largest(float x) {
    return __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(x) & 0x7FFFFFFFu));
}

// new scale and the factor to codes of a block whose largest magnitude is `top`
__device__ __forceinline__ float block_scale(float top, float* factor) {
    const bool finite = __float_as_uint(top) < 0x7F800000u, large = top >= 7.703719777548943e-34f;     // 2^-110
    *factor = finite && large ? __fmul_rn(448.0f, __frcp_rn(top)) : 0.0f;
    return finite ? (large ? __fmul_rn(top, 1.0f / 448.0f) : 0.0f) : __uint_as_float(0x7FFFFFFFu);
}

// A NaN whose lower half is zero: random bits added to it do not carry into the sign.
__device__ __forceinline__ float short_nan(float x) { return x != x ? __uint_as_float(0x7FC00000u) : x; }

// The new moments of eight elements (v: the second moment, root: its square root, fast_root's) and the new param.
template <bool kSubnormal>
struct Step {
    f2 m[4], v[4], root[4], p[4];
    __device__ __forceinline__ void take(const Constants& c, const f2 (&g)[4], float gs) {
        const f2 scale = pair(gs), b1 = pair(c.beta1), c1 = pair(c.one_beta1), b2 = pair(c.beta2), c2 = pair(c.one_beta2);
        const f2 inv_root = pair(c.inv_root), eps = pair(c.eps), decay = pair(c.decay), size = pair(-c.step_size);
        // a product that the compiler cannot fuse with the sum behind it: it does not know that this is -0
        const f2 nothing = pair(c.minus_zero);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const f2 x = mul2(g[j], scale);
            m[j] = add2(fma2(b1, m[j], nothing), fma2(c1, x, nothing));
            v[j] = add2(fma2(b2, v[j], nothing), fma2(mul2(c2, x), x, nothing));
            float r0, r1, d0, d1;
            unpair(v[j], r0, r1);
            root[j] = pair(fast_root<kSubnormal>(r0), fast_root<kSubnormal>(r1));
            unpair(add2(mul2(root[j], inv_root), eps), d0, d1);
            p[j] = fma2(p[j], decay, mul2(size, mul2(m[j], pair(fast_reciprocal(d0), fast_reciprocal(d1)))));
        }
    }
};

__device__ __forceinline__ void as_pairs(const float (&x)[8], f2 (&p)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) p[j] = pair(x[2 * j], x[2 * j + 1]);
}
__device__ __forceinline__ void as_floats(const f2 (&p)[4], float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) unpair(p[j], x[2 * j], x[2 * j + 1]);
}
template <typename T> __device__ __forceinline__ void load_pairs(const T* from, bool wide, int count, f2 (&p)[4]) {
    float x[8];
    load8(from, wide, count, x);
    as_pairs(x, p);
}
__device__ __forceinline__ uint2 load_codes(const uint8_t* from, bool wide, int count) {
    if (wide) return *reinterpret_cast<const uint2*>(from);
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < count) w[i >> 2] |= (uint32_t)from[i] << (8 * (i & 3));
    return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void store_codes(uint8_t* to, bool wide, int count, const uint32_t (&w)[2]) {
    if (wide) {
        *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) to[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
    }
}

// kRuns: blocks of 256 elements that a warp takes one after another; the search for the tensor is shared by them.
template <int kBits, int kCapacity, int kRuns, bool kSubnormal>
__global__ void __launch_bounds__(kThreads, 5) adamw_kernel(const __grid_constant__ Params<kCapacity> a) {
    grid_dependency_wait();
    const int tile = blockIdx.x;
    int lo = 0, hi = a.count - 1;
    while (lo < hi) {                                       // the last tensor that starts at or before this tile
        const int mid = (lo + hi + 1) >> 1;
        if (a.first_tile[mid] <= tile) lo = mid; else hi = mid - 1;
    }
    const Tensor& t = a.tensor[lo];
    const Constants& c = a.c;
    const int lane = threadIdx.x & 31;
    const int64_t block0 = ((int64_t)(tile - a.first_tile[lo]) * (kThreads / 32) + (threadIdx.x >> 5)) * kRuns;
    const uint32_t flags = t.flags;
    const float gs = c.dev_grad_scale ? __fmul_rn(c.grad_scale, *c.dev_grad_scale) : c.grad_scale;
    const bool round_param = c.round_up_at_random && (flags & (kParamBf16 | kMaster)) == kParamBf16;
#pragma unroll 1
    for (int run = 0; run < kRuns; ++run) {
        const int64_t block = block0 + run, i0 = block * kBlock + lane * 8;
        if (block * kBlock >= t.numel) return;              // a whole warp
        const int count = (int)min((int64_t)8, max((int64_t)0, t.numel - i0));
        const bool wide = (flags & kWide) && count == 8;

        // all loads first
        f2 g[4];
        Step<kSubnormal> s;
        uint2 mc = make_uint2(0u, 0u), vc = mc;
        float ms = 0.0f, vs = 0.0f;
        if (flags & kGradBf16) load_pairs(static_cast<const __nv_bfloat16*>(t.grad) + i0, wide, count, g);
        else load_pairs(static_cast<const float*>(t.grad) + i0, wide, count, g);
        if (kBits == 32) {
            load_pairs(static_cast<const float*>(t.m) + i0, wide, count, s.m);
            load_pairs(static_cast<const float*>(t.v) + i0, wide, count, s.v);
        } else {
            mc = load_codes(static_cast<const uint8_t*>(t.m) + i0, wide, count);
            vc = load_codes(static_cast<const uint8_t*>(t.v) + i0, wide, count);
            ms = t.m_scale[block];
            vs = t.v_scale[block];
        }
        if (flags & kMaster) load_pairs(t.master + i0, wide, count, s.p);
        else if (flags & kParamBf16) load_pairs(static_cast<const __nv_bfloat16*>(t.param) + i0, wide, count, s.p);
        else load_pairs(static_cast<const float*>(t.param) + i0, wide, count, s.p);

        uint4 random = make_uint4(0u, 0u, 0u, 0u);
        if (kBits == 8 || round_param)
            random = philox4x32_10((uint64_t)(t.first_block + block) * (kBlock / 8) + lane, a.keys, 2u);
        const uint32_t rw[4] = {random.x, random.y, random.z, random.w};

        if (kBits == 8) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s.m[j] = mul2(e4m3_values((j < 2 ? mc.x : mc.y) >> (16 * (j & 1)) & 0xFFFFu), pair(ms));
                const f2 r = mul2(e4m3_values((j < 2 ? vc.x : vc.y) >> (16 * (j & 1)) & 0xFFFFu), pair(vs));
                s.v[j] = mul2(r, r);
            }
        }
        s.take(c, g, gs);

        if (kBits == 32) {
            float x[8];
            as_floats(s.m, x);
            store8(static_cast<float*>(t.m) + i0, wide, count, x);
            as_floats(s.v, x);
            store8(static_cast<float*>(t.v) + i0, wide, count, x);
        } else {
            float m[8], v[8];
            as_floats(s.m, m);
            as_floats(s.v, v);
            float m_top = m[0], v_top = v[0];
#pragma unroll
            for (int i = 1; i < 8; ++i) {
                m_top = larger(m_top, m[i]);
                v_top = larger(v_top, v[i]);
            }
            // the root grows with v: the largest root is that of the largest v
            float mf, vf;
            ms = block_scale(warp_largest(m_top), &mf);
            vs = block_scale(__fsqrt_rn(warp_largest(v_top)), &vf);
            // The code of sqrt(v) is that of the correctly rounded root also where the approximate one is on the other side of a
            // threshold.  z is raised by 10 2^-24 of itself, against at most 6 2^-24 for the two roots' distance and the roundings: it
            // is above the z of the correctly rounded root by at most 16 units of its last place, and gives the same code unless
            // its sum with the random number is less than that above a carry.  Lanes where one is within 32 units
            // (one in four thousand) take the second way.
            const float raised = vf * 1.00000059604644775390625f;
            float y[8], z[8];
            uint32_t r8[8];
            float least_y = 1.0f, least_z = 1.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                unpair(mul2(s.m[j], pair(mf)), y[2 * j], y[2 * j + 1]);
                unpair(mul2(s.root[j], pair(raised)), z[2 * j], z[2 * j + 1]);
                least_y = fminf(least_y, fminf(fabsf(y[2 * j]), fabsf(y[2 * j + 1])));
                least_z = fminf(least_z, fminf(z[2 * j], z[2 * j + 1]));
                r8[2 * j] = __byte_perm(rw[j], 0u, 0x4014);              // the half-words with their bytes exchanged, << 8
                r8[2 * j + 1] = __byte_perm(rw[j], 0u, 0x4234);
            }
            // bits 8 .. 23 of the sums, two to a word: below 2 within 32 units above a carry
            uint32_t ty[8], tz[8], nearest = 0xFFFFFFFFu;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                ty[i] = carried(y[i], r8[i]);
                tz[i] = carried(z[i], r8[i]);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) nearest = min_halves(nearest, __byte_perm(tz[2 * j], tz[2 * j + 1], 0x6521));
            uint32_t mw[2], vw[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t signs = __byte_perm(__byte_perm(__float_as_uint(y[4 * h]), __float_as_uint(y[4 * h + 1]), 0x0073),
                                                   __byte_perm(__float_as_uint(y[4 * h + 2]), __float_as_uint(y[4 * h + 3]), 0x0073), 0x5410);
                mw[h] = e4m3_codes_normal(ty + 4 * h) | (signs & 0x80808080u);
                vw[h] = e4m3_codes_normal(tz + 4 * h);
            }
            if (least_y < 0.015625f) {
                mw[0] = mw[1] = 0u;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    mw[i >> 2] |= (e4m3_code(fminf(fabsf(y[i]), 448.0f), r8[i] >> 8) | (y[i] < 0.0f ? 0x80u : 0u)) << (8 * (i & 3));
            }
            // below 2^-6 without the raise, or near a carry
            if (least_z < 0.01563f || (nearest & 0xFFFFu) < 2u || nearest < 0x20000u) {
                vw[0] = vw[1] = 0u;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float exact = vf > 0.0f ? __fmul_rn(__fsqrt_rn(v[i]), vf) : 0.0f;
                    vw[i >> 2] |= max(e4m3_code(fminf(exact, 448.0f), r8[i] >> 8), v[i] > 0.0f ? 1u : 0u) << (8 * (i & 3));
                }
            }
            store_codes(static_cast<uint8_t*>(t.m) + i0, wide, count, mw);
            store_codes(static_cast<uint8_t*>(t.v) + i0, wide, count, vw);
            if (lane == 0) {
                t.m_scale[block] = ms;
                t.v_scale[block] = vs;
            }
        }
        float x[8];
        as_floats(s.p, x);
        if (flags & kMaster) store8(t.master + i0, wide, count, x);
        if (flags & kParamBf16) {
            uint32_t w[4];
            float sum;                                       // NaN where one of them is (or two infinities cancel)
            {
                float a0, a1;
                unpair(add2(add2(s.p[0], s.p[1]), add2(s.p[2], s.p[3])), a0, a1);
                sum = a0 + a1;
            }
            if (round_param && sum == sum) {
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = pack_out<true>(x[2 * i], x[2 * i + 1], rw[i]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    w[i] = round_param ? pack_out<true>(short_nan(x[2 * i]), short_nan(x[2 * i + 1]), rw[i]) : pack_bf16x2(x[2 * i], x[2 * i + 1]);
            }
            store8_words(static_cast<__nv_bfloat16*>(t.param) + i0, wide, count, w);
        } else {
            store8(static_cast<float*>(t.param) + i0, wide, count, x);
        }
    }
}

template <int kBits, int kCapacity, int kRuns, bool kSubnormal>
cudaError_t launch(const mvue_adamw_tensor* ts, int64_t count, const Constants& c, uint64_t seed,
                   int64_t* first_block, int64_t* used, cudaStream_t stream) {
    Params<kCapacity> a;
    a.c = c;
    a.keys = make_round_keys(seed);
    int n = 0;
    int64_t tiles = 0, i = 0;
    for (; i < count && n < kCapacity; ++i) {
        const mvue_adamw_tensor& s = ts[i];
        const int64_t blocks = (s.numel + kBlock - 1) / kBlock;
        if (s.numel == 0) continue;
        const int64_t mine = (s.numel + kTile * kRuns - 1) / (kTile * kRuns);
        if (tiles + mine > 0x7FFFFFFF) break;
        Tensor& t = a.tensor[n];
        t = {s.param, static_cast<float*>(s.master), s.grad, s.exp_avg, s.exp_avg_sq, static_cast<float*>(s.exp_avg_scale),
             static_cast<float*>(s.exp_avg_sq_scale), s.numel, *first_block, 0u, 0u};
        t.flags = (s.param_dtype == MVUE_BF16 ? kParamBf16 : 0u) | (s.master ? kMaster : 0u) |
                  (s.grad_dtype == MVUE_BF16 ? kGradBf16 : 0u);
        const uintptr_t all = reinterpret_cast<uintptr_t>(s.param) | reinterpret_cast<uintptr_t>(s.master) |
                              reinterpret_cast<uintptr_t>(s.grad) | reinterpret_cast<uintptr_t>(s.exp_avg) |
                              reinterpret_cast<uintptr_t>(s.exp_avg_sq);
        if ((all & 31u) == 0) t.flags |= kWide;
        a.first_tile[n++] = (int)tiles;
        tiles += mine;
        *first_block += blocks;
    }
    *used = i;
    if (n == 0) return cudaSuccess;
    a.count = n;
    return launch_dependent(&adamw_kernel<kBits, kCapacity, kRuns, kSubnormal>, dim3((unsigned)tiles), dim3(kThreads), 0, stream, a);
}

}  // namespace
}  // namespace mvue

using namespace mvue;

extern "C" int mvue_adamw_step(const mvue_adamw_tensor* tensors, int64_t count, const mvue_adamw_config* cfg, void* stream) {
    if (!cfg || (count > 0 && !tensors)) return MVUE_ERR_NULL;
    if (count < 0 || cfg->step < 1) return MVUE_ERR_SHAPE;
    if (cfg->state_bits != 8 && cfg->state_bits != 32) return MVUE_ERR_DTYPE;
    if (cfg->options & ~(uint32_t)MVUE_OPT_STOCHASTIC_ROUNDING) return MVUE_ERR_OPTION;
    if (!(cfg->beta1 >= 0.0 && cfg->beta1 < 1.0 && cfg->beta2 >= 0.0 && cfg->beta2 < 1.0)) return MVUE_ERR_OPTION;
    for (int64_t i = 0; i < count; ++i) {
        const mvue_adamw_tensor& t = tensors[i];
        if (t.numel < 0 || t.numel > 0x7FFFFFFFll * kTile) return MVUE_ERR_SHAPE;
        if ((t.param_dtype != MVUE_F32 && t.param_dtype != MVUE_BF16) || (t.grad_dtype != MVUE_F32 && t.grad_dtype != MVUE_BF16) ||
            (t.master && t.param_dtype != MVUE_BF16))
            return MVUE_ERR_DTYPE;
        if (t.numel == 0) continue;
        if (!t.param || !t.grad || !t.exp_avg || !t.exp_avg_sq) return MVUE_ERR_NULL;
        if (cfg->state_bits == 8 && (!t.exp_avg_scale || !t.exp_avg_sq_scale)) return MVUE_ERR_NULL;
        const auto off = [](const void* p, uintptr_t size) { return (reinterpret_cast<uintptr_t>(p) & (size - 1)) != 0; };
        if (off(t.param, t.param_dtype == MVUE_BF16 ? 2 : 4) || off(t.grad, t.grad_dtype == MVUE_BF16 ? 2 : 4) || off(t.master, 4) ||
            (cfg->state_bits == 32 ? off(t.exp_avg, 4) || off(t.exp_avg_sq, 4) : off(t.exp_avg_scale, 4) || off(t.exp_avg_sq_scale, 4)))
            return MVUE_ERR_ALIGN;
    }
    DeviceInfo dev;
    if (int s = current_device_info(&dev)) return s;
    const double t = (double)cfg->step;
    Constants c;
    c.beta1 = (float)cfg->beta1;
    c.one_beta1 = (float)(1.0 - cfg->beta1);
    c.beta2 = (float)cfg->beta2;
    c.one_beta2 = (float)(1.0 - cfg->beta2);
    c.inv_root = (float)(1.0 / std::sqrt(1.0 - std::pow(cfg->beta2, t)));
    c.eps = (float)cfg->eps;
    c.decay = (float)(1.0 - cfg->lr * cfg->weight_decay);
    c.step_size = (float)(cfg->lr / (1.0 - std::pow(cfg->beta1, t)));
    c.grad_scale = (float)cfg->grad_scale;
    c.minus_zero = -0.0f;
    c.dev_grad_scale = cfg->dev_grad_scale;
    c.round_up_at_random = (cfg->options & MVUE_OPT_STOCHASTIC_ROUNDING) != 0;
    // 8-bit states: four blocks a warp where that still gives every SM sixteen thread blocks (the step is bound by
    // instructions there; 32-bit states are bound by memory and slower with it: 448 us against 433 us on 24 matrices of 4 M)
    int64_t elements = 0, first_block = 0;
    for (int64_t i = 0; i < count; ++i) elements += tensors[i].numel;
    const bool runs = elements / (4 * kTile) >= 16 * dev.sm_count;
    // 8-bit states: a v' below 2^-126 counts in the step's divisor only where its root, 2^-63 at most, is not lost beside eps: else
    // the root may flush it (2 x 59 M elements: 318 us with such roots, 312 us without; the codes' own root is exact either way).
    // 32-bit states are bound by memory and always take it (439 us either way on 24 matrices of 4 M).
    const bool subnormal = std::ldexp(1.0 / std::sqrt(1.0 - std::pow(cfg->beta2, t)), -63) > std::ldexp(cfg->eps, -26);
    while (count > 0) {
        int64_t used = 0;
        cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
        const auto go = [&](auto kernel) { return kernel(tensors, count, c, cfg->seed, &first_block, &used, st); };
        cudaError_t e;
        if (cfg->state_bits == 32) e = go(count <= 32 ? &launch<32, 32, 1, true> : &launch<32, 320, 1, true>);
        else if (runs && subnormal) e = go(count <= 32 ? &launch<8, 32, 4, true> : &launch<8, 320, 4, true>);
        else if (runs) e = go(count <= 32 ? &launch<8, 32, 4, false> : &launch<8, 320, 4, false>);
        else if (subnormal) e = go(count <= 32 ? &launch<8, 32, 1, true> : &launch<8, 320, 1, true>);
        else e = go(count <= 32 ? &launch<8, 32, 1, false> : &launch<8, 320, 1, false>);
        if (e != cudaSuccess) { set_cuda_error(e, "mvue_adamw_step launch"); return MVUE_ERR_CUDA; }
        tensors += used;
        count -= used;
    }
    return MVUE_OK;
}
