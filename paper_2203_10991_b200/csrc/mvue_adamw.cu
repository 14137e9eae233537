// AdamW over many tensors in one launch, states in 32 bits or in 8.
//
// Element-wise, so bound by HBM: 30 bytes per element with fp32 states, a float copy and fp32 gradients; 10 with
// 8-bit states, a bf16 param and a bf16 gradient.  The list of tensors travels in the kernel's parameters (no table
// in device memory to keep or copy); a thread block finds the tensor of its tile of 2048 elements by binary search.
// A warp owns one block of 256 elements that shares a scale, a lane eight consecutive ones: 16 or 32 bytes per load,
// the block's largest magnitude is one warp-wide integer maximum (the bit patterns of non-negative floats are in
// their order, and a NaN is above all of them), and the lane's eight 16-bit random numbers are one generator call.
#include <cuda_bf16.h>
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
    float beta1, one_beta1, beta2, one_beta2, inv_root, eps, decay, step_size, grad_scale;
    const float* dev_grad_scale;
    bool round_up_at_random;   // a bf16 param without master
};

// Kernel parameters may take 32764 bytes: 300 tensors of 84 bytes.  Short lists go in a small block, since the
// parameters of every launch are copied.
template <int kCapacity>
struct Params {
    Constants c;
    RoundKeys keys;
    int count;
    int first_tile[kCapacity];
    Tensor tensor[kCapacity];
};

// e4m3 magnitude of a code byte: shifted into the place of a binary32's exponent and mantissa it is 2^-120 times its
// value, the codes below 8 (no leading one) included.
__device__ __forceinline__ float e4m3_value(uint32_t byte) {
    const float mag = __fmul_rn(__uint_as_float((byte & 0x7Fu) << 20), 1.329227995784916e36f);   // 2^120
    return __uint_as_float(__float_as_uint(mag) | (byte & 0x80u) << 24);
}

// Code of a magnitude y <= 448: steps of 2^-3 of its power of two (2^-9 below 2^-6), rounded up where the fraction plus
// the random number `unit` in [0, 1) passes one.  The product by a power of two is exact; adding 2^23 rounded down leaves
// the whole steps in the low bits.
__device__ __forceinline__ uint32_t e4m3_code(float y, float unit) {
    const uint32_t e = max(__float_as_uint(y) & 0x7F800000u, 121u << 23);
    const float steps = __fmaf_rn(y, __uint_as_float((257u << 23) - e), unit);
    return (e >> 20) - (121u << 3) + (__float_as_uint(__fadd_rd(steps, 8388608.0f)) - 0x4B000000u);
}

__device__ __forceinline__ float fast_root(float x) {
    float r;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

struct Lane {
    float g[8], m[8], v[8], p[8];     // v: the second moment, after the update of the 8-bit states its root
};

// new scale and the factor to codes of a block whose largest magnitude has the bits `top`
__device__ __forceinline__ float block_scale(uint32_t top, float* factor) {
    const float t = __uint_as_float(top);
    const bool finite = top < 0x7F800000u, large = t >= 7.703719777548943e-34f;     // 2^-110
    *factor = finite && large ? __fmul_rn(448.0f, __frcp_rn(t)) : 0.0f;
    return finite ? (large ? __fmul_rn(t, 1.0f / 448.0f) : 0.0f) : __uint_as_float(0x7FFFFFFFu);
}

// A NaN whose lower half is zero: random bits added to it do not carry into the sign.
__device__ __forceinline__ float short_nan(float x) { return x != x ? __uint_as_float(0x7FC00000u) : x; }

template <int kBits, int kCapacity>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const __grid_constant__ Params<kCapacity> a) {
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
    const int64_t block = (int64_t)(tile - a.first_tile[lo]) * (kTile / kBlock) + (threadIdx.x >> 5);
    const int64_t i0 = block * kBlock + lane * 8;
    if (block * kBlock >= t.numel) return;                  // a whole warp
    const int count = (int)min((int64_t)8, max((int64_t)0, t.numel - i0));
    const bool wide = (t.flags & kWide) && count == 8;

    Lane x;
    uint2 mc = make_uint2(0u, 0u), vc = mc;
    float ms = 0.0f, vs = 0.0f;
    // all loads first
    if (t.flags & kGradBf16) load8(static_cast<const __nv_bfloat16*>(t.grad) + i0, wide, count, x.g);
    else load8(static_cast<const float*>(t.grad) + i0, wide, count, x.g);
    if (kBits == 32) {
        load8(static_cast<const float*>(t.m) + i0, wide, count, x.m);
        load8(static_cast<const float*>(t.v) + i0, wide, count, x.v);
    } else {
        const uint8_t* mb = static_cast<const uint8_t*>(t.m) + i0;
        const uint8_t* vb = static_cast<const uint8_t*>(t.v) + i0;
        if (wide) {
            mc = *reinterpret_cast<const uint2*>(mb);
            vc = *reinterpret_cast<const uint2*>(vb);
        } else {
            uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < count) {
                    w[i >> 2] |= (uint32_t)mb[i] << (8 * (i & 3));
                    w[2 + (i >> 2)] |= (uint32_t)vb[i] << (8 * (i & 3));
                }
            mc = make_uint2(w[0], w[1]);
            vc = make_uint2(w[2], w[3]);
        }
        ms = t.m_scale[block];
        vs = t.v_scale[block];
    }
    if (t.flags & kMaster) load8(t.master + i0, wide, count, x.p);
    else if (t.flags & kParamBf16) load8(static_cast<const __nv_bfloat16*>(t.param) + i0, wide, count, x.p);
    else load8(static_cast<const float*>(t.param) + i0, wide, count, x.p);
    const float gs = c.dev_grad_scale ? __fmul_rn(c.grad_scale, *c.dev_grad_scale) : c.grad_scale;

    const bool round_param = c.round_up_at_random && (t.flags & (kParamBf16 | kMaster)) == kParamBf16;
    uint4 random = make_uint4(0u, 0u, 0u, 0u);
    if (kBits == 8 || round_param)
        random = philox4x32_10((uint64_t)(t.first_block + block) * (kBlock / 8) + lane, a.keys, 2u);
    const uint32_t rw[4] = {random.x, random.y, random.z, random.w};

    uint32_t m_top = 0u, v_top = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (kBits == 8) {
            x.m[i] = __fmul_rn(e4m3_value(((i < 4 ? mc.x : mc.y) >> (8 * (i & 3))) & 0xFFu), ms);
            const float r = __fmul_rn(e4m3_value(((i < 4 ? vc.x : vc.y) >> (8 * (i & 3))) & 0xFFu), vs);
            x.v[i] = __fmul_rn(r, r);
        }
        const float g = __fmul_rn(x.g[i], gs);
        x.m[i] = __fadd_rn(__fmul_rn(c.beta1, x.m[i]), __fmul_rn(c.one_beta1, g));
        x.v[i] = __fadd_rn(__fmul_rn(c.beta2, x.v[i]), __fmul_rn(__fmul_rn(c.one_beta2, g), g));
        // the 8-bit states store the root, rounded as the definition says; elsewhere it only enters the quotient
        const float root = kBits == 8 ? __fsqrt_rn(x.v[i]) : fast_root(x.v[i]);
        if (kBits == 8) {
            x.v[i] = root;
            m_top = max(m_top, __float_as_uint(x.m[i]) & 0x7FFFFFFFu);
            v_top = max(v_top, __float_as_uint(root) & 0x7FFFFFFFu);
        }
        const float den = __fadd_rn(__fmul_rn(root, c.inv_root), c.eps);
        x.p[i] = __fsub_rn(__fmul_rn(x.p[i], c.decay), __fmul_rn(c.step_size, __fdividef(x.m[i], den)));
    }

    if (kBits == 32) {
        store8(static_cast<float*>(t.m) + i0, wide, count, x.m);
        store8(static_cast<float*>(t.v) + i0, wide, count, x.v);
    } else {
        m_top = __reduce_max_sync(0xFFFFFFFFu, m_top);
        v_top = __reduce_max_sync(0xFFFFFFFFu, v_top);
        float mf, vf;
        ms = block_scale(m_top, &mf);
        vs = block_scale(v_top, &vf);
        uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // the half-word with its bytes exchanged, as 1 + r 2^-16 less one
            const uint32_t r = __byte_perm(rw[i >> 1], 0u, i & 1 ? 0x4423 : 0x4401);
            const float unit = __fadd_rn(__uint_as_float(0x3F800000u | r << 7), -1.0f);
            const uint32_t cm = e4m3_code(fminf(__fmul_rn(fabsf(x.m[i]), mf), 448.0f), unit) | (x.m[i] < 0.0f ? 0x80u : 0u);
            const uint32_t cv = max(e4m3_code(fminf(__fmul_rn(x.v[i], vf), 448.0f), unit), x.v[i] > 0.0f ? 1u : 0u);
            w[i >> 2] |= cm << (8 * (i & 3));
            w[2 + (i >> 2)] |= cv << (8 * (i & 3));
        }
        uint8_t* mb = static_cast<uint8_t*>(t.m) + i0;
        uint8_t* vb = static_cast<uint8_t*>(t.v) + i0;
        if (wide) {
            *reinterpret_cast<uint2*>(mb) = make_uint2(w[0], w[1]);
            *reinterpret_cast<uint2*>(vb) = make_uint2(w[2], w[3]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < count) {
                    mb[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
                    vb[i] = (uint8_t)(w[2 + (i >> 2)] >> (8 * (i & 3)));
                }
        }
        if (lane == 0) {
            t.m_scale[block] = ms;
            t.v_scale[block] = vs;
        }
    }
    if (t.flags & kMaster) store8(t.master + i0, wide, count, x.p);
    if (t.flags & kParamBf16) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = round_param ? pack_out<true>(short_nan(x.p[2 * i]), short_nan(x.p[2 * i + 1]), rw[i])
                               : pack_bf16x2(x.p[2 * i], x.p[2 * i + 1]);
        store8_words(static_cast<__nv_bfloat16*>(t.param) + i0, wide, count, w);
    } else {
        store8(static_cast<float*>(t.param) + i0, wide, count, x.p);
    }
}

template <int kCapacity>
cudaError_t launch(const mvue_adamw_tensor* ts, int64_t count, const Constants& c, uint64_t seed, int state_bits,
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
        const int64_t mine = (s.numel + kTile - 1) / kTile;
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
    auto kernel = state_bits == 8 ? &adamw_kernel<8, kCapacity> : &adamw_kernel<32, kCapacity>;
    return launch_dependent(kernel, dim3((unsigned)tiles), dim3(kThreads), 0, stream, a);
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
    c.dev_grad_scale = cfg->dev_grad_scale;
    c.round_up_at_random = (cfg->options & MVUE_OPT_STOCHASTIC_ROUNDING) != 0;
    int64_t first_block = 0;
    while (count > 0) {
        int64_t used = 0;
        cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
        const cudaError_t e = count <= 32 ? launch<32>(tensors, count, c, cfg->seed, cfg->state_bits, &first_block, &used, st)
                                          : launch<320>(tensors, count, c, cfg->seed, cfg->state_bits, &first_block, &used, st);
        if (e != cudaSuccess) { set_cuda_error(e, "mvue_adamw_step launch"); return MVUE_ERR_CUDA; }
        tensors += used;
        count -= used;
    }
    return MVUE_OK;
}
