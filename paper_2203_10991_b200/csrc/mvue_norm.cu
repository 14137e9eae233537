// Group normalisation with an activation on channels-last maps, forward and backward.
//
// x [n, s, c]: a group is c / groups neighbouring channels of one sample over all s positions.  A thread owns eight
// channels (consecutive where rows allow wide accesses) and walks down the rows, so the constants of its channels stay in
// registers and every sum is first a sum per channel; those become sums per group, or per channel over the samples (the
// gradients of gamma and beta), whatever the number of channels in a group is.  Sums are in binary32 in a fixed order
// (no atomics).  Variances: means first, squares of distances from them afterwards, and parts joined by
//   M2 = sum of M2_i + n_i (mean_i - mean)^2,
// so a mean that is large against the deviation costs no digits.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <numeric>

#include "../../include/mvue_train.h"
#include "mvue_device.cuh"
#include "mvue_internal.h"
#include "mvue_train.cuh"

namespace mvue {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 256;
constexpr int kMaxPieces = 32;       // pieces of eight channels that a block is wide: 256 channels
constexpr int kRowsAhead = 4;        // rows that a thread has in flight

struct NormArgs {
    const void *x, *dy;
    void* out;                       // y, or dx
    int64_t n, s, c, ldx, lddy, ldo;
    int groups, group_size;
    const void *gamma, *beta;        // nullptr: ones, zeros
    int affine_bf16;
    float eps;
    float *mean, *rstd;              // [n, groups]
    // the route through memory: blocks of `rows` rows leave sums per channel
    int64_t rows, chunks;
    int pieces, slabs;               // threads of a block along the channels; blocks along them (the grid's x: sample, slab)
    float2* partial;                 // [n, chunks, c]: (mean, M2), backward (sum dz, sum dz xh)
    float2* coef;                    // backward: [n, groups]: means over the group of gamma dz and of gamma dz xh
    float *dgamma, *dbeta;
};

__device__ __forceinline__ float affine(const void* p, int is_bf16, int64_t i, float none) {
    if (!p) return none;
    return is_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]) : static_cast<const float*>(p)[i];
}

// 1 / (1 + exp(-z))
__device__ __forceinline__ f2 sigmoid(f2 z) {
    float a, b;
    unpair(mul2(z, pair(-1.4426950408889634f)), a, b);
    unpair(add2(pair(fast_exp2(a), fast_exp2(b)), pair(1.0f)), a, b);
    return pair(fast_reciprocal(a), fast_reciprocal(b));
}

template <int kAct>
__device__ __forceinline__ f2 act(f2 z) {
    if (kAct == MVUE_ACT_NONE) return z;
    if (kAct == MVUE_ACT_SILU) return mul2(z, sigmoid(z));
    float a, b;
    unpair(z, a, b);
    if (kAct == MVUE_ACT_RELU) {                                                            // NaN stays
        asm("max.NaN.f32 %0, %0, 0f00000000;" : "+f"(a));
        asm("max.NaN.f32 %0, %0, 0f00000000;" : "+f"(b));
        return pair(a, b);
    }
    const f2 e = pair(erff(a * 0.70710678118654752f), erff(b * 0.70710678118654752f));
    return mul2(mul2(z, pair(0.5f)), add2(e, pair(1.0f)));
}
// d act'(z)
template <int kAct>
__device__ __forceinline__ f2 act_grad(f2 z, f2 d) {
    if (kAct == MVUE_ACT_NONE) return d;
    if (kAct == MVUE_ACT_SILU) {                       // s + z s (1 - s)
        const f2 s = sigmoid(z);
        return mul2(d, fma2(mul2(z, s), fma2(s, pair(-1.0f), pair(1.0f)), s));
    }
    float a, b, da, db;
    unpair(z, a, b);
    if (kAct == MVUE_ACT_RELU) {
        unpair(d, da, db);
        return pair(a <= 0.0f ? 0.0f : da, b <= 0.0f ? 0.0f : db);
    }
    const f2 e = pair(erff(a * 0.70710678118654752f), erff(b * 0.70710678118654752f));
    unpair(mul2(mul2(z, z), pair(-0.72134752044448170f)), a, b);                            // -z^2 / 2 in powers of two
    const f2 density = mul2(pair(fast_exp2(a), fast_exp2(b)), pair(0.39894228040143268f));
    return mul2(d, fma2(z, density, fma2(e, pair(0.5f), pair(0.5f))));
}

__device__ __forceinline__ void pairs(const float (&x)[8], f2 (&p)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) p[j] = pair(x[2 * j], x[2 * j + 1]);
}
__device__ __forceinline__ void unpairs(const f2 (&p)[4], float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) unpair(p[j], x[2 * j], x[2 * j + 1]);
}

// A thread's place: its channels, and its rows first, first + stride, ... below end.
template <bool kWide>
struct Place {
    int64_t n, slab0;
    Cols<kWide> cols;
    int64_t row, end;
    int stride;
    __device__ __forceinline__ Place(const NormArgs& a)
        : n(blockIdx.x / a.slabs), slab0((int64_t)(blockIdx.x % a.slabs) * a.pieces * 8), cols(slab0, a.c, threadIdx.x % a.pieces, a.pieces) {
        stride = kThreads / a.pieces;
        const int ty = threadIdx.x / a.pieces;
        const int64_t r0 = (int64_t)blockIdx.y * a.rows;
        end = min(a.s, r0 + a.rows);
        row = r0 + ty;
        if (ty >= stride || cols.count == 0) row = end;          // threads beyond the last whole row of the block
    }
    // channel j of the thread
    __device__ __forceinline__ int64_t channel(int j) const { return cols.first + (int64_t)j * cols.step; }
};

// ---- forward through memory: means and M2 of a chunk of rows, per channel -------------------------------------------
template <typename T, bool kWide>
__global__ void __launch_bounds__(kThreads) norm_stats_kernel(const __grid_constant__ NormArgs a) {
    grid_dependency_wait();
    __shared__ float s_mean[kThreads * 8], s_m2[kThreads * 8];
    Place<kWide> p(a);
    const int64_t n = p.n;
    const T* x = static_cast<const T*>(a.x) + n * a.s * a.ldx;
    float mean[8] = {}, m2[8] = {}, count = 0.0f;
    for (; p.row < p.end; p.row += (int64_t)p.stride * kRowsAhead) {
        float v[kRowsAhead][8];
        const int rows = (int)min((int64_t)kRowsAhead, (p.end - p.row + p.stride - 1) / p.stride);
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u)
            if (u < rows) p.cols.load(x + (p.row + (int64_t)u * p.stride) * a.ldx, v[u]);
        // the new rows by themselves, then joined with those before
        const float some = (float)rows, inv = 1.0f / some, all = count + some;
        const float share = some / all, weight = count * share;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float sum = 0.0f, dev = 0.0f;
#pragma unroll
            for (int u = 0; u < kRowsAhead; ++u) sum += u < rows ? v[u][j] : 0.0f;
            const float m = sum * inv;
#pragma unroll
            for (int u = 0; u < kRowsAhead; ++u) {
                const float d = u < rows ? v[u][j] - m : 0.0f;
                dev = fmaf(d, d, dev);
            }
            const float delta = m - mean[j];
            mean[j] = fmaf(delta, share, mean[j]);
            m2[j] += fmaf(delta * delta, weight, dev);
        }
        count = all;
    }
    // join the block's rows: thread k of the first pieces * 8 has channel k
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        s_mean[j * kThreads + threadIdx.x] = mean[j];
        s_m2[j * kThreads + threadIdx.x] = m2[j];
    }
    __shared__ float s_count[kThreads];
    s_count[threadIdx.x] = count;
    __syncthreads();
    for (int k = threadIdx.x; k < a.pieces * 8; k += kThreads) {
        const int piece = k % a.pieces, j = k / a.pieces;
        float total = 0.0f, sum = 0.0f, dev = 0.0f;
        for (int t = piece; t < p.stride * a.pieces; t += a.pieces) {
            total += s_count[t];
            sum = fmaf(s_count[t], s_mean[j * kThreads + t], sum);
        }
        if (total == 0.0f) continue;
        const float m = sum / total;
        for (int t = piece; t < p.stride * a.pieces; t += a.pieces) {
            const float d = s_mean[j * kThreads + t] - m;
            dev += fmaf(s_count[t] * d, d, s_m2[j * kThreads + t]);
        }
        const Cols<kWide> mine(p.slab0, a.c, piece, a.pieces);
        if (j < mine.count)
            a.partial[(n * a.chunks + blockIdx.y) * a.c + mine.first + (int64_t)j * mine.step] = make_float2(m, dev);
    }
}

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    return x;
}

// A warp joins the chunks and channels of one group of one sample.
__global__ void __launch_bounds__(kThreads) norm_join_kernel(const __grid_constant__ NormArgs a) {
    grid_dependency_wait();
    const int64_t w = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> 5;
    const int lane = threadIdx.x & 31;
    if (w >= a.n * a.groups) return;
    const int64_t n = w / a.groups, g = w % a.groups, parts = a.chunks * a.group_size;
    const float2* part = a.partial + n * a.chunks * a.c + g * a.group_size;
    const auto rows_of = [&](int64_t chunk) { return (float)min(a.rows, a.s - chunk * a.rows); };
    float sum = 0.0f;
    for (int64_t i = lane; i < parts; i += 32) {
        const int64_t chunk = i / a.group_size;
        sum = fmaf(rows_of(chunk), part[chunk * a.c + i % a.group_size].x, sum);
    }
    const float inv = (float)(1.0 / ((double)a.s * a.group_size));
    const float mean = warp_sum(sum) * inv;
    float dev = 0.0f;
    for (int64_t i = lane; i < parts; i += 32) {
        const int64_t chunk = i / a.group_size;
        const float2 q = part[chunk * a.c + i % a.group_size];
        const float d = q.x - mean;
        dev += fmaf(rows_of(chunk) * d, d, q.y);
    }
    dev = warp_sum(dev);
    if (lane == 0) {
        a.mean[w] = mean;
        a.rstd[w] = 1.0f / sqrtf(fmaf(dev, inv, a.eps));
    }
}

// What the elements of eight channels need: z = (x - mean) slope + shift, slope = rstd gamma, shift = beta; backward
// dx = slope dz - level - tilt (x - mean).
struct Channels {
    f2 neg_mean[4], slope[4], shift[4];

    // stat(j): (mean, rstd) of channel j's group; channel(j) its number, for j < count
    template <typename S, typename C> __device__ __forceinline__ void set(const NormArgs& a, int count, S stat, C channel) {
        float m[8], k[8], b[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            m[j] = k[j] = b[j] = 0.0f;
            if (j < count) {
                const float2 q = stat(j);
                m[j] = -q.x;
                k[j] = q.y * affine(a.gamma, a.affine_bf16, channel(j), 1.0f);
                b[j] = affine(a.beta, a.affine_bf16, channel(j), 0.0f);
            }
        }
        pairs(m, neg_mean);
        pairs(k, slope);
        pairs(b, shift);
    }
    template <int kAct> __device__ __forceinline__ void output(f2 (&x)[4]) const {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = act<kAct>(fma2(add2(x[j], neg_mean[j]), slope[j], shift[j]));
    }
    // x becomes x - mean, d becomes dz = d act'(z)
    template <int kAct> __device__ __forceinline__ void gradient(f2 (&x)[4], f2 (&d)[4]) const {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[j] = add2(x[j], neg_mean[j]);
            d[j] = act_grad<kAct>(fma2(x[j], slope[j], shift[j]), d[j]);
        }
    }
};

template <bool kWide>
__device__ __forceinline__ void set_channels(Channels& k, const NormArgs& a, const Place<kWide>& p) {
    k.set(a, p.cols.count,
          [&](int j) { const int64_t g = p.n * a.groups + p.channel(j) / a.group_size; return make_float2(a.mean[g], a.rstd[g]); },
          [&](int j) { return p.channel(j); });
}

template <typename T, bool kWide, int kAct>
__global__ void __launch_bounds__(kThreads) norm_apply_kernel(const __grid_constant__ NormArgs a) {
    grid_dependency_wait();
    Place<kWide> p(a);
    if (p.row >= p.end) return;
    const int64_t n = p.n;
    const T* x = static_cast<const T*>(a.x) + n * a.s * a.ldx;
    T* y = static_cast<T*>(a.out) + n * a.s * a.ldo;
    Channels k;
    set_channels(k, a, p);
    for (; p.row < p.end; p.row += (int64_t)p.stride * kRowsAhead) {
        float v[kRowsAhead][8];
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u)
            if (p.row + (int64_t)u * p.stride < p.end) p.cols.load(x + (p.row + (int64_t)u * p.stride) * a.ldx, v[u]);
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u)
            if (p.row + (int64_t)u * p.stride < p.end) {
                f2 z[4];
                pairs(v[u], z);
                k.output<kAct>(z);
                unpairs(z, v[u]);
                p.cols.store(y + (p.row + (int64_t)u * p.stride) * a.ldo, v[u]);
            }
    }
}

// ---- backward through memory -----------------------------------------------------------------------------------------
// Sums per channel over a chunk of rows of dz = dy act'(z) and of dz (x - mean) rstd.
template <typename T, bool kWide, int kAct>
__global__ void __launch_bounds__(kThreads) norm_grad_sums_kernel(const __grid_constant__ NormArgs a) {
    grid_dependency_wait();
    __shared__ float s_a[kThreads * 8], s_b[kThreads * 8];
    Place<kWide> p(a);
    const int64_t n = p.n;
    const T* x = static_cast<const T*>(a.x) + n * a.s * a.ldx;
    const T* dy = static_cast<const T*>(a.dy) + n * a.s * a.lddy;
    f2 sums[4] = {}, alongs[4] = {};
    if (p.row < p.end) {
        Channels k;
        set_channels(k, a, p);
        for (; p.row < p.end; p.row += (int64_t)p.stride * 2) {
            float v[2][8], d[2][8];
#pragma unroll
            for (int u = 0; u < 2; ++u)
                if (p.row + (int64_t)u * p.stride < p.end) {
                    p.cols.load(x + (p.row + (int64_t)u * p.stride) * a.ldx, v[u]);
                    p.cols.load(dy + (p.row + (int64_t)u * p.stride) * a.lddy, d[u]);
                }
#pragma unroll
            for (int u = 0; u < 2; ++u)
                if (p.row + (int64_t)u * p.stride < p.end) {
                    f2 xc[4], dz[4];
                    pairs(v[u], xc);
                    pairs(d[u], dz);
                    k.gradient<kAct>(xc, dz);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        sums[j] = add2(sums[j], dz[j]);
                        alongs[j] = fma2(dz[j], xc[j], alongs[j]);
                    }
                }
        }
    }
    float sum[8], along[8];
    unpairs(sums, sum);
    unpairs(alongs, along);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        s_a[j * kThreads + threadIdx.x] = sum[j];
        s_b[j * kThreads + threadIdx.x] = along[j];
    }
    __syncthreads();
    for (int k = threadIdx.x; k < a.pieces * 8; k += kThreads) {
        const int piece = k % a.pieces, j = k / a.pieces;
        float ta = 0.0f, tb = 0.0f;
        for (int t = piece; t < p.stride * a.pieces; t += a.pieces) {
            ta += s_a[j * kThreads + t];
            tb += s_b[j * kThreads + t];
        }
        const Cols<kWide> mine(p.slab0, a.c, piece, a.pieces);
        if (j < mine.count) {
            const int64_t c = mine.first + (int64_t)j * mine.step;
            a.partial[(n * a.chunks + blockIdx.y) * a.c + c] = make_float2(ta, tb * a.rstd[n * a.groups + c / a.group_size]);
        }
    }
}

// The first blocks: a warp for the two means of one group of one sample.  The others: sums over samples and chunks for
// 32 channels each, 8 warps share the rows.
__global__ void __launch_bounds__(kThreads) norm_grad_join_kernel(const __grid_constant__ NormArgs a, int64_t group_blocks) {
    grid_dependency_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (blockIdx.x < group_blocks) {
        const int64_t w = (int64_t)blockIdx.x * (kThreads / 32) + warp;
        if (w >= a.n * a.groups) return;
        const int64_t n = w / a.groups, g = w % a.groups, parts = a.chunks * a.group_size;
        const float2* part = a.partial + n * a.chunks * a.c + g * a.group_size;
        float sa = 0.0f, sb = 0.0f;
        for (int64_t i = lane; i < parts; i += 32) {
            const int64_t chunk = i / a.group_size, c = i % a.group_size;
            const float2 q = part[chunk * a.c + c];
            const float gamma = affine(a.gamma, a.affine_bf16, g * a.group_size + c, 1.0f);
            sa = fmaf(gamma, q.x, sa);
            sb = fmaf(gamma, q.y, sb);
        }
        const float inv = (float)(1.0 / ((double)a.s * a.group_size));
        sa = warp_sum(sa) * inv;
        sb = warp_sum(sb) * inv;
        if (lane == 0) a.coef[w] = make_float2(sa, sb);
        return;
    }
    __shared__ float s_a[kThreads], s_b[kThreads];
    const int64_t c = ((int64_t)blockIdx.x - group_blocks) * 32 + lane;
    float sa = 0.0f, sb = 0.0f;
    if (c < a.c)
        for (int64_t i = warp; i < a.n * a.chunks; i += kThreads / 32) {
            const float2 q = a.partial[i * a.c + c];
            sa += q.x;
            sb += q.y;
        }
    s_a[threadIdx.x] = sa;
    s_b[threadIdx.x] = sb;
    __syncthreads();
    if (warp == 0 && c < a.c) {
        for (int w = 1; w < kThreads / 32; ++w) {
            sa += s_a[w * 32 + lane];
            sb += s_b[w * 32 + lane];
        }
        if (a.dbeta) a.dbeta[c] = sa;
        if (a.dgamma) a.dgamma[c] = sb;
    }
}

template <typename T, bool kWide, int kAct>
__global__ void __launch_bounds__(kThreads) norm_grad_apply_kernel(const __grid_constant__ NormArgs a) {
    grid_dependency_wait();
    Place<kWide> p(a);
    if (p.row >= p.end) return;
    const int64_t n = p.n;
    const T* x = static_cast<const T*>(a.x) + n * a.s * a.ldx;
    const T* dy = static_cast<const T*>(a.dy) + n * a.s * a.lddy;
    T* dx = static_cast<T*>(a.out) + n * a.s * a.ldo;
    Channels k;
    set_channels(k, a, p);
    float low[8], off[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int64_t g = n * a.groups + (j < p.cols.count ? p.channel(j) : 0) / a.group_size;
        const float r = a.rstd[g];
        const float2 q = a.coef[g];
        low[j] = -r * q.x;
        off[j] = -r * r * q.y;
    }
    f2 level[4], tilt[4];
    pairs(low, level);
    pairs(off, tilt);
    for (; p.row < p.end; p.row += (int64_t)p.stride * 2) {
        float v[2][8], d[2][8];
#pragma unroll
        for (int u = 0; u < 2; ++u)
            if (p.row + (int64_t)u * p.stride < p.end) {
                p.cols.load(x + (p.row + (int64_t)u * p.stride) * a.ldx, v[u]);
                p.cols.load(dy + (p.row + (int64_t)u * p.stride) * a.lddy, d[u]);
            }
#pragma unroll
        for (int u = 0; u < 2; ++u)
            if (p.row + (int64_t)u * p.stride < p.end) {
                f2 xc[4], dz[4];
                pairs(v[u], xc);
                pairs(d[u], dz);
                k.gradient<kAct>(xc, dz);
#pragma unroll
                for (int j = 0; j < 4; ++j) xc[j] = fma2(k.slope[j], dz[j], fma2(xc[j], tilt[j], level[j]));
                unpairs(xc, v[u]);
                p.cols.store(dx + (p.row + (int64_t)u * p.stride) * a.ldo, v[u]);
            }
    }
}

// ---- resident: a cluster of blocks keeps its part of one sample in shared memory ---------------------------------------
// The route through memory reads x twice (three passes over HBM in all, five in the backward pass).  Here a cluster of up
// to eight blocks takes one slab of whole groups of one sample, every block a run of its rows: the rows are copied to shared
// memory once, a thread reads back only what it copied itself (no barrier between the copy and its use), the blocks
// exchange their groups' sums through distributed shared memory, and the output is formed from the same copy.  One read
// and one write of HBM.
struct ResidentArgs {
    NormArgs norm;
    int cluster, rows, iters;        // blocks of a cluster; rows of a block and of a thread at most
    int fold;                        // a warp holds whole rows of the slab (a power of two of at most 16 pieces)
};

__device__ __forceinline__ void copy16(uint32_t smem, const void* global) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(global) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory"); }

// A thread's rows of one tensor in shared memory: 16-byte slots, consecutive threads side by side.
template <typename T>
struct Slots {
    static constexpr int kHalves = sizeof(T) * 8 / 16, kRowBytes = kHalves * kThreads * 16;
    static __device__ __forceinline__ void fetch(const char* slot, const T* from) {
        const uint32_t to = (uint32_t)__cvta_generic_to_shared(slot);
#pragma unroll
        for (int h = 0; h < kHalves; ++h) copy16(to + h * (kThreads * 16), reinterpret_cast<const char*>(from) + 16 * h);
    }
    static __device__ __forceinline__ void read(const char* slot, f2 (&x)[4]) {
        uint4 w[kHalves];
#pragma unroll
        for (int h = 0; h < kHalves; ++h) w[h] = *reinterpret_cast<const uint4*>(slot + h * (kThreads * 16));
        if (kHalves == 1) {
            x[0] = pair(bf16_lo(w[0].x), bf16_hi(w[0].x));
            x[1] = pair(bf16_lo(w[0].y), bf16_hi(w[0].y));
            x[2] = pair(bf16_lo(w[0].z), bf16_hi(w[0].z));
            x[3] = pair(bf16_lo(w[0].w), bf16_hi(w[0].w));
        } else {
            const uint4 v = w[kHalves - 1];
            x[0] = pair(__uint_as_float(w[0].x), __uint_as_float(w[0].y));
            x[1] = pair(__uint_as_float(w[0].z), __uint_as_float(w[0].w));
            x[2] = pair(__uint_as_float(v.x), __uint_as_float(v.y));
            x[3] = pair(__uint_as_float(v.z), __uint_as_float(v.w));
        }
    }
};
__device__ __forceinline__ void store_row(float* to, const f2 (&x)[4]) {
    float v[8];
    unpairs(x, v);
    store8(to, true, 8, v);
}
__device__ __forceinline__ void store_row(__nv_bfloat16* to, const f2 (&x)[4]) {
    float v[8];
    unpairs(x, v);
    const uint32_t w[4] = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    store8_words(to, true, 8, w);
}
__device__ __forceinline__ void read8(const float* p, f2 (&x)[4]) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    x[0] = pair(a.x, a.y);
    x[1] = pair(a.z, a.w);
    x[2] = pair(b.x, b.y);
    x[3] = pair(b.z, b.w);
}

// Where a block of the cluster stands, and its shared memory.  Values per channel are worked out once per block, by the
// thread that has the channel's number, and read back eight at a time.
template <typename T, int kTensors>
struct Resident {
    const ResidentArgs& a;
    int piece, ty, threads_down, width, channels, groups, rank, rows_here, iters;   // iters: rows of this thread
    int64_t n, c0, row0;             // row0: the thread's first row of the sample
    char* slots[2];
    float *part, *one, *two, *slope, *shift, *group;     // group: two values for each group and block of the cluster

    __device__ __forceinline__ Resident(const ResidentArgs& args, char* smem) : a(args) {
        const NormArgs& q = a.norm;
        const unsigned unit = blockIdx.x / (unsigned)a.cluster;
        rank = (int)(blockIdx.x - unit * a.cluster);
        const unsigned sample = unit / (unsigned)q.slabs;
        n = sample;
        width = q.pieces * 8;
        c0 = (int64_t)(unit - sample * q.slabs) * width;
        channels = (int)min((int64_t)width, q.c - c0);
        groups = channels / q.group_size;
        threads_down = kThreads / q.pieces;
        ty = threadIdx.x / (unsigned)q.pieces;
        piece = threadIdx.x - ty * q.pieces;
        const int r0 = min((int)q.s, rank * a.rows);
        rows_here = min((int)q.s, r0 + a.rows) - r0;
        row0 = r0 + ty;
        const bool mine = ty < threads_down && piece * 8 < channels && ty < rows_here;
        iters = mine ? (rows_here - ty + threads_down - 1) / threads_down : 0;
        const size_t bytes = (size_t)a.iters * Slots<T>::kRowBytes;
        slots[0] = smem + threadIdx.x * 16;
        slots[kTensors - 1] = slots[0] + (kTensors - 1) * bytes;
        float* f = reinterpret_cast<float*>(smem + kTensors * bytes);
        one = f;
        two = one + width;
        slope = two + width;
        shift = slope + width;
        part = shift + width;
        group = part + (a.fold ? kThreads / 32 : threads_down) * width;
    }
    // rows [k / 4, (k + 1) / 4) of the thread
    __device__ __forceinline__ void quarter(int k, int& begin, int& end) const {
        const int q = (a.iters + 3) >> 2;
        begin = k * q;
        end = min(begin + q, iters);
    }
    // sums over the block's rows of every thread's eight values -> into[0 .. channels)
    __device__ __forceinline__ void channel_sums(const f2 (&x)[4], float* into) const {
        f2 v[4] = {x[0], x[1], x[2], x[3]};
        bool writes = ty < threads_down;
        int at = ty;
        if (a.fold) {
            for (int o = a.norm.pieces; o < 32; o <<= 1)
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = add2(v[j], f2{__shfl_xor_sync(0xFFFFFFFFu, v[j].v, o)});
            writes = (threadIdx.x & 31) < (unsigned)a.norm.pieces;
            at = threadIdx.x >> 5;
        }
        if (writes) {
            float w[8];
            unpairs(v, w);
            float4* p = reinterpret_cast<float4*>(part + at * width + piece * 8);
            p[0] = make_float4(w[0], w[1], w[2], w[3]);
            p[1] = make_float4(w[4], w[5], w[6], w[7]);
        }
        __syncthreads();
        const int down = a.fold ? kThreads / 32 : threads_down;
        for (int k = threadIdx.x; k < channels; k += kThreads) {
            const float* p = part + k;
            float s0 = 0.0f, s1 = 0.0f, s2 = 0.0f, s3 = 0.0f;
            int t = 0;
            for (; t + 3 < down; t += 4, p += 4 * width) {
                s0 += p[0];
                s1 += p[width];
                s2 += p[2 * width];
                s3 += p[3 * width];
            }
            for (; t < down; ++t, p += width) s0 += p[0];
            into[k] = (s0 + s1) + (s2 + s3);
        }
        __syncthreads();
    }
    // a warp adds p over the channels of a group; put(group, sum) on every lane
    template <typename P> __device__ __forceinline__ void group_sums(const float* p, P put) const {
        const int lane = threadIdx.x & 31, size = a.norm.group_size;
        for (int g = threadIdx.x >> 5; g < groups; g += kThreads / 32) {
            float s = 0.0f;
            for (int c = lane; c < size; c += 32) s += p[g * size + c];
            put(g, warp_sum(s));
        }
    }
    // this block's two values of a group to all blocks of the cluster, a lane for each
    __device__ __forceinline__ void send(int g, float x, float y) const {
        const int lane = threadIdx.x & 31;
        if (lane >= a.cluster) return;
        float* to = a.cluster > 1 ? cg::this_cluster().map_shared_rank(group, lane) : group;
        *reinterpret_cast<float2*>(to + (rank * groups + g) * 2) = make_float2(x, y);
    }
    __device__ __forceinline__ float2 sent(int block, int g) const { return *reinterpret_cast<const float2*>(group + (block * groups + g) * 2); }
    __device__ __forceinline__ void meet() const {
        if (a.cluster > 1) cg::this_cluster().sync(); else __syncthreads();
    }
};

template <typename T, int kAct>
__global__ void __launch_bounds__(kThreads) norm_resident_kernel(const __grid_constant__ ResidentArgs a) {
    grid_dependency_wait();
    extern __shared__ __align__(16) char smem[];
    const Resident<T, 1> r(a, smem);
    const NormArgs& q = a.norm;
    using S = Slots<T>;
    {
        const int64_t step = (int64_t)r.threads_down * q.ldx;
        const T* x = static_cast<const T*>(q.x) + (r.n * q.s + r.row0) * q.ldx + r.c0 + r.piece * 8;
        char* slot = r.slots[0];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            int i, end;
            for (r.quarter(k, i, end); i < end; ++i, x += step, slot += S::kRowBytes) S::fetch(slot, x);
            copies_end();
        }
    }
    for (int k = threadIdx.x; k < r.channels; k += kThreads) {
        r.slope[k] = affine(q.gamma, q.affine_bf16, r.c0 + k, 1.0f);
        r.shift[k] = affine(q.beta, q.affine_bf16, r.c0 + k, 0.0f);
    }
    if (a.cluster > 1) cg::this_cluster().sync();              // every block of the cluster runs: its memory may be written
    f2 sum[4] = {};
    const auto add = [&](int k) {
        int i, end;
        r.quarter(k, i, end);
        const char* slot = r.slots[0] + i * S::kRowBytes;
#pragma unroll 4
        for (; i < end; ++i, slot += S::kRowBytes) {
            f2 v[4];
            S::read(slot, v);
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[j] = add2(sum[j], v[j]);
        }
    };
    copies_wait<3>(); add(0);
    copies_wait<2>(); add(1);
    copies_wait<1>(); add(2);
    copies_wait<0>(); add(3);
    r.channel_sums(sum, r.one);
    const float own = (float)r.rows_here * q.group_size, inv = own > 0.0f ? 1.0f / own : 0.0f;
    const int lane = threadIdx.x & 31;
    r.group_sums(r.one, [&](int g, float s) {
        __syncwarp();
        for (int c = lane; c < q.group_size; c += 32) r.one[g * q.group_size + c] = -s * inv;     // the block's own mean, per channel
    });
    __syncthreads();
    // squares about the block's own means, from shared memory
    f2 neg_mean[4] = {};
    if (r.iters) read8(r.one + r.piece * 8, neg_mean);
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[j] = pair(0.0f);
    const char* slot = r.slots[0];
#pragma unroll 4
    for (int i = 0; i < r.iters; ++i, slot += S::kRowBytes) {
        f2 v[4];
        S::read(slot, v);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const f2 d = add2(v[j], neg_mean[j]);
            sum[j] = fma2(d, d, sum[j]);
        }
    }
    r.channel_sums(sum, r.two);
    r.group_sums(r.two, [&](int g, float s) { r.send(g, -r.one[g * q.group_size], s); });
    r.meet();
    for (int g = threadIdx.x >> 5; g < r.groups; g += kThreads / 32) {
        // a warp per group, a lane per block of the cluster
        const float2 p = lane < a.cluster ? r.sent(lane, g) : make_float2(0.0f, 0.0f);
        const float rows = lane < a.cluster ? (float)max(0, min(a.rows, (int)q.s - lane * a.rows)) : 0.0f;
        const float mean = warp_sum(rows * p.x) / (float)q.s;
        const float d = p.x - mean;
        const float dev = warp_sum(fmaf(rows * q.group_size * d, d, p.y));
        const float rstd = 1.0f / sqrtf(dev / ((float)q.s * q.group_size) + q.eps);
        for (int c = g * q.group_size + lane; c < (g + 1) * q.group_size; c += 32) {
            r.one[c] = -mean;
            r.slope[c] *= rstd;
        }
        if (r.rank == 0 && lane == 0) {
            const int64_t at = r.n * q.groups + (int)r.c0 / q.group_size + g;
            q.mean[at] = mean;
            q.rstd[at] = rstd;
        }
    }
    __syncthreads();
    if (r.iters == 0) return;
    Channels k8;
    read8(r.one + r.piece * 8, k8.neg_mean);
    read8(r.slope + r.piece * 8, k8.slope);
    read8(r.shift + r.piece * 8, k8.shift);
    T* y = static_cast<T*>(q.out) + (r.n * q.s + r.row0) * q.ldo + r.c0 + r.piece * 8;
    const int64_t down = (int64_t)r.threads_down * q.ldo;
    slot = r.slots[0];
#pragma unroll 2
    for (int i = 0; i < r.iters; ++i, y += down, slot += S::kRowBytes) {
        f2 v[4];
        S::read(slot, v);
        k8.output<kAct>(v);
        store_row(y, v);
    }
}

// Backward: x and dy resident; the block's sums per channel go to `partial` for the gradients of gamma and beta
// (norm_grad_join_kernel), the groups' means through the cluster.
template <typename T, int kAct>
__global__ void __launch_bounds__(kThreads, 2) norm_resident_grad_kernel(const __grid_constant__ ResidentArgs a) {
    grid_dependency_wait();
    extern __shared__ __align__(16) char smem[];
    const Resident<T, 2> r(a, smem);
    const NormArgs& q = a.norm;
    using S = Slots<T>;
    {
        const int64_t step = (int64_t)r.threads_down * q.ldx, dstep = (int64_t)r.threads_down * q.lddy;
        const T* x = static_cast<const T*>(q.x) + (r.n * q.s + r.row0) * q.ldx + r.c0 + r.piece * 8;
        const T* dy = static_cast<const T*>(q.dy) + (r.n * q.s + r.row0) * q.lddy + r.c0 + r.piece * 8;
        char *slot = r.slots[0], *dslot = r.slots[1];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            int i, end;
            for (r.quarter(k, i, end); i < end; ++i, x += step, dy += dstep, slot += S::kRowBytes, dslot += S::kRowBytes) {
                S::fetch(slot, x);
                S::fetch(dslot, dy);
            }
            copies_end();
        }
    }
    const int64_t g0 = r.n * q.groups + (int)r.c0 / q.group_size;
    for (int k = threadIdx.x; k < r.channels; k += kThreads) {
        const int64_t g = g0 + k / q.group_size;
        r.one[k] = -q.mean[g];
        r.slope[k] = q.rstd[g] * affine(q.gamma, q.affine_bf16, r.c0 + k, 1.0f);
        r.shift[k] = affine(q.beta, q.affine_bf16, r.c0 + k, 0.0f);
    }
    r.meet();                        // also: every block of the cluster runs, its memory may be written
    Channels k8 = {};
    if (r.iters) {
        read8(r.one + r.piece * 8, k8.neg_mean);
        read8(r.slope + r.piece * 8, k8.slope);
        read8(r.shift + r.piece * 8, k8.shift);
    }
    f2 sum[4] = {}, along[4] = {};
    const auto add = [&](int k) {
        int i, end;
        r.quarter(k, i, end);
        const char *slot = r.slots[0] + i * S::kRowBytes, *dslot = r.slots[1] + i * S::kRowBytes;
        for (; i < end; ++i, slot += S::kRowBytes, dslot += S::kRowBytes) {
            f2 v[4], d[4];
            S::read(slot, v);
            S::read(dslot, d);
            k8.gradient<kAct>(v, d);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                sum[j] = add2(sum[j], d[j]);
                along[j] = fma2(d[j], v[j], along[j]);
            }
        }
    };
    copies_wait<3>(); add(0);
    copies_wait<2>(); add(1);
    copies_wait<1>(); add(2);
    copies_wait<0>(); add(3);
    __syncthreads();                 // all have read r.one
    r.channel_sums(sum, r.one);
    r.channel_sums(along, r.two);
    for (int k = threadIdx.x; k < r.channels; k += kThreads) {
        const float rstd = q.rstd[g0 + k / q.group_size], gamma = affine(q.gamma, q.affine_bf16, r.c0 + k, 1.0f);
        const float2 s = make_float2(r.one[k], r.two[k] * rstd);
        q.partial[(r.n * a.cluster + r.rank) * q.c + r.c0 + k] = s;
        r.one[k] = gamma * s.x;
        r.two[k] = gamma * s.y;
    }
    __syncthreads();
    const int lane = threadIdx.x & 31;
    r.group_sums(r.one, [&](int g, float s) {
        float t = 0.0f;
        for (int c = lane; c < q.group_size; c += 32) t += r.two[g * q.group_size + c];
        r.send(g, s, warp_sum(t));
    });
    r.meet();
    const float inv = 1.0f / ((float)q.s * q.group_size);
    for (int g = threadIdx.x >> 5; g < r.groups; g += kThreads / 32) {
        const float2 p = lane < a.cluster ? r.sent(lane, g) : make_float2(0.0f, 0.0f);
        const float rstd = q.rstd[g0 + g];
        const float level = -rstd * (warp_sum(p.x) * inv), tilt = -rstd * rstd * (warp_sum(p.y) * inv);
        for (int c = g * q.group_size + lane; c < (g + 1) * q.group_size; c += 32) {
            r.one[c] = level;
            r.two[c] = tilt;
        }
    }
    __syncthreads();
    if (r.iters == 0) return;
    f2 level[4], tilt[4];            // dx = slope dz + level + tilt (x - mean)
    read8(r.one + r.piece * 8, level);
    read8(r.two + r.piece * 8, tilt);
    T* dx = static_cast<T*>(q.out) + (r.n * q.s + r.row0) * q.ldo + r.c0 + r.piece * 8;
    const int64_t down = (int64_t)r.threads_down * q.ldo;
    const char *slot = r.slots[0], *dslot = r.slots[1];
    for (int i = 0; i < r.iters; ++i, dx += down, slot += S::kRowBytes, dslot += S::kRowBytes) {
        f2 v[4], d[4];
        S::read(slot, v);
        S::read(dslot, d);
        k8.gradient<kAct>(v, d);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = fma2(k8.slope[j], d[j], fma2(v[j], tilt[j], level[j]));
        store_row(dx, v);
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------
int64_t size_of(int dtype) { return dtype == MVUE_BF16 ? 2 : 4; }
bool off(const void* p, int64_t size) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(size - 1)) != 0; }
bool wide_rows(const void* p, int64_t ld, int64_t cols, int dtype) { return !off(p, 8 * size_of(dtype)) && cols % 8 == 0 && ld % 8 == 0; }

struct Split {
    int pieces, slabs;
    int64_t rows, chunks;
};
// Blocks of 256 threads, up to 32 along the channels: enough chunks of rows for six blocks on each of 148 SMs, but no
// fewer rows than every thread has in flight at once.
Split split_of(int64_t n, int64_t s, int64_t c) {
    Split p;
    const int64_t all = (c + 7) / 8;
    p.slabs = (int)((all + kMaxPieces - 1) / kMaxPieces);
    p.pieces = (int)((all + p.slabs - 1) / p.slabs);
    const int64_t least = (int64_t)(kThreads / p.pieces) * kRowsAhead;
    const int64_t want = (6 * 148 + n * p.slabs - 1) / std::max<int64_t>(1, n * p.slabs);
    p.chunks = std::max<int64_t>(1, std::min({want, (s + least - 1) / least, (int64_t)65535}));
    p.rows = (s + p.chunks - 1) / p.chunks;
    p.chunks = (s + p.rows - 1) / p.rows;
    return p;
}

constexpr int kMaxCluster = 8;
constexpr size_t kBlockBytes[4] = {56 << 10, 75 << 10, 113 << 10, 226 << 10};     // shared memory of four, three, two and one blocks on an SM

struct Keep {
    int pieces = 0, slabs, cluster, rows, iters, fold;      // pieces = 0: the slab of one sample does not fit a cluster
    size_t smem;
};
// A slab is the fewest whole groups that are whole pieces of eight channels and 128 bytes of a row (or all channels); small
// maps take more, as long as two blocks are left for every SM.  Then the fewest blocks that hold a slab in the
// smallest of the four shares of shared memory that does, and more where the grid would leave SMs idle.
Keep keep_of(int64_t n, int64_t s, int64_t c, int groups, int64_t esz, int tensors) {
    Keep k;
    const int64_t cg = c / groups, least = std::lcm(cg, (int64_t)8);
    if (c % 8 != 0 || least > kThreads * 8) return k;
    int64_t width = std::min(c, (128 / esz + least - 1) / least * least);
    while (width * 2 <= std::min<int64_t>(c, kThreads * 8) && s * width * esz < (8 << 10) && n * ((c + 2 * width - 1) / (2 * width)) >= 2 * 148)
        width *= 2;
    const int pieces = (int)(width / 8), down = kThreads / pieces;
    const int64_t slabs = (c + width - 1) / width, most = width / cg;
    k.fold = pieces <= 16 && (pieces & (pieces - 1)) == 0;
    const auto try_cluster = [&](int cluster, size_t limit) {
        const int64_t rows = (s + cluster - 1) / cluster, iters = (rows + down - 1) / down;
        if (iters > (1 << 16)) return false;
        const size_t smem = (size_t)tensors * iters * esz * 8 * kThreads + 4 * ((4 + (k.fold ? kThreads / 32 : down)) * width + 2 * most * cluster);
        if (smem > limit) return false;
        k.rows = (int)rows;
        k.iters = (int)iters;
        k.cluster = cluster;
        k.smem = smem;
        return true;
    };
    bool found = false;
    for (int level = 0; level < 4 && !found; ++level)
        for (int cluster = 1; cluster <= kMaxCluster && !found; cluster *= 2) found = try_cluster(cluster, kBlockBytes[level]);
    if (!found) return k;
    while (k.cluster < kMaxCluster && n * slabs * k.cluster * 2 <= 2 * 148 && s >= (int64_t)k.cluster * 2 * down)
        if (!try_cluster(k.cluster * 2, kBlockBytes[3])) break;
    if (n * slabs > 0x7FFFFFFF / kMaxCluster) return k;
    k.pieces = pieces;
    k.slabs = (int)slabs;
    return k;
}

template <typename K>
cudaError_t launch_resident(K kernel, PerDeviceOnce& once, const ResidentArgs& a, const Keep& k, cudaStream_t st) {
    cudaError_t e = once_per_device(once, [&](int) {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kBlockBytes[3]);
    });
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.norm.n * k.slabs * k.cluster));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = k.smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)k.cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}

struct Layout {
    size_t partial, coef, mean, rstd, bytes;
};
Layout layout_of(int64_t n, int64_t s, int64_t c, int groups) {
    Layout l;
    size_t at = 0;
    const auto take = [&](size_t b) { const size_t here = at; at += (b + 255) / 256 * 256; return here; };
    l.partial = take((size_t)n * (size_t)std::max<int64_t>(split_of(n, s, c).chunks, kMaxCluster) * (size_t)c * sizeof(float2));
    l.coef = take((size_t)n * groups * sizeof(float2));
    l.mean = take((size_t)n * groups * 4);
    l.rstd = take((size_t)n * groups * 4);
    l.bytes = at;
    return l;
}

template <typename T, bool kWide, int kAct>
cudaError_t forward(const NormArgs& a, dim3 grid, cudaStream_t st) {
    cudaError_t e = launch_dependent(&norm_stats_kernel<T, kWide>, grid, dim3(kThreads), 0, st, a);
    const unsigned joins = (unsigned)((a.n * a.groups + kThreads / 32 - 1) / (kThreads / 32));
    if (e == cudaSuccess) e = launch_dependent(&norm_join_kernel, dim3(joins), dim3(kThreads), 0, st, a);
    if (e == cudaSuccess) e = launch_dependent(&norm_apply_kernel<T, kWide, kAct>, grid, dim3(kThreads), 0, st, a);
    return e;
}
template <typename T, bool kWide, int kAct>
cudaError_t backward(const NormArgs& a, dim3 grid, cudaStream_t st) {
    cudaError_t e = launch_dependent(&norm_grad_sums_kernel<T, kWide, kAct>, grid, dim3(kThreads), 0, st, a);
    const int64_t joins = (a.n * a.groups + kThreads / 32 - 1) / (kThreads / 32);
    const int64_t sums = a.dgamma || a.dbeta ? (a.c + 31) / 32 : 0;
    if (e == cudaSuccess) e = launch_dependent(&norm_grad_join_kernel, dim3((unsigned)(joins + sums)), dim3(kThreads), 0, st, a, joins);
    if (e == cudaSuccess) e = launch_dependent(&norm_grad_apply_kernel<T, kWide, kAct>, grid, dim3(kThreads), 0, st, a);
    return e;
}
template <typename T, bool kWide, int kAct>
cudaError_t either(const NormArgs& a, dim3 grid, cudaStream_t st) {
    if constexpr (kWide) {
        const Keep k = keep_of(a.n, a.s, a.c, a.groups, sizeof(T), a.dy ? 2 : 1);
        if (k.pieces) {
            ResidentArgs r{a, k.cluster, k.rows, k.iters, k.fold};
            r.norm.pieces = k.pieces;
            r.norm.slabs = k.slabs;
            r.norm.chunks = k.cluster;
            static PerDeviceOnce once[2];
            if (!a.dy) return launch_resident(&norm_resident_kernel<T, kAct>, once[0], r, k, st);
            cudaError_t e = launch_resident(&norm_resident_grad_kernel<T, kAct>, once[1], r, k, st);
            if (e == cudaSuccess && (a.dgamma || a.dbeta))
                e = launch_dependent(&norm_grad_join_kernel, dim3((unsigned)((a.c + 31) / 32)), dim3(kThreads), 0, st, r.norm, (int64_t)0);
            return e;
        }
    }
    return a.dy ? backward<T, kWide, kAct>(a, grid, st) : forward<T, kWide, kAct>(a, grid, st);
}
template <typename T, bool kWide>
cudaError_t by_act(const NormArgs& a, int act, dim3 grid, cudaStream_t st) {
    switch (act) {
        case MVUE_ACT_RELU: return either<T, kWide, MVUE_ACT_RELU>(a, grid, st);
        case MVUE_ACT_SILU: return either<T, kWide, MVUE_ACT_SILU>(a, grid, st);
        case MVUE_ACT_GELU: return either<T, kWide, MVUE_ACT_GELU>(a, grid, st);
        default: return either<T, kWide, MVUE_ACT_NONE>(a, grid, st);
    }
}

int check(int dtype, int64_t n, int64_t s, int64_t c, int groups, int affine_dtype, const void* gamma, const void* beta, int act) {
    if (n < 0 || s <= 0 || c <= 0 || groups <= 0 || c % groups != 0) return MVUE_ERR_SHAPE;
    // the grids count samples x slabs of channels and samples x groups
    if (c > 0x7FFFFFFF || s > 0x7FFFFFFF || n > 0x7FFFFFFFll / ((c + 7) / 8) || n > 0x7FFFFFFFll / groups) return MVUE_ERR_SHAPE;
    if (dtype != MVUE_F32 && dtype != MVUE_BF16) return MVUE_ERR_DTYPE;
    if ((gamma || beta) && affine_dtype != MVUE_F32 && affine_dtype != MVUE_BF16) return MVUE_ERR_DTYPE;
    if (act < MVUE_ACT_NONE || act > MVUE_ACT_GELU) return MVUE_ERR_ACT;
    return MVUE_OK;
}

int run(NormArgs& a, int dtype, int act, bool wide, void* workspace, size_t workspace_bytes, void* stream, const char* what) {
    // a forward pass whose samples stay in shared memory leaves nothing outside when it is given room for mean and rstd
    const bool none = wide && !a.dy && a.mean && a.rstd && keep_of(a.n, a.s, a.c, a.groups, size_of(dtype), 1).pieces;
    const Layout l = layout_of(a.n, a.s, a.c, a.groups);
    if (!none && (!workspace || workspace_bytes < l.bytes || off(workspace, 16))) return MVUE_ERR_WORKSPACE;
    DeviceInfo dev;
    if (int e = current_device_info(&dev)) return e;
    char* ws = static_cast<char*>(workspace);
    const Split sp = split_of(a.n, a.s, a.c);
    a.rows = sp.rows;
    a.chunks = sp.chunks;
    a.pieces = sp.pieces;
    a.slabs = sp.slabs;
    a.partial = reinterpret_cast<float2*>(ws + l.partial);
    a.coef = reinterpret_cast<float2*>(ws + l.coef);
    if (!a.mean) a.mean = reinterpret_cast<float*>(ws + l.mean);
    if (!a.rstd) a.rstd = reinterpret_cast<float*>(ws + l.rstd);
    const dim3 grid((unsigned)(a.n * sp.slabs), (unsigned)sp.chunks);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (dtype == MVUE_BF16) e = wide ? by_act<__nv_bfloat16, true>(a, act, grid, st) : by_act<__nv_bfloat16, false>(a, act, grid, st);
    else e = wide ? by_act<float, true>(a, act, grid, st) : by_act<float, false>(a, act, grid, st);
    if (e != cudaSuccess) { set_cuda_error(e, what); return MVUE_ERR_CUDA; }
    return MVUE_OK;
}

}  // namespace
}  // namespace mvue

using namespace mvue;

extern "C" {

int mvue_group_norm_workspace_bytes(int64_t n, int64_t s, int64_t c, int groups, size_t* bytes) {
    if (!bytes) return MVUE_ERR_NULL;
    if (int e = check(MVUE_F32, n, s, c, groups, MVUE_F32, nullptr, nullptr, MVUE_ACT_NONE)) return e;
    *bytes = n == 0 ? 0 : layout_of(n, s, c, groups).bytes;
    return MVUE_OK;
}

int mvue_group_norm_act(const void* x, int dtype, int64_t n, int64_t s, int64_t c, int64_t ldx, int groups, const void* gamma,
                        const void* beta, int affine_dtype, float eps, int act, void* y, int64_t ldy, float* mean, float* rstd,
                        void* workspace, size_t workspace_bytes, void* stream) {
    if (int e = check(dtype, n, s, c, groups, affine_dtype, gamma, beta, act)) return e;
    if (ldx < c || ldy < c) return MVUE_ERR_SHAPE;
    if (n == 0) return MVUE_OK;
    if (!x || !y) return MVUE_ERR_NULL;
    const int64_t esz = size_of(dtype), asz = size_of(affine_dtype);
    if (off(x, esz) || off(y, esz) || off(gamma, asz) || off(beta, asz) || off(mean, 4) || off(rstd, 4)) return MVUE_ERR_ALIGN;
    NormArgs a = {};
    a.x = x; a.out = y; a.n = n; a.s = s; a.c = c; a.ldx = ldx; a.ldo = ldy;
    a.groups = groups; a.group_size = (int)(c / groups);
    a.gamma = gamma; a.beta = beta; a.affine_bf16 = affine_dtype == MVUE_BF16;
    a.eps = eps; a.mean = mean; a.rstd = rstd;
    return run(a, dtype, act, wide_rows(x, ldx, c, dtype) && wide_rows(y, ldy, c, dtype), workspace, workspace_bytes, stream,
               "mvue_group_norm_act launch");
}

int mvue_group_norm_act_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, int dtype, int64_t n, int64_t s, int64_t c,
                                 int groups, const float* mean, const float* rstd, const void* gamma, const void* beta, int affine_dtype,
                                 int act, void* dx, int64_t lddx, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes,
                                 void* stream) {
    if (int e = check(dtype, n, s, c, groups, affine_dtype, gamma, beta, act)) return e;
    if (ldx < c || lddy < c || lddx < c) return MVUE_ERR_SHAPE;
    if (n > 0 && (!x || !dy || !dx || !mean || !rstd)) return MVUE_ERR_NULL;
    const int64_t esz = size_of(dtype), asz = size_of(affine_dtype);
    if (off(x, esz) || off(dy, esz) || off(dx, esz) || off(gamma, asz) || off(beta, asz) || off(mean, 4) || off(rstd, 4) || off(dgamma, 4) ||
        off(dbeta, 4))
        return MVUE_ERR_ALIGN;
    if (n == 0) {
        cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
        cudaError_t e = dgamma ? cudaMemsetAsync(dgamma, 0, (size_t)c * 4, st) : cudaSuccess;
        if (e == cudaSuccess && dbeta) e = cudaMemsetAsync(dbeta, 0, (size_t)c * 4, st);
        if (e != cudaSuccess) { set_cuda_error(e, "mvue_group_norm_act_backward memset"); return MVUE_ERR_CUDA; }
        return MVUE_OK;
    }
    NormArgs a = {};
    a.x = x; a.dy = dy; a.out = dx; a.n = n; a.s = s; a.c = c; a.ldx = ldx; a.lddy = lddy; a.ldo = lddx;
    a.groups = groups; a.group_size = (int)(c / groups);
    a.gamma = gamma; a.beta = beta; a.affine_bf16 = affine_dtype == MVUE_BF16;
    a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);      // only read here
    a.dgamma = dgamma; a.dbeta = dbeta;
    return run(a, dtype, act, wide_rows(x, ldx, c, dtype) && wide_rows(dy, lddy, c, dtype) && wide_rows(dx, lddx, c, dtype), workspace,
               workspace_bytes, stream, "mvue_group_norm_act_backward launch");
}

}  // extern "C"
