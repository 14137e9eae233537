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
    int* dev_status;
    uint32_t polls;                  // after which a wait between the blocks of a cluster gives up
    int mute;                        // nothing is sent between them (the self-test of that exit)
};
constexpr uint32_t kPolls = 1u << 22;         // of 4 us each (measured): 17 s

__device__ __forceinline__ float affine(const void* p, int is_bf16, int64_t i, float none) {
    if (!p) return none;
    return is_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]) : static_cast<const float*>(p)[i];
}

// 1 / (1 + exp(-z)) of two numbers.  Each: by itself, from the exponential of -|z|, which does not overflow; subnormal results
// included, and what is not finite stays on its side.
struct Each {
    static __device__ __forceinline__ float one(float t) {              // t = -z in powers of two
        float e;
        asm("ex2.approx.f32 %0, %1;" : "=f"(e) : "f"(-fabsf(t)));
        return (t > 0.0f ? e : 1.0f) * fast_reciprocal(1.0f + e);
    }
    __device__ __forceinline__ f2 sigmoid(f2 z) {
        float a, b;
        unpair(mul2(z, pair(-1.4426950408889634f)), a, b);
        return pair(one(a), one(b));
    }
};
// Both with one reciprocal, that of the product of the two denominators: the special-function unit takes 16 values a cycle, and
// two each hold up the folded kernels (64 x 3136 x 256 bf16: 53 us against 52 us forward, 107 us against 102 us backward).
// The product is finite while both exponentials are at most 2^60 (z above -41.6); where `held` says that they were not, or
// that there was a NaN, the caller goes over its rows again with Each.  A test of every pair on the way costs 119 us, one of every
// four pairs 108 us.  (3 x 11811 x 320 fp32 through memory: forward 30.6 us against 31.8 us with Each throughout.)
struct Shared {
    float top = 0.0f;
    __device__ __forceinline__ f2 sigmoid(f2 z) {
        float a, b;
        unpair(mul2(z, pair(-1.4426950408889634f)), a, b);
        asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(top) : "f"(a), "f"(b));
        unpair(add2(pair(fast_exp2(a), fast_exp2(b)), pair(1.0f)), a, b);
        return mul2(pair(fast_reciprocal(a * b)), pair(b, a));
    }
    __device__ __forceinline__ bool held() const { return top <= 60.0f; }
};

template <int kAct, typename How>
__device__ __forceinline__ f2 act(f2 z, How& how) {
    if (kAct == MVUE_ACT_NONE) return z;
    if (kAct == MVUE_ACT_SILU) return mul2(z, how.sigmoid(z));
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
template <int kAct, typename How>
__device__ __forceinline__ f2 act_grad(f2 z, f2 d, How& how) {
    if (kAct == MVUE_ACT_NONE) return d;
    if (kAct == MVUE_ACT_SILU) {                       // s + z s (1 - s)
        const f2 s = how.sigmoid(z);
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
template <int kVec>
struct Place {
    int64_t n, slab0;
    Cols<kVec> cols;
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
    __device__ __forceinline__ int64_t channel(int j) const { return cols.at(j); }
};

// Sums over a block's rows of what its threads left per channel: the block's threads share the channels (pieces x 8) and, where
// that leaves threads over, the rows of each.
struct Columns {
    int piece, j, row0, rows, step, share;     // share: threads of a channel
    bool first;
    __device__ __forceinline__ Columns(int pieces) {
        const int channels = pieces * 8, k = threadIdx.x % (unsigned)channels;
        share = kThreads / channels;
        row0 = threadIdx.x / (unsigned)channels;
        piece = k % (unsigned)pieces;
        j = k / (unsigned)pieces;
        first = row0 == 0;
        rows = row0 < share ? kThreads / pieces : 0;
        step = pieces;
    }
    // f(thread, j) for the threads of this channel, added up; the sum on all threads of the channel
    template <typename F> __device__ __forceinline__ float2 sum(F f) const {
        __shared__ float2 s[kThreads];
        __syncthreads();
        float2 t = make_float2(0.0f, 0.0f);
        for (int r = row0; r < rows; r += share) {
            const float2 v = f(piece + r * step, j);
            t.x += v.x;
            t.y += v.y;
        }
        s[threadIdx.x] = t;
        __syncthreads();
        t = make_float2(0.0f, 0.0f);
        if (rows)
            for (int r = 0; r < share; ++r) {
                const float2 v = s[threadIdx.x - (row0 - r) * step * 8];
                t.x += v.x;
                t.y += v.y;
            }
        return t;
    }
};

// ---- forward through memory: means and M2 of a chunk of rows, per channel -------------------------------------------
template <typename T, int kVec>
__global__ void __launch_bounds__(kThreads) norm_stats_kernel(const __grid_constant__ NormArgs a) {
    grid_dependency_wait();
    __shared__ float s_mean[kThreads * 8], s_m2[kThreads * 8];
    Place<kVec> p(a);
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
            m2[j] += fmaf(delta * weight, delta, dev);          // weight first: it is 0 with the first rows, where delta^2 may overflow
        }
        count = all;
    }
    // join the block's rows
    __shared__ float s_count[kThreads];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        s_mean[j * kThreads + threadIdx.x] = mean[j];
        s_m2[j * kThreads + threadIdx.x] = m2[j];
    }
    s_count[threadIdx.x] = count;
    const Columns col(a.pieces);
    const float2 t = col.sum([&](int thread, int j) {
        return make_float2(s_count[thread] * s_mean[j * kThreads + thread], s_count[thread]);
    });
    const float m = t.y > 0.0f ? t.x / t.y : 0.0f;
    const float2 dev = col.sum([&](int thread, int j) {
        const float d = s_mean[j * kThreads + thread] - m;
        return make_float2(fmaf(s_count[thread] * d, d, s_m2[j * kThreads + thread]), 0.0f);
    });
    const Cols<kVec> mine(p.slab0, a.c, col.piece, a.pieces);
    if (col.first && col.j < mine.count)
        a.partial[(n * a.chunks + blockIdx.y) * a.c + mine.at(col.j)] = make_float2(m, dev.x);
}

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    return x;
}

// sum over the block's threads, on all of them
__device__ __forceinline__ float block_total(float x, float* s) {
    x = warp_sum(x);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = x;
    __syncthreads();
    return warp_sum((threadIdx.x & 31) < kThreads / 32 ? s[threadIdx.x & 31] : 0.0f);
}

// A block joins the chunks and channels of one group of one sample (148 chunks of ten channels on a map of 11811
// positions: 42 us with a warp for each group, 64-bit divisions and one load in flight).
__global__ void __launch_bounds__(kThreads) norm_join_kernel(const __grid_constant__ NormArgs a) {
    grid_dependency_wait();
    __shared__ float s[kThreads / 32];
    const int64_t n = blockIdx.x / (unsigned)a.groups;
    const unsigned g = blockIdx.x % (unsigned)a.groups, size = a.group_size, parts = (unsigned)a.chunks * size;
    const float2* part = a.partial + n * a.chunks * a.c + (int64_t)g * size;
    const auto rows_of = [&](unsigned chunk) { return (float)min((int)a.rows, (int)a.s - (int)chunk * (int)a.rows); };
    float sum = 0.0f;
#pragma unroll 4
    for (unsigned i = threadIdx.x; i < parts; i += kThreads) {
        const unsigned chunk = i / size;
        sum = fmaf(rows_of(chunk), part[chunk * a.c + (i - chunk * size)].x, sum);
    }
    const float inv = (float)(1.0 / ((double)a.s * size));
    const float mean = block_total(sum, s) * inv;
    float dev = 0.0f;
#pragma unroll 4
    for (unsigned i = threadIdx.x; i < parts; i += kThreads) {
        const unsigned chunk = i / size;
        const float2 q = part[chunk * a.c + (i - chunk * size)];
        const float d = q.x - mean;
        dev += fmaf(rows_of(chunk) * d, d, q.y);
    }
    dev = block_total(dev, s);
    if (threadIdx.x == 0) {
        a.mean[blockIdx.x] = mean;
        a.rstd[blockIdx.x] = 1.0f / sqrtf(fmaf(dev, inv, a.eps));
    }
}

// The factor of dx: 0 where a group is one element, whose output does not depend on it (the sum of its terms is then the difference
// of two roundings of one product, times rstd).
__device__ __forceinline__ float more_than_one(const NormArgs& a) { return a.s * a.group_size > 1 ? 1.0f : 0.0f; }

// What the elements of a thread's channels need: z = (x - mean) slope + shift, slope = rstd gamma, shift = beta; backward
// dx = slope dz + level + tilt (x - mean).
struct Channels {
    f2 neg_mean[4], slope[4], shift[4];

    template <int kAct, typename How> __device__ __forceinline__ void output(f2 (&x)[4], How& how) const {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = act<kAct>(fma2(add2(x[j], neg_mean[j]), slope[j], shift[j]), how);
    }
    // x becomes x - mean, d becomes dz = d act'(z)
    template <int kAct, typename How> __device__ __forceinline__ void gradient(f2 (&x)[4], f2 (&d)[4], How& how) const {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[j] = add2(x[j], neg_mean[j]);
            d[j] = act_grad<kAct>(fma2(x[j], slope[j], shift[j]), d[j], how);
        }
    }
};

template <int kVec>
__device__ __forceinline__ void set_channels(Channels& k, const NormArgs& a, const Place<kVec>& p) {
    float m[8], t[8], b[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        m[j] = t[j] = b[j] = 0.0f;
        if (j < p.cols.count) {
            const int64_t c = p.channel(j), g = p.n * a.groups + c / a.group_size;
            m[j] = -a.mean[g];
            t[j] = a.rstd[g] * affine(a.gamma, a.affine_bf16, c, 1.0f);
            b[j] = affine(a.beta, a.affine_bf16, c, 0.0f);
        }
    }
    pairs(m, k.neg_mean);
    pairs(t, k.slope);
    pairs(b, k.shift);
}

template <typename T, int kVec, int kAct>
__global__ void __launch_bounds__(kThreads) norm_apply_kernel(const __grid_constant__ NormArgs a) {
    grid_dependency_wait();
    Place<kVec> p(a);
    if (p.row >= p.end) return;
    const int64_t n = p.n;
    const T* x = static_cast<const T*>(a.x) + n * a.s * a.ldx;
    T* y = static_cast<T*>(a.out) + n * a.s * a.ldo;
    Channels k;
    set_channels(k, a, p);
    const auto output = [&](auto& how) {
        for (int64_t row = p.row; row < p.end; row += (int64_t)p.stride * kRowsAhead) {
            float v[kRowsAhead][8];
#pragma unroll
            for (int u = 0; u < kRowsAhead; ++u)
                if (row + (int64_t)u * p.stride < p.end) p.cols.load(x + (row + (int64_t)u * p.stride) * a.ldx, v[u]);
#pragma unroll
            for (int u = 0; u < kRowsAhead; ++u)
                if (row + (int64_t)u * p.stride < p.end) {
                    f2 z[4];
                    pairs(v[u], z);
                    k.output<kAct>(z, how);
                    unpairs(z, v[u]);
                    p.cols.store(y + (row + (int64_t)u * p.stride) * a.ldo, v[u]);
                }
        }
    };
    Shared shared;
    const bool in_place = kAct == MVUE_ACT_SILU && a.out == a.x;      // then the rows cannot be gone over again
    if (!in_place) output(shared);
    if (kAct == MVUE_ACT_SILU && (in_place || !shared.held())) {
        Each each;
        output(each);
    }
}

// ---- backward through memory -----------------------------------------------------------------------------------------
// Sums per channel over a chunk of rows of dz = dy act'(z) and of dz (x - mean) rstd.
template <typename T, int kVec, int kAct>
__global__ void __launch_bounds__(kThreads) norm_grad_sums_kernel(const __grid_constant__ NormArgs a) {
    grid_dependency_wait();
    __shared__ float s_a[kThreads * 8], s_b[kThreads * 8];
    Place<kVec> p(a);
    const int64_t n = p.n;
    const T* x = static_cast<const T*>(a.x) + n * a.s * a.ldx;
    const T* dy = static_cast<const T*>(a.dy) + n * a.s * a.lddy;
    f2 sums[4] = {}, alongs[4] = {};
    if (p.row < p.end) {
        Channels k;
        set_channels(k, a, p);
        const auto add_up = [&](auto& how) {
#pragma unroll
            for (int j = 0; j < 4; ++j) sums[j] = alongs[j] = pair(0.0f);
            for (int64_t row = p.row; row < p.end; row += (int64_t)p.stride * 2) {
                float v[2][8], d[2][8];
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    if (row + (int64_t)u * p.stride < p.end) {
                        p.cols.load(x + (row + (int64_t)u * p.stride) * a.ldx, v[u]);
                        p.cols.load(dy + (row + (int64_t)u * p.stride) * a.lddy, d[u]);
                    }
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    if (row + (int64_t)u * p.stride < p.end) {
                        f2 xc[4], dz[4];
                        pairs(v[u], xc);
                        pairs(d[u], dz);
                        k.gradient<kAct>(xc, dz, how);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            sums[j] = add2(sums[j], dz[j]);
                            alongs[j] = fma2(dz[j], xc[j], alongs[j]);
                        }
                    }
            }
        };
        Shared shared;
        add_up(shared);
        if (kAct == MVUE_ACT_SILU && !shared.held()) {
            Each each;
            add_up(each);
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
    const Columns col(a.pieces);
    const float2 t = col.sum([&](int thread, int j) { return make_float2(s_a[j * kThreads + thread], s_b[j * kThreads + thread]); });
    const Cols<kVec> mine(p.slab0, a.c, col.piece, a.pieces);
    if (col.first && col.j < mine.count) {
        const int64_t c = mine.at(col.j);
        a.partial[(n * a.chunks + blockIdx.y) * a.c + c] = make_float2(t.x, t.y * a.rstd[n * a.groups + c / a.group_size]);
    }
}

// The first blocks: one for the two means of one group of one sample.  The others: sums over samples and chunks for
// 32 channels each, 8 warps share the rows.
__global__ void __launch_bounds__(kThreads) norm_grad_join_kernel(const __grid_constant__ NormArgs a, int64_t group_blocks) {
    grid_dependency_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (blockIdx.x < group_blocks) {
        __shared__ float s[kThreads / 32];
        const int64_t n = blockIdx.x / (unsigned)a.groups;
        const unsigned g = blockIdx.x % (unsigned)a.groups, size = a.group_size, parts = (unsigned)a.chunks * size;
        const float2* part = a.partial + n * a.chunks * a.c + (int64_t)g * size;
        float sa = 0.0f, sb = 0.0f;
#pragma unroll 4
        for (unsigned i = threadIdx.x; i < parts; i += kThreads) {
            const unsigned chunk = i / size, c = i - chunk * size;
            const float2 q = part[chunk * a.c + c];
            const float gamma = affine(a.gamma, a.affine_bf16, (int64_t)g * size + c, 1.0f);
            sa = fmaf(gamma, q.x, sa);
            sb = fmaf(gamma, q.y, sb);
        }
        const float inv = (float)(1.0 / ((double)a.s * size));
        sa = block_total(sa, s) * inv;
        sb = block_total(sb, s) * inv;
        if (threadIdx.x == 0) a.coef[blockIdx.x] = make_float2(sa, sb);
        return;
    }
    __shared__ float s_a[kThreads], s_b[kThreads];
    const int64_t c = ((int64_t)blockIdx.x - group_blocks) * 32 + lane;
    float sa = 0.0f, sb = 0.0f;
    if (c < a.c)
#pragma unroll 4
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

template <typename T, int kVec, int kAct>
__global__ void __launch_bounds__(kThreads) norm_grad_apply_kernel(const __grid_constant__ NormArgs a) {
    grid_dependency_wait();
    Place<kVec> p(a);
    if (p.row >= p.end) return;
    const int64_t n = p.n;
    const T* x = static_cast<const T*>(a.x) + n * a.s * a.ldx;
    const T* dy = static_cast<const T*>(a.dy) + n * a.s * a.lddy;
    T* dx = static_cast<T*>(a.out) + n * a.s * a.ldo;
    Channels k;
    set_channels(k, a, p);
    const float some = more_than_one(a);
    float low[8], off[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int64_t g = n * a.groups + (j < p.cols.count ? p.channel(j) : 0) / a.group_size;
        const float r = a.rstd[g] * some;
        const float2 q = a.coef[g];
        low[j] = -r * q.x;
        off[j] = -r * a.rstd[g] * q.y;
    }
    f2 level[4], tilt[4];
    pairs(low, level);
    pairs(off, tilt);
#pragma unroll
    for (int j = 0; j < 4; ++j) k.slope[j] = mul2(k.slope[j], pair(some));
    const auto output = [&](auto& how) {
        for (int64_t row = p.row; row < p.end; row += (int64_t)p.stride * 2) {
            float v[2][8], d[2][8];
#pragma unroll
            for (int u = 0; u < 2; ++u)
                if (row + (int64_t)u * p.stride < p.end) {
                    p.cols.load(x + (row + (int64_t)u * p.stride) * a.ldx, v[u]);
                    p.cols.load(dy + (row + (int64_t)u * p.stride) * a.lddy, d[u]);
                }
#pragma unroll
            for (int u = 0; u < 2; ++u)
                if (row + (int64_t)u * p.stride < p.end) {
                    f2 xc[4], dz[4];
                    pairs(v[u], xc);
                    pairs(d[u], dz);
                    k.gradient<kAct>(xc, dz, how);
#pragma unroll
                    for (int j = 0; j < 4; ++j) xc[j] = fma2(k.slope[j], dz[j], fma2(xc[j], tilt[j], level[j]));
                    unpairs(xc, v[u]);
                    p.cols.store(dx + (row + (int64_t)u * p.stride) * a.ldo, v[u]);
                }
        }
    };
    Shared shared;
    const bool in_place = kAct == MVUE_ACT_SILU && (a.out == a.dy || a.out == a.x);
    if (!in_place) output(shared);
    if (kAct == MVUE_ACT_SILU && (in_place || !shared.held())) {
        Each each;
        output(each);
    }
}

// ---- resident: a cluster of blocks keeps its part of one sample in shared memory ---------------------------------------
// The route through memory reads x twice (three passes over HBM in all, five in the backward pass).  Here a cluster of up
// to eight blocks takes one slab of whole groups of one sample, every block a run of its rows: the rows are copied to shared
// memory once,a thread reads back only what it copied itself (no barrier between the copy and its use), the blocks
// exchange their groups' sums through distributed shared memory, and the output is formed from the same copy.  One read
// and one write of HBM.  64 x 3136 x 256 bf16 in 32 groups: forward 46 us (ReLU) and 52 us (SiLU) against 31 us of HBM time and
// 101 us through memory, backward 75 us and 102 us against 47 us and 269 us.  Bound by instructions and their latency: 26 and 47
// million warp instructions, 59 % and 45 % of the issue slots with four and two blocks on an SM (registers).  Measured and not
// kept: a second buffer for the next sample (49 us forward, 102 us backward with half the blocks), copies of the next sample
// rolling in behind the last pass (49 us, 110 us: the loops no longer unroll), four channels a thread with four blocks on an SM
// (128 us backward), three blocks at 80 registers (111 us).
struct ResidentArgs {
    NormArgs norm;
    int cluster, rows, iters;        // blocks of a cluster; rows of a block and of a thread at most
    int fold;                        // a warp holds whole rows of the slab (a power of two of at most 16 pieces)
    int units;                       // slabs of all samples
};

__device__ __forceinline__ void copy16(uint32_t smem, const void* global) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(global) : "memory");
}
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// A thread's rows of one tensor in shared memory, eight channels of each: slots of 16 bytes, consecutive threads side by
// side (no bank conflict), two planes of them for fp32.
template <typename T>
struct Slots {
    static constexpr int kParts = sizeof(T) / 2, kRowBytes = kParts * kThreads * 16;
    static __device__ __forceinline__ void fetch(uint32_t to, const T* from) {
#pragma unroll
        for (int h = 0; h < kParts; ++h) copy16(to + h * (kThreads * 16), reinterpret_cast<const char*>(from) + 16 * h);
    }
    static __device__ __forceinline__ void read(const char* slot, f2 (&x)[4]) {
        const uint4 v = *reinterpret_cast<const uint4*>(slot);
        if constexpr (sizeof(T) == 2) {
            x[0] = pair(bf16_lo(v.x), bf16_hi(v.x));
            x[1] = pair(bf16_lo(v.y), bf16_hi(v.y));
            x[2] = pair(bf16_lo(v.z), bf16_hi(v.z));
            x[3] = pair(bf16_lo(v.w), bf16_hi(v.w));
        } else {
            const uint4 w = *reinterpret_cast<const uint4*>(slot + kThreads * 16);
            x[0] = pair(__uint_as_float(v.x), __uint_as_float(v.y));
            x[1] = pair(__uint_as_float(v.z), __uint_as_float(v.w));
            x[2] = pair(__uint_as_float(w.x), __uint_as_float(w.y));
            x[3] = pair(__uint_as_float(w.z), __uint_as_float(w.w));
        }
    }
    static __device__ __forceinline__ void store(T* to, const f2 (&x)[4]) {
        float v[8];
        unpairs(x, v);
        if constexpr (sizeof(T) == 2) {
            const uint32_t w[4] = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
            store8_words(to, true, 8, w);
        } else {
            store8(to, true, 8, v);
        }
    }
};
// eight values per channel from shared memory
__device__ __forceinline__ void read_values(const float* p, f2 (&x)[4]) {
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
    using S = Slots<T>;
    const ResidentArgs& a;
    int piece, ty, threads_down, width, rank, rows_here, iters, row0;      // iters: rows of this thread below row0, its first one
    int channels, groups;            // of the unit at hand
    int64_t n, c0;
    bool mine;                       // the thread's piece exists in the unit at hand
    bool lost = false;               // a wait of this thread ran out
    char* smem;
    size_t tensor_bytes;
    float *part, *one, *two, *slope, *shift, *group;     // group: two values for each group and block of the cluster, two units deep
    unsigned long long* bars;

    __device__ __forceinline__ Resident(const ResidentArgs& args, char* shared) : a(args), smem(shared) {
        const NormArgs& q = a.norm;
        rank = (int)(blockIdx.x % (unsigned)a.cluster);
        width = q.pieces * 8;
        threads_down = kThreads / q.pieces;
        ty = threadIdx.x / (unsigned)q.pieces;
        piece = threadIdx.x - ty * q.pieces;
        const int r0 = min((int)q.s, rank * a.rows);
        rows_here = min((int)q.s, r0 + a.rows) - r0;
        row0 = r0 + ty;
        iters = ty < threads_down && ty < rows_here ? (rows_here - ty + threads_down - 1) / threads_down : 0;
        tensor_bytes = (size_t)a.iters * S::kRowBytes;
        bars = reinterpret_cast<unsigned long long*>(smem + kTensors * tensor_bytes);
        one = reinterpret_cast<float*>(bars + 2);
        two = one + width;
        slope = two + width;
        shift = slope + width;
        part = shift + width;
        group = part + (a.fold ? kThreads / 32 : threads_down) * width;
    }
    __device__ __forceinline__ void place(unsigned unit, int64_t& sample, int64_t& first) const {
        const unsigned i = unit / (unsigned)a.norm.slabs;
        sample = i;
        first = (int64_t)(unit - i * a.norm.slabs) * width;
    }
    __device__ __forceinline__ void enter(unsigned unit) {
        place(unit, n, c0);
        channels = (int)min((int64_t)width, a.norm.c - c0);
        groups = channels / a.norm.group_size;
        mine = iters > 0 && exists();
    }
    __device__ __forceinline__ bool exists() const { return piece * 8 < channels; }
    __device__ __forceinline__ int64_t channel() const { return c0 + piece * 8; }      // the thread's first one
    // the thread's first slot of a tensor
    __device__ __forceinline__ char* slots(int tensor) const { return smem + tensor * tensor_bytes + threadIdx.x * 16; }
    // the thread's channels of its first row of this unit
    template <typename P> __device__ __forceinline__ P* at(P* base, int64_t ld) const { return base + (n * a.norm.s + row0) * ld + channel(); }
    // starts the copies of a unit's rows
    __device__ __forceinline__ void fetch(unsigned unit) const {
        int64_t sample, first;
        place(unit, sample, first);
        const NormArgs& q = a.norm;
        if (piece * 8 < q.c - first)
#pragma unroll
            for (int t = 0; t < kTensors; ++t) {
                const int64_t ld = t ? q.lddy : q.ldx, step = (int64_t)threads_down * ld;
                const T* from = static_cast<const T*>(t ? q.dy : q.x) + (sample * q.s + row0) * ld + first + piece * 8;
                uint32_t to = (uint32_t)__cvta_generic_to_shared(slots(t));
#pragma unroll 2
                for (int i = 0; i < iters; ++i, from += step, to += S::kRowBytes) S::fetch(to, from);
            }
    }
    // sums over the block's rows of every thread's values -> into[0 .. channels)
    __device__ __forceinline__ void channel_sums(const f2 (&x)[4], float* into) const {
        f2 v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = x[j];
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
#pragma unroll
            for (int j = 0; j < 8; j += 4)
                *reinterpret_cast<float4*>(part + at * width + piece * 8 + j) = make_float4(w[j], w[j + 1], w[j + 2], w[j + 3]);
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
    // Exchange of two values per group: each block stores its own into every block's shared memory, where the stores count
    // towards an mbarrier that the block waits on -- unlike a barrier of the cluster this does not wait for the block's
    // earlier stores to global memory.  Units alternate between two places: a block may send those of the next unit while
    // another still reads these, but not those of the one after, since it has to have the other's of the next one first.
    __device__ __forceinline__ float* place_of(int turn, int block, int g) const {
        return group + ((turn * a.cluster + block) * (width / a.norm.group_size) + g) * 2;
    }
    __device__ __forceinline__ uint32_t bar(int turn) const { return (uint32_t)__cvta_generic_to_shared(bars + turn); }
    // once: the barriers exist and every block of the cluster runs
    __device__ __forceinline__ void open() const {
        if (a.cluster == 1) return;
        if (threadIdx.x == 0) {
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar(0)));
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar(1)));
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        cg::this_cluster().sync();
    }
    __device__ __forceinline__ void expect(int turn) const {
        if (a.cluster > 1 && threadIdx.x == 0 && !lost)
            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar(turn)), "r"(a.cluster * groups * 8) : "memory");
    }
    // to the block `block` of the cluster
    __device__ __forceinline__ void send(int turn, int block, int g, float x, float y) const {
        float* to = place_of(turn, rank, g);
        if (a.cluster == 1) {
            *reinterpret_cast<float2*>(to) = make_float2(x, y);
            return;
        }
        if (lost || a.norm.mute) return;                     // after a wait that ran out nobody counts any more
        uint32_t there, counter;
        asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"((uint32_t)__cvta_generic_to_shared(to)), "r"(block));
        asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(counter) : "r"(bar(turn)), "r"(block));
        asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(there), "f"(x), "f"(y),
                     "r"(counter) : "memory");
    }
    __device__ __forceinline__ float2 sent(int turn, int block, int g) const { return *reinterpret_cast<const float2*>(place_of(turn, block, g)); }
    // Waits for the values of all blocks.  When they do not come: MVUE_ERR_DEVICE_TIMEOUT in dev_status, and the thread waits no
    // more (`lost`) but takes the rest of the way as it is, with NaN in the place of what it has not got, so that all threads
    // meet at the same barriers to the end and nobody takes the outputs for results.
    __device__ __forceinline__ void meet(int turn, uint32_t parity) {
        if (a.cluster == 1) {
            __syncthreads();
            return;
        }
        if (lost) return;
        for (uint32_t spin = 0; spin < a.norm.polls; ++spin) {
            uint32_t done;
            asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                         : "=r"(done) : "r"(bar(turn)), "r"(parity) : "memory");
            if (done) return;
            if (spin > 64) __nanosleep(spin > 4096 ? 256 : 32);
        }
        lost = true;
        if (a.norm.dev_status) *a.norm.dev_status = MVUE_ERR_DEVICE_TIMEOUT;
    }
    // x, or NaN where the wait before it ran out
    __device__ __forceinline__ float got(float x) const { return lost ? __uint_as_float(0x7FC00000u) : x; }
    // Before the block ends: nobody stores into its shared memory any more.  Behind the cluster's barrier nothing more is sent,
    // and where every wait of the block has ended all that was sent has arrived.  After one that ran out some of it may
    // still be on its way, for a microsecond or so: the block stays for 200 more.
    __device__ __forceinline__ void close() const {
        if (a.cluster == 1) return;
        cg::this_cluster().sync();
        if (!__syncthreads_or(lost)) return;
        const long long from = clock64();
        for (int i = 0; i < (1 << 16) && clock64() - from < 400000; ++i) __nanosleep(100);
    }
};

// Clusters take units in turn: cluster i the units i, i + clusters, ...
template <typename T, int kAct>
__global__ void __launch_bounds__(kThreads, 2) norm_resident_kernel(const __grid_constant__ ResidentArgs a) {
    grid_dependency_wait();
    extern __shared__ __align__(16) char smem[];
    Resident<T, 1> r(a, smem);
    const NormArgs& q = a.norm;
    using S = Slots<T>;
    const unsigned clusters = gridDim.x / (unsigned)a.cluster;
    unsigned unit = blockIdx.x / (unsigned)a.cluster;
    const int lane = threadIdx.x & 31;
    const float own = (float)r.rows_here * q.group_size, inv = own > 0.0f ? 1.0f / own : 0.0f;
    const float all = (float)q.s * q.group_size;
    const float lane_rows = lane < a.cluster ? (float)max(0, min(a.rows, (int)q.s - lane * a.rows)) : 0.0f;
    r.fetch(unit);
    r.open();
    int turn = 0;
    uint32_t parity = 0;
    for (; unit < (unsigned)a.units; unit += clusters, parity ^= turn, turn ^= 1) {
        r.enter(unit);
        r.expect(turn);
        copies_wait();
        f2 sum[4] = {};
        const int iters = r.mine ? r.iters : 0;
        const char* const first = r.slots(0);
        const char* slot = first;
#pragma unroll 4
        for (int i = 0; i < iters; ++i, slot += S::kRowBytes) {
            f2 v[4];
            S::read(slot, v);
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[j] = add2(sum[j], v[j]);
        }
        r.channel_sums(sum, r.one);
        for (int k = threadIdx.x; k < r.channels; k += kThreads) {
            r.slope[k] = affine(q.gamma, q.affine_bf16, r.c0 + k, 1.0f);
            r.shift[k] = affine(q.beta, q.affine_bf16, r.c0 + k, 0.0f);
        }
        r.group_sums(r.one, [&](int g, float s) {
            __syncwarp();
            for (int c = lane; c < q.group_size; c += 32) r.one[g * q.group_size + c] = -s * inv;     // the block's own mean, per channel
        });
        __syncthreads();
        // squares about the block's own means, from shared memory
        f2 neg_mean[4];
        read_values(r.one + r.piece * 8, neg_mean);
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] = pair(0.0f);
        slot = first;
#pragma unroll 4
        for (int i = 0; i < iters; ++i, slot += S::kRowBytes) {
            f2 v[4];
            S::read(slot, v);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f2 d = add2(v[j], neg_mean[j]);
                sum[j] = fma2(d, d, sum[j]);
            }
        }
        r.channel_sums(sum, r.two);
        r.group_sums(r.two, [&](int g, float s) { if (lane < a.cluster) r.send(turn, lane, g, -r.one[g * q.group_size], s); });
        r.meet(turn, parity);
        for (int g = threadIdx.x >> 5; g < r.groups; g += kThreads / 32) {
            // a warp per group, a lane per block of the cluster
            const float2 p = lane < a.cluster ? r.sent(turn, lane, g) : make_float2(0.0f, 0.0f);
            const float mean = warp_sum(r.got(lane_rows * p.x)) / (float)q.s;
            const float d = p.x - mean;
            const float dev = warp_sum(fmaf(lane_rows * q.group_size * d, d, p.y));
            const float rstd = 1.0f / sqrtf(dev / all + q.eps);
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
        Channels k8;
        read_values(r.one + r.piece * 8, k8.neg_mean);
        read_values(r.slope + r.piece * 8, k8.slope);
        read_values(r.shift + r.piece * 8, k8.shift);
        T* const y0 = r.at(static_cast<T*>(q.out), q.ldo);
        const int64_t down = (int64_t)r.threads_down * q.ldo;
        const auto output = [&](auto& how) {
            T* y = y0;
            const char* from = first;
#pragma unroll 2
            for (int i = 0; i < iters; ++i, y += down, from += S::kRowBytes) {
                f2 v[4];
                S::read(from, v);
                k8.output<kAct>(v, how);
                S::store(y, v);
            }
        };
        Shared shared;
        output(shared);
        if (kAct == MVUE_ACT_SILU && !shared.held()) {
            Each each;
            output(each);
        }
        if (unit + clusters < (unsigned)a.units) r.fetch(unit + clusters);     // each thread has read what it replaces
    }
    copies_wait();
    r.close();
}

// Backward: x and dy resident; the block's sums per channel go to `partial` for the gradients of gamma and beta
// (norm_grad_join_kernel), the groups' means through the cluster.
template <typename T, int kAct>
__global__ void __launch_bounds__(kThreads, 2) norm_resident_grad_kernel(const __grid_constant__ ResidentArgs a) {
    grid_dependency_wait();
    extern __shared__ __align__(16) char smem[];
    Resident<T, 2> r(a, smem);
    const NormArgs& q = a.norm;
    using S = Slots<T>;
    const unsigned clusters = gridDim.x / (unsigned)a.cluster;
    unsigned unit = blockIdx.x / (unsigned)a.cluster;
    const int lane = threadIdx.x & 31;
    const float some = more_than_one(q);
    const float inv = 1.0f / ((float)q.s * q.group_size);
    r.fetch(unit);
    r.open();
    int turn = 0;
    uint32_t parity = 0;
    for (; unit < (unsigned)a.units; unit += clusters, parity ^= turn, turn ^= 1) {
        r.enter(unit);
        r.expect(turn);
        const int64_t g0 = r.n * q.groups + (int)r.c0 / q.group_size;
        __syncthreads();             // the last unit's values per channel have been read
        for (int k = threadIdx.x; k < r.channels; k += kThreads) {
            const int64_t g = g0 + k / q.group_size;
            r.one[k] = -q.mean[g];
            r.slope[k] = q.rstd[g] * affine(q.gamma, q.affine_bf16, r.c0 + k, 1.0f);
            r.shift[k] = affine(q.beta, q.affine_bf16, r.c0 + k, 0.0f);
        }
        copies_wait();
        __syncthreads();
        Channels k8;
        read_values(r.one + r.piece * 8, k8.neg_mean);
        read_values(r.slope + r.piece * 8, k8.slope);
        read_values(r.shift + r.piece * 8, k8.shift);
        f2 sum[4], along[4];
        const int iters = r.mine ? r.iters : 0;
        const auto sums = [&](auto& how) {
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[j] = along[j] = pair(0.0f);
            const char *slot = r.slots(0), *dslot = r.slots(1);
            for (int i = 0; i < iters; ++i, slot += S::kRowBytes, dslot += S::kRowBytes) {
                f2 v[4], d[4];
                S::read(slot, v);
                S::read(dslot, d);
                k8.gradient<kAct>(v, d, how);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    sum[j] = add2(sum[j], d[j]);
                    along[j] = fma2(d[j], v[j], along[j]);
                }
            }
        };
        Shared shared;
        Each each;
        sums(shared);
        const bool held = kAct != MVUE_ACT_SILU || shared.held();
        if (!held) sums(each);
        __syncthreads();             // all have read r.one
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
        r.group_sums(r.one, [&](int g, float s) {
            float t = 0.0f;
            for (int c = lane; c < q.group_size; c += 32) t += r.two[g * q.group_size + c];
            t = warp_sum(t);
            if (lane < a.cluster) r.send(turn, lane, g, s, t);
        });
        r.meet(turn, parity);
        for (int g = threadIdx.x >> 5; g < r.groups; g += kThreads / 32) {
            const float2 p = lane < a.cluster ? r.sent(turn, lane, g) : make_float2(0.0f, 0.0f);
            const float rstd = q.rstd[g0 + g] * some;
            const float level = -rstd * (warp_sum(r.got(p.x)) * inv), tilt = -rstd * rstd * (warp_sum(p.y) * inv);
            for (int c = g * q.group_size + lane; c < (g + 1) * q.group_size; c += 32) {
                r.one[c] = level;
                r.two[c] = tilt;
            }
        }
        __syncthreads();
        f2 level[4], tilt[4];            // dx = slope dz + level + tilt (x - mean)
        read_values(r.one + r.piece * 8, level);
        read_values(r.two + r.piece * 8, tilt);
#pragma unroll
        for (int j = 0; j < 4; ++j) k8.slope[j] = mul2(k8.slope[j], pair(some));
        const int64_t down = (int64_t)r.threads_down * q.ldo;
        const auto output = [&](auto& how) {
            T* dx = r.at(static_cast<T*>(q.out), q.ldo);
            const char *slot = r.slots(0), *dslot = r.slots(1);
            for (int i = 0; i < iters; ++i, dx += down, slot += S::kRowBytes, dslot += S::kRowBytes) {
                f2 v[4], d[4];
                S::read(slot, v);
                S::read(dslot, d);
                k8.gradient<kAct>(v, d, how);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = fma2(k8.slope[j], d[j], fma2(v[j], tilt[j], level[j]));
                S::store(dx, v);
            }
        };
        if (held) output(shared);
        else output(each);
        if (unit + clusters < (unsigned)a.units) r.fetch(unit + clusters);     // each thread has read what it replaces
    }
    copies_wait();
    r.close();
}

// The common case: a warp holds whole rows of the slab and every group is whole pieces of eight channels.  Then a thread's
// eight channels are of one group, a sum over a group is a handful of shuffles and eight values in shared memory, and
// every thread works the group's statistics out for itself: two barriers of the block a unit (one backward), no values per
// channel in shared memory (64 x 3136 x 256 bf16: 57 -> 46 us forward, 129 -> 102 us backward with SiLU).
template <typename T, int kTensors>
struct Folded : Resident<T, kTensors> {
    using Base = Resident<T, kTensors>;
    int per_group, g;                // pieces of a group; the thread's group in the unit
    float* sums;                     // [2][8 warps][pieces][2]

    __device__ __forceinline__ Folded(const ResidentArgs& args, char* shared) : Base(args, shared) {
        per_group = args.norm.group_size / 8;
        g = this->piece / (unsigned)per_group;
        sums = this->one;
        this->group = sums + 2 * (kThreads / 32) * args.norm.pieces * 2;
    }
    // over the warp's lanes of this thread's group
    __device__ __forceinline__ float fold(float x) const {
        for (int o = 1; o < per_group; o <<= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
        for (int o = this->a.norm.pieces; o < 32; o <<= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
        return x;
    }
    // over the block's threads of this thread's group; `half`: calls in turn use different halves, one barrier each
    __device__ __forceinline__ float2 block_sum(float x, float y, int half) const {
        const int pieces = this->a.norm.pieces;
        float2* s = reinterpret_cast<float2*>(sums) + half * (kThreads / 32) * pieces;
        x = fold(x);
        y = fold(y);
        if ((threadIdx.x & 31) < (unsigned)pieces) s[(threadIdx.x >> 5) * pieces + this->piece] = make_float2(x, y);
        __syncthreads();
        float2 t = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) {
            const float2 v = s[w * pieces + this->piece];
            t.x += v.x;
            t.y += v.y;
        }
        return t;
    }
    __device__ __forceinline__ float block_sum(float x, int half) const {
        const int pieces = this->a.norm.pieces;
        float* s = sums + half * (kThreads / 32) * pieces * 2;
        x = fold(x);
        if ((threadIdx.x & 31) < (unsigned)pieces) s[(threadIdx.x >> 5) * pieces + this->piece] = x;
        __syncthreads();
        float t = 0.0f;
#pragma unroll
        for (int w = 0; w < kThreads / 32; ++w) t += s[w * pieces + this->piece];
        return t;
    }
    // one thread for each group of the unit and block of the cluster
    __device__ __forceinline__ bool sends() const {
        return this->ty < this->a.cluster && this->piece == g * per_group && this->exists();
    }
};

__device__ __forceinline__ float total(const f2 (&x)[4]) {
    f2 s = x[0];
#pragma unroll
    for (int j = 1; j < 4; ++j) s = add2(s, x[j]);
    float a, b;
    unpair(s, a, b);
    return a + b;
}
// a thread's values of gamma or beta from channel c on
__device__ __forceinline__ void affine_values(const void* p, int is_bf16, int64_t c, float none, f2 (&x)[4]) {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = affine(p, is_bf16, c + j, none);
    pairs(v, x);
}

template <typename T, int kAct>
__global__ void __launch_bounds__(kThreads, 4) norm_folded_kernel(const __grid_constant__ ResidentArgs a) {
    grid_dependency_wait();
    extern __shared__ __align__(16) char smem[];
    Folded<T, 1> r(a, smem);
    const NormArgs& q = a.norm;
    using S = Slots<T>;
    const unsigned clusters = gridDim.x / (unsigned)a.cluster;
    unsigned unit = blockIdx.x / (unsigned)a.cluster;
    const float own = (float)r.rows_here * q.group_size, inv = own > 0.0f ? 1.0f / own : 0.0f;
    const float all = (float)q.s * q.group_size;
    r.fetch(unit);
    r.open();
    int turn = 0;
    uint32_t parity = 0;
    for (; unit < (unsigned)a.units; unit += clusters, parity ^= turn, turn ^= 1) {
        r.enter(unit);
        r.expect(turn);
        Channels k8;
        if (r.exists()) {
            affine_values(q.gamma, q.affine_bf16, r.channel(), 1.0f, k8.slope);
            affine_values(q.beta, q.affine_bf16, r.channel(), 0.0f, k8.shift);
        }
        copies_wait();
        f2 sum[4] = {};
        const int iters = r.mine ? r.iters : 0;
        const char* const first = r.slots(0);
        const char* slot = first;
#pragma unroll 4
        for (int i = 0; i < iters; ++i, slot += S::kRowBytes) {
            f2 v[4];
            S::read(slot, v);
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[j] = add2(sum[j], v[j]);
        }
        const float block_mean = r.block_sum(total(sum), 0) * inv;
        // squares about the block's own mean, from shared memory
        const f2 low = pair(-block_mean);
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] = pair(0.0f);
        slot = first;
#pragma unroll 4
        for (int i = 0; i < iters; ++i, slot += S::kRowBytes) {
            f2 v[4];
            S::read(slot, v);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f2 d = add2(v[j], low);
                sum[j] = fma2(d, d, sum[j]);
            }
        }
        const float block_dev = r.block_sum(total(sum), 1);
        if (r.sends()) r.send(turn, r.ty, r.g, block_mean, block_dev);
        r.meet(turn, parity);
        float mean = 0.0f, dev = 0.0f;
        int left = (int)q.s;
        for (int b = 0; b < a.cluster; ++b, left -= a.rows) mean = fmaf((float)max(0, min(a.rows, left)), r.sent(turn, b, r.g).x, mean);
        mean = r.got(mean / (float)q.s);
        left = (int)q.s;
        for (int b = 0; b < a.cluster; ++b, left -= a.rows) {
            const float2 p = r.sent(turn, b, r.g);
            const float d = p.x - mean;
            dev += fmaf((float)max(0, min(a.rows, left)) * q.group_size * d, d, p.y);
        }
        const float rstd = 1.0f / sqrtf(dev / all + q.eps);
        if (r.rank == 0 && r.ty == 0 && r.sends()) {
            const int64_t at = r.n * q.groups + (int)r.c0 / q.group_size + r.g;
            q.mean[at] = mean;
            q.rstd[at] = rstd;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            k8.neg_mean[j] = pair(-mean);
            k8.slope[j] = mul2(k8.slope[j], pair(rstd));
        }
        T* const y0 = r.at(static_cast<T*>(q.out), q.ldo);
        const int64_t down = (int64_t)r.threads_down * q.ldo;
        const auto output = [&](auto& how) {
            T* y = y0;
            const char* from = first;
#pragma unroll 2
            for (int i = 0; i < iters; ++i, y += down, from += S::kRowBytes) {
                f2 v[4];
                S::read(from, v);
                k8.output<kAct>(v, how);
                S::store(y, v);
            }
        };
        Shared shared;
        output(shared);
        if (kAct == MVUE_ACT_SILU && !shared.held()) {
            Each each;
            output(each);
        }
        if (unit + clusters < (unsigned)a.units) r.fetch(unit + clusters);     // each thread has read what it replaces
    }
    copies_wait();
    r.close();
}

// Backward.  The grid's clusters are a multiple of the slabs (or there is one for each unit), so a cluster stays with its
// channels and the sums for the gradients of gamma and beta stay in registers until its last sample.
template <typename T, int kAct>
__global__ void __launch_bounds__(kThreads, 2) norm_folded_grad_kernel(const __grid_constant__ ResidentArgs a) {
    grid_dependency_wait();
    extern __shared__ __align__(16) char smem[];
    Folded<T, 2> r(a, smem);
    const NormArgs& q = a.norm;
    using S = Slots<T>;
    const unsigned clusters = gridDim.x / (unsigned)a.cluster;
    const unsigned mine = blockIdx.x / (unsigned)a.cluster;
    unsigned unit = mine;
    const float inv = 1.0f / ((float)q.s * q.group_size);
    r.fetch(unit);
    r.enter(unit);
    const bool has = r.exists();
    f2 gamma[4] = {}, all_sum[4] = {}, all_along[4] = {};
    Channels k8 = {};
    if (has) {
        affine_values(q.gamma, q.affine_bf16, r.channel(), 1.0f, gamma);
        affine_values(q.beta, q.affine_bf16, r.channel(), 0.0f, k8.shift);
    }
    r.open();
    int turn = 0;
    uint32_t parity = 0;
    for (; unit < (unsigned)a.units; unit += clusters, parity ^= turn, turn ^= 1) {
        r.enter(unit);
        r.expect(turn);
        const int64_t g = r.n * q.groups + (int)r.c0 / q.group_size + r.g;
        const float mean = has ? q.mean[g] : 0.0f, rstd = has ? q.rstd[g] : 0.0f;
        copies_wait();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            k8.neg_mean[j] = pair(-mean);
            k8.slope[j] = mul2(gamma[j], pair(rstd));
        }
        f2 sum[4], along[4];
        const int iters = r.mine ? r.iters : 0;
        const auto sums = [&](auto& how) {
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[j] = along[j] = pair(0.0f);
            const char *slot = r.slots(0), *dslot = r.slots(1);
            for (int i = 0; i < iters; ++i, slot += S::kRowBytes, dslot += S::kRowBytes) {
                f2 v[4], d[4];
                S::read(slot, v);
                S::read(dslot, d);
                k8.gradient<kAct>(v, d, how);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    sum[j] = add2(sum[j], d[j]);
                    along[j] = fma2(d[j], v[j], along[j]);
                }
            }
        };
        Shared shared;
        Each each;
        sums(shared);
        const bool held = kAct != MVUE_ACT_SILU || shared.held();
        if (!held) sums(each);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            all_sum[j] = add2(all_sum[j], sum[j]);
            all_along[j] = fma2(along[j], pair(rstd), all_along[j]);
            sum[j] = mul2(sum[j], gamma[j]);
            along[j] = mul2(along[j], gamma[j]);
        }
        const float2 block = r.block_sum(total(sum), total(along), turn);
        if (r.sends()) r.send(turn, r.ty, r.g, block.x, block.y);
        r.meet(turn, parity);
        float sa = 0.0f, sb = 0.0f;
        for (int b = 0; b < a.cluster; ++b) {
            const float2 p = r.sent(turn, b, r.g);
            sa += p.x;
            sb += p.y;
        }
        const f2 level = pair(-rstd * (r.got(sa) * inv)), tilt = pair(-rstd * rstd * (rstd * sb * inv));    // dx = slope dz + level + tilt (x - mean)
        const int64_t down = (int64_t)r.threads_down * q.ldo;
        const auto output = [&](auto& how) {
            T* dx = r.at(static_cast<T*>(q.out), q.ldo);
            const char *slot = r.slots(0), *dslot = r.slots(1);
            for (int i = 0; i < iters; ++i, dx += down, slot += S::kRowBytes, dslot += S::kRowBytes) {
                f2 v[4], d[4];
                S::read(slot, v);
                S::read(dslot, d);
                k8.gradient<kAct>(v, d, how);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = fma2(k8.slope[j], d[j], fma2(v[j], tilt, level));
                S::store(dx, v);
            }
        };
        if (held) output(shared);
        else output(each);
        if (unit + clusters < (unsigned)a.units) r.fetch(unit + clusters);     // each thread has read what it replaces
    }
    copies_wait();
    r.close();
    // the cluster's channels, summed over its samples: the warps' sums through the buffers, which are free now
    __syncthreads();
    float sum[8], along[8];
    unpairs(all_sum, sum);
    unpairs(all_along, along);
    float* scratch = reinterpret_cast<float*>(smem);
    const int pieces = q.pieces, lane = threadIdx.x & 31;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        for (int o = pieces; o < 32; o <<= 1) {
            sum[j] += __shfl_xor_sync(0xFFFFFFFFu, sum[j], o);
            along[j] += __shfl_xor_sync(0xFFFFFFFFu, along[j], o);
        }
        if (lane < pieces) *reinterpret_cast<float2*>(scratch + (((threadIdx.x >> 5) * pieces + lane) * 8 + j) * 2) = make_float2(sum[j], along[j]);
    }
    __syncthreads();
    for (int k = threadIdx.x; k < r.channels; k += kThreads) {
        float2 t = make_float2(0.0f, 0.0f);
        for (int w = 0; w < kThreads / 32; ++w) {
            const float2 v = *reinterpret_cast<const float2*>(scratch + (w * pieces * 8 + k) * 2);
            t.x += v.x;
            t.y += v.y;
        }
        q.partial[((int64_t)(mine / (unsigned)q.slabs) * a.cluster + r.rank) * q.c + r.c0 + k] = t;
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------

struct Split {
    int pieces, slabs;
    int64_t rows, chunks;
};
// Blocks of 256 threads, up to 32 along the channels: as many chunks of rows as two blocks on each of 148 SMs take (six were
// slower, 34 us against 28 us on 3 x 11811 x 320 fp32: every block joins its threads' sums at its end), but no
// fewer rows than every thread has in flight at once.
Split split_of(int64_t n, int64_t s, int64_t c) {
    Split p;
    const int64_t all = (c + 7) / 8;
    p.slabs = (int)((all + kMaxPieces - 1) / kMaxPieces);
    p.pieces = (int)((all + p.slabs - 1) / p.slabs);
    const int64_t least = (int64_t)(kThreads / p.pieces) * kRowsAhead;
    const int64_t want = 2 * 148 / std::max<int64_t>(1, n * p.slabs);
    p.chunks = std::max<int64_t>(1, std::min({want, (s + least - 1) / least, (int64_t)65535}));
    p.rows = (s + p.chunks - 1) / p.chunks;
    p.chunks = (s + p.rows - 1) / p.rows;
    return p;
}

constexpr int kMaxCluster = 8;
// shared memory of a block when four, two and one are on an SM
constexpr size_t kShare[3] = {56 << 10, 113 << 10, 226 << 10};

struct Keep {
    int pieces = 0, slabs, cluster, rows, iters, fold;      // pieces = 0: the slab of one sample does not fit a cluster
    bool folded;                     // the folded kernels: whole rows in a warp, groups of whole pieces
    size_t smem;
};
// A slab is the fewest whole groups that are 64 bytes of a row (two sectors; 128 bytes need twice the blocks to a cluster
// for the same share of shared memory and were no faster) and a multiple of eight channels; small maps take more, as long as two blocks are left for
// every SM.  Then the fewest blocks that hold a slab in the smallest share of shared memory that does (four blocks
// on an SM need 64 registers a thread: the folded forward kernel), and more where the grid would leave SMs idle.
Keep keep_of(int64_t n, int64_t s, int64_t c, int groups, int64_t esz, int tensors) {
    Keep k;
    const int64_t cg = c / groups, least = std::lcm(cg, (int64_t)8);
    if (c % 8 != 0 || least > kThreads * 8) return k;
    const int64_t row = 64 / esz;
    int64_t width = std::min(c, (row + least - 1) / least * least);
    const auto spare = [&](int64_t w) { return s * w * esz < (8 << 10) && n * ((c + 2 * w - 1) / (2 * w)) >= 2 * 148; };
    while (width * 2 <= std::min<int64_t>(c, kThreads * 4) && spare(width)) width *= 2;
    constexpr int cols = 8;
    const int pieces = (int)(width / cols), down = kThreads / pieces;
    const int64_t slabs = (c + width - 1) / width, most = width / cg;
    if (n * slabs > 0x7FFFFFFF / kMaxCluster) return k;
    k.fold = pieces <= 16 && (pieces & (pieces - 1)) == 0;
    k.folded = k.fold && cg % cols == 0;
    const auto fits = [&](int cluster, size_t limit) {
        const int64_t rows = (s + cluster - 1) / cluster, iters = (rows + down - 1) / down;
        if (iters > (1 << 16)) return false;
        const int64_t sums = k.folded ? 4 * (kThreads / 32) * pieces : (4 + (k.fold ? kThreads / 32 : down)) * width;
        const size_t smem = std::max<size_t>((size_t)tensors * iters * esz * cols * kThreads, k.folded && tensors == 2 ? 64 * width : 0) + 16 +
                            4 * (sums + 4 * most * cluster);
        if (smem > limit) return false;
        k.rows = (int)rows;
        k.iters = (int)iters;
        k.cluster = cluster;
        k.smem = smem;
        return true;
    };
    bool found = false;
    for (int share = k.folded && tensors == 1 ? 0 : 1; share < 3 && !found; ++share)
        for (int cluster = 1; cluster <= kMaxCluster && !found; cluster *= 2) found = fits(cluster, kShare[share]);
    if (!found) return k;
    while (k.cluster < kMaxCluster && n * slabs * k.cluster * 2 <= 2 * 148 && s >= (int64_t)k.cluster * 2 * down)
        if (!fits(k.cluster * 2, kShare[2])) break;
    k.pieces = pieces;
    k.slabs = (int)slabs;
    return k;
}

// What a launch needs to know of the device: how many clusters of a size and an amount of shared memory are resident at once.
struct ClusterFacts {
    std::mutex mu;
    struct { int dev, cluster, count; size_t smem; } known[16];
    int filled = 0, next = 0;
};
template <typename K>
cudaError_t launch_resident(K kernel, PerDeviceOnce& once, ClusterFacts& facts, const ResidentArgs& a, const Keep& k, int multiple,
                            int* launched, cudaStream_t st) {
    cudaError_t e = once_per_device(once, [&](int) {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kShare[2]);
    });
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = k.smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)k.cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int clusters = a.units;
    if ((int64_t)a.units * k.cluster > 148) {
        int dev = 0;
        e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        std::lock_guard<std::mutex> lock(facts.mu);
        int count = 0;
        for (int i = 0; i < facts.filled; ++i)
            if (facts.known[i].dev == dev && facts.known[i].cluster == k.cluster && facts.known[i].smem == k.smem) count = facts.known[i].count;
        if (count == 0) {
            cfg.gridDim = dim3((unsigned)k.cluster);
            e = cudaOccupancyMaxActiveClusters(&count, kernel, &cfg);
            if (e != cudaSuccess) return e;
            facts.known[facts.next] = {dev, k.cluster, count, k.smem};
            facts.next = (facts.next + 1) % 16;
            facts.filled = std::min(16, facts.filled + 1);
        }
        // each cluster with one slab of the channels where that is asked for
        if (count < clusters) clusters = std::max(multiple, count / multiple * multiple);
    }
    *launched = clusters;
    cfg.gridDim = dim3((unsigned)(clusters * k.cluster));
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

template <typename T, int kVec, int kAct>
cudaError_t forward(const NormArgs& a, dim3 grid, cudaStream_t st) {
    cudaError_t e = launch_dependent(&norm_stats_kernel<T, kVec>, grid, dim3(kThreads), 0, st, a);
    const unsigned joins = (unsigned)(a.n * a.groups);
    if (e == cudaSuccess) e = launch_dependent(&norm_join_kernel, dim3(joins), dim3(kThreads), 0, st, a);
    if (e == cudaSuccess) e = launch_dependent(&norm_apply_kernel<T, kVec, kAct>, grid, dim3(kThreads), 0, st, a);
    return e;
}
template <typename T, int kVec, int kAct>
cudaError_t backward(const NormArgs& a, dim3 grid, cudaStream_t st) {
    cudaError_t e = launch_dependent(&norm_grad_sums_kernel<T, kVec, kAct>, grid, dim3(kThreads), 0, st, a);
    const int64_t joins = a.n * a.groups;
    const int64_t sums = a.dgamma || a.dbeta ? (a.c + 31) / 32 : 0;
    if (e == cudaSuccess) e = launch_dependent(&norm_grad_join_kernel, dim3((unsigned)(joins + sums)), dim3(kThreads), 0, st, a, joins);
    if (e == cudaSuccess) e = launch_dependent(&norm_grad_apply_kernel<T, kVec, kAct>, grid, dim3(kThreads), 0, st, a);
    return e;
}
template <typename T, int kVec, int kAct>
cudaError_t either(const NormArgs& a, dim3 grid, cudaStream_t st) {
    if constexpr (kVec == 8) {
        const Keep k = keep_of(a.n, a.s, a.c, a.groups, sizeof(T), a.dy ? 2 : 1);
        if (k.pieces) {
            ResidentArgs r{a, k.cluster, k.rows, k.iters, k.fold, (int)(a.n * k.slabs)};
            r.norm.pieces = k.pieces;
            r.norm.slabs = k.slabs;
            r.norm.chunks = k.cluster;
            static PerDeviceOnce once[4];
            static ClusterFacts facts[4];
            const bool folded = k.folded;
            int clusters = 0;
            if (!a.dy)
                return folded ? launch_resident(&norm_folded_kernel<T, kAct>, once[0], facts[0], r, k, 1, &clusters, st)
                              : launch_resident(&norm_resident_kernel<T, kAct>, once[1], facts[1], r, k, 1, &clusters, st);
            cudaError_t e = folded ? launch_resident(&norm_folded_grad_kernel<T, kAct>, once[2], facts[2], r, k, k.slabs, &clusters, st)
                                   : launch_resident(&norm_resident_grad_kernel<T, kAct>, once[3], facts[3], r, k, 1, &clusters, st);
            if (folded) {            // a row of sums per cluster and block, not per sample and block
                r.norm.n = clusters / k.slabs;
            }
            if (e == cudaSuccess && (a.dgamma || a.dbeta))
                e = launch_dependent(&norm_grad_join_kernel, dim3((unsigned)((a.c + 31) / 32)), dim3(kThreads), 0, st, r.norm, (int64_t)0);
            return e;
        }
    }
    return a.dy ? backward<T, kVec, kAct>(a, grid, st) : forward<T, kVec, kAct>(a, grid, st);
}
template <typename T, int kVec>
cudaError_t by_act(const NormArgs& a, int act, dim3 grid, cudaStream_t st) {
    switch (act) {
        case MVUE_ACT_RELU: return either<T, kVec, MVUE_ACT_RELU>(a, grid, st);
        case MVUE_ACT_SILU: return either<T, kVec, MVUE_ACT_SILU>(a, grid, st);
        case MVUE_ACT_GELU: return either<T, kVec, MVUE_ACT_GELU>(a, grid, st);
        default: return either<T, kVec, MVUE_ACT_NONE>(a, grid, st);
    }
}

int check(int dtype, int64_t n, int64_t s, int64_t c, int groups, int affine_dtype, const void* gamma, const void* beta, int act) {
    if (n < 0 || s <= 0 || c <= 0 || groups <= 0 || c % groups != 0) return MVUE_ERR_SHAPE;
    // the grids count samples x slabs of channels and samples x groups, the joins chunks (at most 65535) x channels of a group
    if (c > 0x7FFFFFFF || s > 0x7FFFFFFF || n > 0x7FFFFFFFll / ((c + 7) / 8) || n > 0x7FFFFFFFll / groups ||
        split_of(n, s, c).chunks * (c / groups) > 0x7FFFFFFF)
        return MVUE_ERR_SHAPE;
    if (dtype != MVUE_F32 && dtype != MVUE_BF16) return MVUE_ERR_DTYPE;
    if ((gamma || beta) && affine_dtype != MVUE_F32 && affine_dtype != MVUE_BF16) return MVUE_ERR_DTYPE;
    if (act < MVUE_ACT_NONE || act > MVUE_ACT_GELU) return MVUE_ERR_ACT;
    return MVUE_OK;
}

int run(NormArgs& a, int dtype, int act, int vec, void* workspace, size_t workspace_bytes, void* stream, const char* what) {
    // a forward pass whose samples stay in shared memory leaves nothing outside when it is given room for mean and rstd
    const bool none = vec == 8 && !a.dy && a.mean && a.rstd && keep_of(a.n, a.s, a.c, a.groups, size_of(dtype), 1).pieces;
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
    if (dtype == MVUE_BF16) e = vec == 8 ? by_act<__nv_bfloat16, 8>(a, act, grid, st) : vec == 2 ? by_act<__nv_bfloat16, 2>(a, act, grid, st) : by_act<__nv_bfloat16, 1>(a, act, grid, st);
    else e = vec == 8 ? by_act<float, 8>(a, act, grid, st) : vec == 2 ? by_act<float, 2>(a, act, grid, st) : by_act<float, 1>(a, act, grid, st);
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
                        void* workspace, size_t workspace_bytes, int* dev_status, void* stream) {
    if (int e = check(dtype, n, s, c, groups, affine_dtype, gamma, beta, act)) return e;
    if (ldx < c || ldy < c) return MVUE_ERR_SHAPE;
    if (n == 0) return MVUE_OK;
    if (!x || !y) return MVUE_ERR_NULL;
    const int64_t esz = size_of(dtype), asz = size_of(affine_dtype);
    if (off(x, esz) || off(y, esz) || off(gamma, asz) || off(beta, asz) || off(mean, 4) || off(rstd, 4) || off(dev_status, 4)) return MVUE_ERR_ALIGN;
    NormArgs a = {};
    a.x = x; a.out = y; a.n = n; a.s = s; a.c = c; a.ldx = ldx; a.ldo = ldy;
    a.groups = groups; a.group_size = (int)(c / groups);
    a.gamma = gamma; a.beta = beta; a.affine_bf16 = affine_dtype == MVUE_BF16;
    a.eps = eps; a.mean = mean; a.rstd = rstd; a.dev_status = dev_status; a.polls = kPolls;
    return run(a, dtype, act, std::min(row_vector(x, ldx, c, dtype), row_vector(y, ldy, c, dtype)), workspace, workspace_bytes, stream,
               "mvue_group_norm_act launch");
}

int mvue_group_norm_act_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, int dtype, int64_t n, int64_t s, int64_t c,
                                 int groups, const float* mean, const float* rstd, const void* gamma, const void* beta, int affine_dtype,
                                 int act, void* dx, int64_t lddx, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes,
                                 int* dev_status, void* stream) {
    if (int e = check(dtype, n, s, c, groups, affine_dtype, gamma, beta, act)) return e;
    if (ldx < c || lddy < c || lddx < c) return MVUE_ERR_SHAPE;
    if (n > 0 && (!x || !dy || !dx || !mean || !rstd)) return MVUE_ERR_NULL;
    const int64_t esz = size_of(dtype), asz = size_of(affine_dtype);
    if (off(x, esz) || off(dy, esz) || off(dx, esz) || off(gamma, asz) || off(beta, asz) || off(mean, 4) || off(rstd, 4) || off(dgamma, 4) ||
        off(dbeta, 4) || off(dev_status, 4))
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
    a.dgamma = dgamma; a.dbeta = dbeta; a.dev_status = dev_status; a.polls = kPolls;
    return run(a, dtype, act, std::min({row_vector(x, ldx, c, dtype), row_vector(dy, lddy, c, dtype), row_vector(dx, lddx, c, dtype)}), workspace,
               workspace_bytes, stream, "mvue_group_norm_act_backward launch");
}

int mvue_selftest_group_norm_timeout(int polls, const void* x, const void* dy, int dtype, int64_t n, int64_t s, int64_t c, int groups,
                                     float* mean, float* rstd, void* out, void* workspace, size_t workspace_bytes, int* dev_status,
                                     void* stream) {
    if (int e = check(dtype, n, s, c, groups, MVUE_F32, nullptr, nullptr, MVUE_ACT_NONE)) return e;
    if (polls <= 0 || polls > (1 << 16) || n == 0) return MVUE_ERR_SHAPE;
    if (!x || !mean || !rstd || !out || !dev_status) return MVUE_ERR_NULL;
    const int64_t esz = size_of(dtype);
    if (off(x, 8 * esz) || off(dy, 8 * esz) || off(out, 8 * esz) || off(mean, 4) || off(rstd, 4) || off(dev_status, 4)) return MVUE_ERR_ALIGN;
    const Keep k = keep_of(n, s, c, groups, esz, dy ? 2 : 1);
    if (!k.pieces || k.cluster < 2) return MVUE_ERR_SHAPE;
    NormArgs a = {};
    a.x = x; a.dy = dy; a.out = out; a.n = n; a.s = s; a.c = c; a.ldx = a.lddy = a.ldo = c;
    a.groups = groups; a.group_size = (int)(c / groups);
    a.eps = 1.0f; a.mean = mean; a.rstd = rstd; a.dev_status = dev_status; a.polls = (uint32_t)polls; a.mute = 1;
    return run(a, dtype, MVUE_ACT_NONE, 8, workspace, workspace_bytes, stream, "mvue_selftest_group_norm_timeout launch");
}

}  // extern "C"
