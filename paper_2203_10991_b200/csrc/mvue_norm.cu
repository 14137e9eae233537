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

__device__ __forceinline__ float sigmoid(float z) { return __fdividef(1.0f, 1.0f + __expf(-z)); }

template <int kAct>
__device__ __forceinline__ float act(float z) {
    if (kAct == MVUE_ACT_RELU) return z < 0.0f ? 0.0f : z;                       // NaN stays
    if (kAct == MVUE_ACT_SILU) return z * sigmoid(z);
    if (kAct == MVUE_ACT_GELU) return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
    return z;
}
template <int kAct>
__device__ __forceinline__ float act_grad(float z) {
    if (kAct == MVUE_ACT_RELU) return z <= 0.0f ? 0.0f : 1.0f;
    if (kAct == MVUE_ACT_SILU) { const float s = sigmoid(z); return fmaf(z * s, 1.0f - s, s); }
    if (kAct == MVUE_ACT_GELU)
        return fmaf(z * 0.39894228040143268f, __expf(-0.5f * z * z), fmaf(0.5f, erff(z * 0.70710678118654752f), 0.5f));
    return 1.0f;
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

// mean, rstd gamma and beta of the thread's channels in sample n
template <bool kWide>
struct Constants {
    float mean[8], slope[8], shift[8];
    __device__ __forceinline__ Constants(const NormArgs& a, const Place<kWide>& p, int64_t n) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool in = j < p.cols.count;
            const int64_t c = in ? p.channel(j) : 0, g = n * a.groups + c / a.group_size;
            mean[j] = in ? a.mean[g] : 0.0f;
            slope[j] = in ? a.rstd[g] * affine(a.gamma, a.affine_bf16, c, 1.0f) : 0.0f;
            shift[j] = in ? affine(a.beta, a.affine_bf16, c, 0.0f) : 0.0f;
        }
    }
};

template <typename T, bool kWide, int kAct>
__global__ void __launch_bounds__(kThreads) norm_apply_kernel(const __grid_constant__ NormArgs a) {
    grid_dependency_wait();
    Place<kWide> p(a);
    if (p.row >= p.end) return;
    const int64_t n = p.n;
    const T* x = static_cast<const T*>(a.x) + n * a.s * a.ldx;
    T* y = static_cast<T*>(a.out) + n * a.s * a.ldo;
    const Constants<kWide> k(a, p, n);
    for (; p.row < p.end; p.row += (int64_t)p.stride * kRowsAhead) {
        float v[kRowsAhead][8];
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u)
            if (p.row + (int64_t)u * p.stride < p.end) p.cols.load(x + (p.row + (int64_t)u * p.stride) * a.ldx, v[u]);
#pragma unroll
        for (int u = 0; u < kRowsAhead; ++u)
            if (p.row + (int64_t)u * p.stride < p.end) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[u][j] = act<kAct>(fmaf(v[u][j] - k.mean[j], k.slope[j], k.shift[j]));
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
    float sum[8] = {}, along[8] = {};
    if (p.row < p.end) {
        const Constants<kWide> k(a, p, n);
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
                if (p.row + (int64_t)u * p.stride < p.end)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float xc = v[u][j] - k.mean[j];
                        const float dz = d[u][j] * act_grad<kAct>(fmaf(xc, k.slope[j], k.shift[j]));
                        sum[j] += dz;
                        along[j] = fmaf(dz, xc, along[j]);
                    }
        }
    }
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
    const Constants<kWide> k(a, p, n);
    float level[8], tilt[8];          // dx = slope dz - level - tilt (x - mean)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int64_t g = n * a.groups + (j < p.cols.count ? p.channel(j) : 0) / a.group_size;
        const float r = a.rstd[g];
        const float2 q = a.coef[g];
        level[j] = r * q.x;
        tilt[j] = r * r * q.y;
    }
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
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float xc = v[u][j] - k.mean[j];
                    const float dz = d[u][j] * act_grad<kAct>(fmaf(xc, k.slope[j], k.shift[j]));
                    v[u][j] = fmaf(k.slope[j], dz, fmaf(xc, -tilt[j], -level[j]));
                }
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
    int cluster, iters;              // blocks of a cluster; rows of a thread at most
    int64_t rows;                    // rows of a block
};

constexpr int kPartPitch = kThreads + 1;

__device__ __forceinline__ void copy16(void* smem, const void* global) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(global) : "memory");
}
template <int kLeft> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory"); }

// A thread's rows of one tensor in shared memory: 16-byte slots, consecutive threads side by side.
template <typename T>
struct Slots {
    static constexpr int kHalves = sizeof(T) * 8 / 16;
    char* base;
    __device__ __forceinline__ Slots(char* area) : base(area + threadIdx.x * 16) {}
    __device__ __forceinline__ void fetch(int i, const T* from) const {
#pragma unroll
        for (int h = 0; h < kHalves; ++h) copy16(base + (i * kHalves + h) * (kThreads * 16), reinterpret_cast<const char*>(from) + 16 * h);
    }
    __device__ __forceinline__ void read(int i, float (&x)[8]) const {
        uint4 w[kHalves];
#pragma unroll
        for (int h = 0; h < kHalves; ++h) w[h] = *reinterpret_cast<const uint4*>(base + (i * kHalves + h) * (kThreads * 16));
        if (kHalves == 1) {
            x[0] = bf16_lo(w[0].x); x[1] = bf16_hi(w[0].x); x[2] = bf16_lo(w[0].y); x[3] = bf16_hi(w[0].y);
            x[4] = bf16_lo(w[0].z); x[5] = bf16_hi(w[0].z); x[6] = bf16_lo(w[0].w); x[7] = bf16_hi(w[0].w);
        } else {
            const uint4 v = w[kHalves - 1];
            x[0] = __uint_as_float(w[0].x); x[1] = __uint_as_float(w[0].y); x[2] = __uint_as_float(w[0].z); x[3] = __uint_as_float(w[0].w);
            x[4] = __uint_as_float(v.x); x[5] = __uint_as_float(v.y); x[6] = __uint_as_float(v.z); x[7] = __uint_as_float(v.w);
        }
    }
};

// Where a block of the cluster stands, and its shared memory.
template <typename T, int kTensors>
struct Resident {
    int pieces, ty, threads_down, group_size, groups_here, channels_here, rank, cluster;
    int64_t n, c0, r0;
    int rows_here, iters;            // of the block; of this thread (0: it has no channels)
    char* area[2];
    float *part, *channel, *group_a, *group_b, *all;

    __device__ __forceinline__ Resident(const ResidentArgs& a, char* smem) {
        const NormArgs& q = a.norm;
        pieces = q.pieces;
        cluster = a.cluster;
        rank = blockIdx.x % cluster;
        const int64_t unit = blockIdx.x / cluster;
        n = unit / q.slabs;
        c0 = (unit % q.slabs) * pieces * 8;
        channels_here = (int)min((int64_t)pieces * 8, q.c - c0);
        group_size = q.group_size;
        groups_here = channels_here / group_size;
        threads_down = kThreads / pieces;
        ty = threadIdx.x / pieces;
        r0 = min(q.s, rank * a.rows);
        rows_here = (int)(min(q.s, r0 + a.rows) - r0);
        const bool mine = ty < threads_down && (int)(threadIdx.x % pieces) * 8 < channels_here;
        iters = mine && ty < rows_here ? (rows_here - ty + threads_down - 1) / threads_down : 0;
        const size_t slots = (size_t)a.iters * Slots<T>::kHalves * kThreads * 16;
        area[0] = smem;
        area[1] = smem + (kTensors - 1) * slots;
        part = reinterpret_cast<float*>(smem + kTensors * slots);
        channel = part + 8 * kPartPitch;
        const int width = pieces * 8, most = width / group_size;
        group_a = channel + 2 * width;
        group_b = group_a + most;
        all = group_b + most;        // [cluster][groups][2]
    }
    __device__ __forceinline__ int64_t first_channel() const { return c0 + (threadIdx.x % pieces) * 8; }
    __device__ __forceinline__ int64_t row(int i) const { return r0 + ty + (int64_t)i * threads_down; }

    // sums over the block's rows of every thread's eight values -> channel[0 .. channels_here)
    __device__ __forceinline__ void channel_sums(const float (&x)[8], float* into) const {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) part[j * kPartPitch + threadIdx.x] = x[j];
        __syncthreads();
        for (int k = threadIdx.x; k < channels_here; k += kThreads) {
            const float* p = part + (k & 7) * kPartPitch + (k >> 3);
            float s0 = 0.0f, s1 = 0.0f;
            int t = 0;
            for (; t + 1 < threads_down; t += 2) {
                s0 += p[t * pieces];
                s1 += p[(t + 1) * pieces];
            }
            if (t < threads_down) s0 += p[t * pieces];
            into[k] = s0 + s1;
        }
        __syncthreads();
    }
    // a warp adds f(channel) over each group and hands the sum to `put(group, sum)` on every lane
    template <typename F, typename P> __device__ __forceinline__ void group_sums(F f, P put) const {
        const int lane = threadIdx.x & 31;
        for (int g = threadIdx.x >> 5; g < groups_here; g += kThreads / 32) {
            float s = 0.0f;
            for (int c = lane; c < group_size; c += 32) s += f(g * group_size + c);
            put(g, warp_sum(s));
        }
    }
    // block `to`'s copy of p (the same place in its shared memory)
    __device__ __forceinline__ float* remote(float* p, int to) const { return cg::this_cluster().map_shared_rank(p, to); }
};

template <typename T, int kAct>
__global__ void __launch_bounds__(kThreads) norm_resident_kernel(const __grid_constant__ ResidentArgs a) {
    grid_dependency_wait();
    extern __shared__ __align__(16) char smem[];
    const Resident<T, 1> r(a, smem);
    const NormArgs& q = a.norm;
    const int64_t c = r.first_channel();
    const T* x = static_cast<const T*>(q.x) + (r.n * q.s + r.row(0)) * q.ldx + c;
    const Slots<T> xs(r.area[0]);
    const int64_t step = (int64_t)r.threads_down * q.ldx;
    const int quarter = (a.iters + 3) / 4;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        for (int i = k * quarter; i < min((k + 1) * quarter, r.iters); ++i) xs.fetch(i, x + i * step);
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    if (r.cluster > 1) cg::this_cluster().sync();              // every block of the cluster runs: its memory may be written
    float sum[8] = {};
    const auto add = [&](int k) {
        for (int i = k * quarter; i < min((k + 1) * quarter, r.iters); ++i) {
            float v[8];
            xs.read(i, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += v[j];
        }
    };
    copies_wait<3>(); add(0);
    copies_wait<2>(); add(1);
    copies_wait<1>(); add(2);
    copies_wait<0>(); add(3);
    r.channel_sums(sum, r.channel);
    const float mine = (float)r.rows_here * r.group_size, inv = mine > 0.0f ? 1.0f / mine : 0.0f;
    r.group_sums([&](int k) { return r.channel[k]; }, [&](int g, float s) { r.group_a[g] = s * inv; });
    __syncthreads();
    // squares about the block's own means, from shared memory
    float mean[8];
    const int first = (int)(c - r.c0);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        mean[j] = r.iters ? r.group_a[(first + j) / r.group_size] : 0.0f;
        sum[j] = 0.0f;
    }
    for (int i = 0; i < r.iters; ++i) {
        float v[8];
        xs.read(i, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float d = v[j] - mean[j];
            sum[j] = fmaf(d, d, sum[j]);
        }
    }
    r.channel_sums(sum, r.channel);
    r.group_sums([&](int k) { return r.channel[k]; }, [&](int g, float s) {
        const int lane = threadIdx.x & 31;
        if (lane < r.cluster) {
            float* to = r.cluster > 1 ? r.remote(r.all, lane) : r.all;
            to[(r.rank * r.groups_here + g) * 2] = r.group_a[g];
            to[(r.rank * r.groups_here + g) * 2 + 1] = s;
        }
    });
    if (r.cluster > 1) cg::this_cluster().sync(); else __syncthreads();
    for (int g = threadIdx.x; g < r.groups_here; g += kThreads) {
        const auto rows_of = [&](int b) { return (float)max((int64_t)0, min(a.rows, q.s - b * a.rows)); };
        const float per_row = 1.0f / (float)q.s;
        float m = 0.0f, dev = 0.0f;
        for (int b = 0; b < r.cluster; ++b) m = fmaf(rows_of(b), r.all[(b * r.groups_here + g) * 2], m);
        m *= per_row;
        for (int b = 0; b < r.cluster; ++b) {
            const float d = r.all[(b * r.groups_here + g) * 2] - m;
            dev += fmaf(rows_of(b) * r.group_size * d, d, r.all[(b * r.groups_here + g) * 2 + 1]);
        }
        const float rstd = 1.0f / sqrtf(dev / ((float)q.s * r.group_size) + q.eps);
        r.group_a[g] = m;
        r.group_b[g] = rstd;
        if (r.rank == 0) {
            const int64_t at = r.n * q.groups + r.c0 / r.group_size + g;
            q.mean[at] = m;
            q.rstd[at] = rstd;
        }
    }
    __syncthreads();
    if (r.iters == 0) return;
    float slope[8], shift[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int g = (first + j) / r.group_size;
        mean[j] = r.group_a[g];
        slope[j] = r.group_b[g] * affine(q.gamma, q.affine_bf16, c + j, 1.0f);
        shift[j] = affine(q.beta, q.affine_bf16, c + j, 0.0f);
    }
    T* y = static_cast<T*>(q.out) + (r.n * q.s + r.row(0)) * q.ldo;
    const Cols<true> cols(c, q.c, 0, 1);
    for (int i = 0; i < r.iters; ++i) {
        float v[8];
        xs.read(i, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = act<kAct>(fmaf(v[j] - mean[j], slope[j], shift[j]));
        cols.store(y + (int64_t)i * r.threads_down * q.ldo, v);
    }
}

// Backward: x and dy resident; the block's sums per channel go to `partial` for the gradients of gamma and beta
// (norm_grad_join_kernel), the groups' means through the cluster.
template <typename T, int kAct>
__global__ void __launch_bounds__(kThreads) norm_resident_grad_kernel(const __grid_constant__ ResidentArgs a) {
    grid_dependency_wait();
    extern __shared__ __align__(16) char smem[];
    const Resident<T, 2> r(a, smem);
    const NormArgs& q = a.norm;
    const int64_t c = r.first_channel();
    const T* x = static_cast<const T*>(q.x) + (r.n * q.s + r.row(0)) * q.ldx + c;
    const T* dy = static_cast<const T*>(q.dy) + (r.n * q.s + r.row(0)) * q.lddy + c;
    const Slots<T> xs(r.area[0]), ds(r.area[1]);
    const int quarter = (a.iters + 3) / 4;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        for (int i = k * quarter; i < min((k + 1) * quarter, r.iters); ++i) {
            xs.fetch(i, x + (int64_t)i * r.threads_down * q.ldx);
            ds.fetch(i, dy + (int64_t)i * r.threads_down * q.lddy);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    if (r.cluster > 1) cg::this_cluster().sync();
    float mean[8], slope[8], shift[8], sum[8] = {}, along[8] = {};
    const int64_t g0 = r.n * q.groups;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int64_t g = g0 + (c + j) / r.group_size;
        mean[j] = r.iters ? q.mean[g] : 0.0f;
        slope[j] = r.iters ? q.rstd[g] * affine(q.gamma, q.affine_bf16, c + j, 1.0f) : 0.0f;
        shift[j] = r.iters ? affine(q.beta, q.affine_bf16, c + j, 0.0f) : 0.0f;
    }
    const auto add = [&](int k) {
        for (int i = k * quarter; i < min((k + 1) * quarter, r.iters); ++i) {
            float v[8], d[8];
            xs.read(i, v);
            ds.read(i, d);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float xc = v[j] - mean[j];
                const float dz = d[j] * act_grad<kAct>(fmaf(xc, slope[j], shift[j]));
                sum[j] += dz;
                along[j] = fmaf(dz, xc, along[j]);
            }
        }
    };
    copies_wait<3>(); add(0);
    copies_wait<2>(); add(1);
    copies_wait<1>(); add(2);
    copies_wait<0>(); add(3);
    float* channel_b = r.channel + r.pieces * 8;
    r.channel_sums(sum, r.channel);
    r.channel_sums(along, channel_b);
    for (int k = threadIdx.x; k < r.channels_here; k += kThreads) {
        const float2 s = make_float2(r.channel[k], channel_b[k] * q.rstd[g0 + (r.c0 + k) / r.group_size]);
        const float gamma = affine(q.gamma, q.affine_bf16, r.c0 + k, 1.0f);
        q.partial[((r.n * r.cluster) + r.rank) * q.c + r.c0 + k] = s;
        r.channel[k] = gamma * s.x;
        channel_b[k] = gamma * s.y;
    }
    __syncthreads();
    const auto send = [&](int which) {
        return [&r, which](int g, float s) {
            const int lane = threadIdx.x & 31;
            if (lane < r.cluster) (r.cluster > 1 ? r.remote(r.all, lane) : r.all)[(r.rank * r.groups_here + g) * 2 + which] = s;
        };
    };
    r.group_sums([&](int k) { return r.channel[k]; }, send(0));
    r.group_sums([&](int k) { return channel_b[k]; }, send(1));
    if (r.cluster > 1) cg::this_cluster().sync(); else __syncthreads();
    const float inv = (float)(1.0 / ((double)q.s * r.group_size));
    for (int g = threadIdx.x; g < r.groups_here; g += kThreads) {
        float sa = 0.0f, sb = 0.0f;
        for (int b = 0; b < r.cluster; ++b) {
            sa += r.all[(b * r.groups_here + g) * 2];
            sb += r.all[(b * r.groups_here + g) * 2 + 1];
        }
        const float rstd = q.rstd[g0 + r.c0 / r.group_size + g];
        r.group_a[g] = rstd * (sa * inv);
        r.group_b[g] = rstd * rstd * (sb * inv);
    }
    __syncthreads();
    if (r.iters == 0) return;
    float level[8], tilt[8];          // dx = slope dz - level - tilt (x - mean)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int g = (int)(c - r.c0 + j) / r.group_size;
        level[j] = r.group_a[g];
        tilt[j] = r.group_b[g];
    }
    T* dx = static_cast<T*>(q.out) + (r.n * q.s + r.row(0)) * q.ldo;
    const Cols<true> cols(c, q.c, 0, 1);
    for (int i = 0; i < r.iters; ++i) {
        float v[8], d[8];
        xs.read(i, v);
        ds.read(i, d);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float xc = v[j] - mean[j];
            const float dz = d[j] * act_grad<kAct>(fmaf(xc, slope[j], shift[j]));
            v[j] = fmaf(slope[j], dz, fmaf(xc, -tilt[j], -level[j]));
        }
        cols.store(dx + (int64_t)i * r.threads_down * q.ldo, v);
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
constexpr size_t kBlockBytes[3] = {56 << 10, 113 << 10, 226 << 10};     // shared memory of four, two and one blocks on an SM

struct Keep {
    int pieces = 0, slabs, cluster, iters;      // pieces = 0: the slab of one sample does not fit a cluster
    int64_t rows;
    size_t smem;
};
// A slab is the fewest whole groups that are whole pieces of eight channels and 128 bytes of a row (or all channels); small
// maps take more, as long as two blocks are left for every SM.  Then the fewest blocks that hold a slab in the
// smallest of the three shares of shared memory that does, and more where the grid would leave SMs idle.
Keep keep_of(int64_t n, int64_t s, int64_t c, int groups, int64_t esz, int tensors) {
    Keep k;
    const int64_t cg = c / groups, least = std::lcm(cg, (int64_t)8);
    if (c % 8 != 0 || least > kThreads * 8) return k;
    int64_t width = std::min(c, (128 / esz + least - 1) / least * least);
    while (width * 2 <= std::min<int64_t>(c, kThreads * 8) && s * width * esz < (8 << 10) && n * ((c + 2 * width - 1) / (2 * width)) >= 2 * 148)
        width *= 2;
    const int pieces = (int)(width / 8), down = kThreads / pieces;
    const int64_t slabs = (c + width - 1) / width, most = width / cg;
    const auto try_cluster = [&](int cluster, size_t limit) {
        const int64_t rows = (s + cluster - 1) / cluster, iters = (rows + down - 1) / down;
        if (iters > (1 << 16)) return false;
        const size_t smem = (size_t)tensors * iters * esz * 8 * kThreads + 4 * (8 * kPartPitch + 2 * width + 2 * most + 2 * most * cluster);
        if (smem > limit) return false;
        k.rows = rows;
        k.iters = (int)iters;
        k.cluster = cluster;
        k.smem = smem;
        return true;
    };
    bool found = false;
    for (int level = 0; level < 3 && !found; ++level)
        for (int cluster = 1; cluster <= kMaxCluster && !found; cluster *= 2) found = try_cluster(cluster, kBlockBytes[level]);
    if (!found) return k;
    while (k.cluster < kMaxCluster && n * slabs * k.cluster * 2 <= 2 * 148 && s >= (int64_t)k.cluster * 2 * down)
        if (!try_cluster(k.cluster * 2, kBlockBytes[2])) break;
    if (n * slabs > 0x7FFFFFFF / kMaxCluster) return k;
    k.pieces = pieces;
    k.slabs = (int)slabs;
    return k;
}

template <typename K>
cudaError_t launch_resident(K kernel, PerDeviceOnce& once, const ResidentArgs& a, const Keep& k, cudaStream_t st) {
    cudaError_t e = once_per_device(once, [&](int) {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kBlockBytes[2]);
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
            ResidentArgs r{a, k.cluster, k.iters, k.rows};
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
    const Layout l = layout_of(a.n, a.s, a.c, a.groups);
    if (!workspace || workspace_bytes < l.bytes || off(workspace, 16)) return MVUE_ERR_WORKSPACE;
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
