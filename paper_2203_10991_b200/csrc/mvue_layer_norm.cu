// Layer normalisation over the columns of a matrix, forward and backward.
//
// Bytes: the forward pass reads x and writes y, the backward pass reads x and dy and writes dx.  A team of threads owns rows,
// a thread eight of their columns for all of the team's rows: weight, bias and the backward pass's column sums stay in its
// registers, a row is read once and waits there for its sums.  Variances are taken about the mean, from the registers.
// Rows are taken several at a time, so that one barrier (and six shuffles instead of twenty) serves four sums: four
// rows in the forward pass, the two sums of two rows in the backward pass.
// Weight and bias gradients: a block's teams join in shared memory, blocks leave one partial sum each, and a second launch
// adds those in order: equal inputs give equal bits.
// Rows of more than 8192 columns do not fit a block's threads: they are gone over again, from L2 (wide kernels).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "../../include/mvue_layer.h"
#include "mvue_device.cuh"
#include "mvue_internal.h"
#include "mvue_train.cuh"

namespace mvue {
namespace {

constexpr int kMaxTeam = 1024;                   // threads; eight columns each
constexpr int kWideThreads = 1024;
constexpr int kColumnRows = 8;                   // wide: teams of a warp in a column block

struct Params {
    const void *x, *dy, *gamma, *beta;
    void *y, *dx;
    float *mean, *rstd;
    const float *mean_in, *rstd_in;
    float* partial;                              // [blocks][2][cols]: sums of dy xh, of dy
    int64_t rows, cols, ldx, lddy, ldy;
    float eps, inv_cols;
    int affine_bf16;
};

// Eight columns of weight or bias; `none` where there is no such tensor.
template <int kVec> __device__ __forceinline__ void load_affine(const Cols<kVec>& c, const void* from, int bf16, float none, float (&v)[8]) {
    if (!from) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = none;
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        v[j] = j >= c.count ? 0.0f : bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(from)[c.at(j)]) : static_cast<const float*>(from)[c.at(j)];
}

__device__ __forceinline__ void team_barrier(int team, int threads) {
    if (threads == 32) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(threads) : "memory");
}

// Sums of four values over a team.  Within a warp the lanes fold: after two exchanges a lane holds one of the four values for
// its four neighbours, and three more add up.  `sums`: the team's slots, four for each of its warps; not used again before another
// barrier of the team.
__device__ __forceinline__ void team_sum4(float (&v)[4], float (*sums)[4], int team, int threads, int warp, int lane) {
    const bool b0 = lane & 1, b1 = lane & 2;
    float p = (b0 ? v[2] : v[0]) + __shfl_xor_sync(0xFFFFFFFFu, b0 ? v[0] : v[2], 1);
    float q = (b0 ? v[3] : v[1]) + __shfl_xor_sync(0xFFFFFFFFu, b0 ? v[1] : v[3], 1);
    float t = (b1 ? q : p) + __shfl_xor_sync(0xFFFFFFFFu, b1 ? p : q, 2);           // value 2 (lane & 1) + (lane >> 1 & 1)
#pragma unroll
    for (int d = 4; d < 32; d <<= 1) t += __shfl_xor_sync(0xFFFFFFFFu, t, d);
    if (threads > 32) {
        if (lane < 4) sums[warp][lane] = t;
        team_barrier(team, threads);
        t = 0.0f;
        for (int w = lane >> 2; w < (threads >> 5); w += 8) t += sums[w][lane & 3];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) t += __shfl_xor_sync(0xFFFFFFFFu, t, d);
    }
    v[0] = __shfl_sync(0xFFFFFFFFu, t, 0);
    v[1] = __shfl_sync(0xFFFFFFFFu, t, 2);
    v[2] = __shfl_sync(0xFFFFFFFFu, t, 1);
    v[3] = __shfl_sync(0xFFFFFFFFu, t, 3);
}
__device__ __forceinline__ void team_sum1(float& v, float (*sums)[4], int team, int threads, int warp, int lane) {
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    if (threads > 32) {
        if (lane == 0) sums[warp][0] = v;
        team_barrier(team, threads);
        v = lane < (threads >> 5) ? sums[lane][0] : 0.0f;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    }
}

// Block: blockDim.x threads a team, blockDim.y teams.  kR rows at a time: 4, or 1 where there are few.
template <typename T, int kVec, int kR>
__global__ void __launch_bounds__(1024) forward_kernel(const __grid_constant__ Params p) {
    __shared__ float slots[2][32][4];
    grid_dependency_wait();
    const int threads = blockDim.x, team = threadIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float(*sums0)[4] = slots[0] + team * (threads >> 5);
    float(*sums1)[4] = slots[1] + team * (threads >> 5);
    const Cols<kVec> c(0, p.cols, threadIdx.x, threads);
    float gamma[8], beta[8];
    load_affine(c, p.gamma, p.affine_bf16, 1.0f, gamma);
    load_affine(c, p.beta, p.affine_bf16, 0.0f, beta);
    const T* x = static_cast<const T*>(p.x);
    T* y = static_cast<T*>(p.y);
    const bool mine = c.count > 0;
    for (int64_t row = ((int64_t)blockIdx.x * blockDim.y + team) * kR; row < p.rows; row += (int64_t)gridDim.x * blockDim.y * kR) {
        float v[kR][8], s[kR];
#pragma unroll
        for (int r = 0; r < kR; ++r) {
            if (mine && row + r < p.rows) c.load(x + (row + r) * p.ldx, v[r]);
            else {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[r][j] = 0.0f;
            }
        }
#pragma unroll
        for (int r = 0; r < kR; ++r) s[r] = ((v[r][0] + v[r][1]) + (v[r][2] + v[r][3])) + ((v[r][4] + v[r][5]) + (v[r][6] + v[r][7]));
        if constexpr (kR == 4) team_sum4(s, sums0, team, threads, warp, lane);
        else team_sum1(s[0], sums0, team, threads, warp, lane);
        float mean[kR];
#pragma unroll
        for (int r = 0; r < kR; ++r) {
            mean[r] = s[r] * p.inv_cols;
            s[r] = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[r][j] = j < c.count ? v[r][j] - mean[r] : 0.0f;
                s[r] = fmaf(v[r][j], v[r][j], s[r]);
            }
        }
        if constexpr (kR == 4) team_sum4(s, sums1, team, threads, warp, lane);
        else team_sum1(s[0], sums1, team, threads, warp, lane);
#pragma unroll
        for (int r = 0; r < kR; ++r) {
            if (row + r >= p.rows) break;
            const float rstd = rsqrtf(fmaf(s[r], p.inv_cols, p.eps));
            if (threadIdx.x == 0) {
                if (p.mean) p.mean[row + r] = mean[r];
                if (p.rstd) p.rstd[row + r] = rstd;
            }
            if (mine) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[r][j] = fmaf(v[r][j] * rstd, gamma[j], beta[j]);
                c.store(y + (row + r) * p.ldy, v[r]);
            }
        }
    }
}

// Two rows at a time.  kSums: the column sums are wanted too.
template <typename T, int kVec, bool kSums>
__global__ void __launch_bounds__(1024) backward_kernel(const __grid_constant__ Params p) {
    __shared__ float slots[2][32][4];
    extern __shared__ float joined[];                       // [2][blockDim.x * 8] where there are several teams
    grid_dependency_wait();
    const int threads = blockDim.x, team = threadIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Cols<kVec> c(0, p.cols, threadIdx.x, threads);
    float gamma[8], dgamma[8], dbeta[8];
    load_affine(c, p.gamma, p.affine_bf16, 1.0f, gamma);
#pragma unroll
    for (int j = 0; j < 8; ++j) dgamma[j] = dbeta[j] = 0.0f;
    const T *x = static_cast<const T*>(p.x), *dy = static_cast<const T*>(p.dy);
    T* dx = static_cast<T*>(p.dx);
    const bool mine = c.count > 0;
    int turn = 0;
    for (int64_t row = ((int64_t)blockIdx.x * blockDim.y + team) * 2; row < p.rows; row += (int64_t)gridDim.x * blockDim.y * 2, turn ^= 1) {
        float xh[2][8], g[2][8], s[4], rstd[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const bool there = row + r < p.rows;
            if (mine && there) {
                c.load(x + (row + r) * p.ldx, xh[r]);
                c.load(dy + (row + r) * p.lddy, g[r]);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) xh[r][j] = g[r][j] = 0.0f;
            }
            const float mean = there ? p.mean_in[row + r] : 0.0f;
            rstd[r] = there ? p.rstd_in[row + r] : 0.0f;
            s[2 * r] = s[2 * r + 1] = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                xh[r][j] = j < c.count ? (xh[r][j] - mean) * rstd[r] : 0.0f;
                if (kSums) {
                    dgamma[j] = fmaf(g[r][j], xh[r][j], dgamma[j]);
                    dbeta[j] += g[r][j];
                }
                g[r][j] *= gamma[j];
                s[2 * r] += g[r][j];
                s[2 * r + 1] = fmaf(g[r][j], xh[r][j], s[2 * r + 1]);
            }
        }
        team_sum4(s, slots[turn] + team * (threads >> 5), team, threads, warp, lane);
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            if (row + r >= p.rows || !mine) break;
            const float m0 = s[2 * r] * p.inv_cols, m1 = s[2 * r + 1] * p.inv_cols;
#pragma unroll
            for (int j = 0; j < 8; ++j) g[r][j] = rstd[r] * (g[r][j] - fmaf(xh[r][j], m1, m0));
            c.store(dx + (row + r) * p.ldy, g[r]);
        }
    }
    if constexpr (kSums) {
        float* out = p.partial + (int64_t)blockIdx.x * 2 * p.cols;
        if (blockDim.y > 1) {
            // the teams add up in order, each thread its own places
            float* at = joined + threadIdx.x * 8;
            for (int t = 0; t < (int)blockDim.y; ++t) {
                if (t == team) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        at[j] = t == 0 ? dgamma[j] : at[j] + dgamma[j];
                        at[threads * 8 + j] = t == 0 ? dbeta[j] : at[threads * 8 + j] + dbeta[j];
                    }
                }
                __syncthreads();
            }
            if (team != 0) return;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                dgamma[j] = at[j];
                dbeta[j] = at[threads * 8 + j];
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < c.count) {
                out[c.at(j)] = dgamma[j];
                out[p.cols + c.at(j)] = dbeta[j];
            }
    }
}

// The column sums of the blocks, in order.  Thirty-two columns a block, a warp every eighth partial sum.
__global__ void __launch_bounds__(256) join_kernel(const float* __restrict__ partial, int blocks, int64_t cols, float* dgamma, float* dbeta) {
    __shared__ float part[8][32];
    grid_dependency_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t i = (int64_t)blockIdx.x * 32 + lane;      // of 2 cols
    float s = 0.0f;
    if (i < 2 * cols) {
#pragma unroll 8
        for (int b = warp; b < blocks; b += 8) s += partial[(int64_t)b * 2 * cols + i];
    }
    part[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && i < 2 * cols) {
#pragma unroll
        for (int w = 1; w < 8; ++w) s += part[w][lane];
        if (i < cols) {
            if (dgamma) dgamma[i] = s;
        } else if (dbeta) {
            dbeta[i - cols] = s;
        }
    }
}

// ---- rows wider than a block ----
__device__ __forceinline__ float block_sum(float v, float* slots) {
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    const int lane = threadIdx.x & 31;
    if (lane == 0) slots[threadIdx.x >> 5] = v;
    __syncthreads();
    v = slots[lane];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    __syncthreads();
    return v;
}

template <typename T, int kVec>
__global__ void __launch_bounds__(kWideThreads) wide_forward_kernel(const __grid_constant__ Params p) {
    __shared__ float slots[32];
    grid_dependency_wait();
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(p.x) + row * p.ldx;
        T* y = static_cast<T*>(p.y) + row * p.ldy;
        float s = 0.0f, v[8];
        for (int64_t c0 = 0; c0 < p.cols; c0 += 8 * kWideThreads) {
            const Cols<kVec> c(c0, p.cols, threadIdx.x, kWideThreads);
            if (c.count == 0) break;
            c.load(x, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) s += j < c.count ? v[j] : 0.0f;
        }
        const float mean = block_sum(s, slots) * p.inv_cols;
        s = 0.0f;
        for (int64_t c0 = 0; c0 < p.cols; c0 += 8 * kWideThreads) {
            const Cols<kVec> c(c0, p.cols, threadIdx.x, kWideThreads);
            if (c.count == 0) break;
            c.load(x, v);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < c.count) s = fmaf(v[j] - mean, v[j] - mean, s);
        }
        const float rstd = rsqrtf(fmaf(block_sum(s, slots), p.inv_cols, p.eps));
        for (int64_t c0 = 0; c0 < p.cols; c0 += 8 * kWideThreads) {
            const Cols<kVec> c(c0, p.cols, threadIdx.x, kWideThreads);
            if (c.count == 0) break;
            float gamma[8], beta[8];
            c.load(x, v);
            load_affine(c, p.gamma, p.affine_bf16, 1.0f, gamma);
            load_affine(c, p.beta, p.affine_bf16, 0.0f, beta);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = fmaf((v[j] - mean) * rstd, gamma[j], beta[j]);
            c.store(y, v);
        }
        if (threadIdx.x == 0) {
            if (p.mean) p.mean[row] = mean;
            if (p.rstd) p.rstd[row] = rstd;
        }
    }
}

template <typename T, int kVec>
__global__ void __launch_bounds__(kWideThreads) wide_backward_kernel(const __grid_constant__ Params p) {
    __shared__ float slots[32];
    grid_dependency_wait();
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const T *x = static_cast<const T*>(p.x) + row * p.ldx, *dy = static_cast<const T*>(p.dy) + row * p.lddy;
        T* dx = static_cast<T*>(p.dx) + row * p.ldy;
        const float mean = p.mean_in[row], rstd = p.rstd_in[row];
        float s0 = 0.0f, s1 = 0.0f, v[8], g[8], gamma[8];
        const auto take = [&](const Cols<kVec>& c) {
            c.load(x, v);
            c.load(dy, g);
            load_affine(c, p.gamma, p.affine_bf16, 1.0f, gamma);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = j < c.count ? (v[j] - mean) * rstd : 0.0f;
                g[j] *= gamma[j];
            }
        };
        for (int64_t c0 = 0; c0 < p.cols; c0 += 8 * kWideThreads) {
            const Cols<kVec> c(c0, p.cols, threadIdx.x, kWideThreads);
            if (c.count == 0) break;
            take(c);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < c.count) {
                    s0 += g[j];
                    s1 = fmaf(g[j], v[j], s1);
                }
        }
        const float m0 = block_sum(s0, slots) * p.inv_cols, m1 = block_sum(s1, slots) * p.inv_cols;
        for (int64_t c0 = 0; c0 < p.cols; c0 += 8 * kWideThreads) {
            const Cols<kVec> c(c0, p.cols, threadIdx.x, kWideThreads);
            if (c.count == 0) break;
            take(c);
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = rstd * (g[j] - fmaf(v[j], m1, m0));
            c.store(dx, g);
        }
    }
}

// Column sums alone: a block owns 256 columns of a share of the rows (before dx is written, which may be dy).
template <typename T, int kVec>
__global__ void __launch_bounds__(32 * kColumnRows) wide_column_kernel(const __grid_constant__ Params p) {
    __shared__ float part[kColumnRows][32][17];
    grid_dependency_wait();
    const int lane = threadIdx.x, team = threadIdx.y;
    const Cols<kVec> c((int64_t)blockIdx.x * 256, min((int64_t)(blockIdx.x + 1) * 256, p.cols), lane, 32);
    float dgamma[8], dbeta[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) dgamma[j] = dbeta[j] = 0.0f;
    if (c.count > 0) {
        for (int64_t row = (int64_t)blockIdx.y * kColumnRows + team; row < p.rows; row += (int64_t)gridDim.y * kColumnRows) {
            float v[8], g[8];
            c.load(static_cast<const T*>(p.x) + row * p.ldx, v);
            c.load(static_cast<const T*>(p.dy) + row * p.lddy, g);
            const float mean = p.mean_in[row], rstd = p.rstd_in[row];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                dgamma[j] = fmaf(g[j], (v[j] - mean) * rstd, dgamma[j]);
                dbeta[j] += g[j];
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        part[team][lane][j] = dgamma[j];
        part[team][lane][8 + j] = dbeta[j];
    }
    __syncthreads();
    if (team != 0) return;
    float* out = p.partial + (int64_t)blockIdx.y * 2 * p.cols;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        for (int t = 1; t < kColumnRows; ++t) {
            dgamma[j] += part[t][lane][j];
            dbeta[j] += part[t][lane][8 + j];
        }
        if (j < c.count) {
            out[c.at(j)] = dgamma[j];
            out[p.cols + c.at(j)] = dbeta[j];
        }
    }
}

// ---- host ----
struct Plan {
    bool wide;
    int team, teams, blocks;                  // wide: blocks of rows
    int parts;                                // partial sums of the backward pass
    dim3 columns;                             // wide: grid of the column sums
};
Plan plan(int64_t rows, int64_t cols, int rows_at_once, int sm_count) {
    Plan q = {};
    q.wide = cols > 8 * kMaxTeam;
    if (q.wide) {
        q.blocks = (int)std::min<int64_t>(rows, 2 * (int64_t)sm_count);
        const int64_t slabs = (cols + 255) / 256;
        q.parts = (int)std::max<int64_t>(1, std::min<int64_t>((rows + 4 * kColumnRows - 1) / (4 * kColumnRows), 8 * (int64_t)sm_count / slabs));
        q.columns = dim3((unsigned)slabs, (unsigned)q.parts);
        return q;
    }
    q.team = (int)((cols + 255) / 256 * 32);
    q.teams = std::max(1, 256 / q.team);
    const int64_t per_block = (int64_t)q.teams * rows_at_once;
    q.blocks = (int)std::min<int64_t>((rows + per_block - 1) / per_block, (int64_t)sm_count * std::max(1, 1024 / (q.team * q.teams)));
    q.parts = q.blocks;
    return q;
}

template <typename T, int kVec> cudaError_t forward(const Plan& q, int at_once, const Params& p, cudaStream_t st) {
    if (q.wide) return launch_dependent(&wide_forward_kernel<T, kVec>, dim3(q.blocks), dim3(kWideThreads), 0, st, p);
    const dim3 block(q.team, q.teams);
    if (at_once == 4) return launch_dependent(&forward_kernel<T, kVec, 4>, dim3(q.blocks), block, 0, st, p);
    return launch_dependent(&forward_kernel<T, kVec, 1>, dim3(q.blocks), block, 0, st, p);
}
template <typename T, int kVec> cudaError_t backward(const Plan& q, bool sums, const Params& p, cudaStream_t st) {
    if (q.wide) {
        cudaError_t e = cudaSuccess;
        if (sums) e = launch_dependent(&wide_column_kernel<T, kVec>, q.columns, dim3(32, kColumnRows), 0, st, p);
        if (e != cudaSuccess) return e;
        return launch_dependent(&wide_backward_kernel<T, kVec>, dim3(q.blocks), dim3(kWideThreads), 0, st, p);
    }
    const dim3 block(q.team, q.teams);
    if (!sums) return launch_dependent(&backward_kernel<T, kVec, false>, dim3(q.blocks), block, 0, st, p);
    return launch_dependent(&backward_kernel<T, kVec, true>, dim3(q.blocks), block, q.teams > 1 ? q.team * 64 : 0, st, p);
}
int widest(int v, const void* p, int64_t ld, int64_t cols, int64_t rows, int dtype) { return std::min(v, row_vector(p, rows > 1 ? ld : cols, cols, dtype)); }

size_t workspace_bytes_of(int64_t rows, int64_t cols, int sm_count) { return (size_t)plan(rows, cols, 2, sm_count).parts * 2 * (size_t)cols * sizeof(float); }

int check(const void* x, int dtype, int64_t rows, int64_t cols, int affine_dtype, const void* gamma, const void* beta) {
    if (dtype != MVUE_F32 && dtype != MVUE_BF16) return MVUE_ERR_DTYPE;
    if (affine_dtype != MVUE_F32 && affine_dtype != MVUE_BF16) return MVUE_ERR_DTYPE;
    if (rows < 0 || cols < 1 || cols > 0x7FFFFFFF || rows > 0x7FFFFFFFFFll) return MVUE_ERR_SHAPE;
    if (rows > 0 && !x) return MVUE_ERR_NULL;
    if (off(x, size_of(dtype)) || off(gamma, size_of(affine_dtype)) || off(beta, size_of(affine_dtype))) return MVUE_ERR_ALIGN;
    return MVUE_OK;
}

}  // namespace
}  // namespace mvue

using namespace mvue;

extern "C" int mvue_layer_norm(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx, const void* gamma, const void* beta,
                               int affine_dtype, float eps, void* y, int64_t ldy, float* mean, float* rstd, void* stream) {
    if (int s = check(x, dtype, rows, cols, affine_dtype, gamma, beta)) return s;
    if (ldx < cols || ldy < cols) return MVUE_ERR_SHAPE;
    if (rows > 0 && !y) return MVUE_ERR_NULL;
    if (off(y, size_of(dtype)) || off(mean, 4) || off(rstd, 4)) return MVUE_ERR_ALIGN;
    if (rows == 0) return MVUE_OK;
    DeviceInfo dev;
    if (int s = current_device_info(&dev)) return s;
    Params p = {};
    p.x = x; p.y = y; p.gamma = gamma; p.beta = beta; p.mean = mean; p.rstd = rstd;
    p.rows = rows; p.cols = cols; p.ldx = ldx; p.ldy = ldy;
    p.eps = eps; p.inv_cols = (float)(1.0 / (double)cols); p.affine_bf16 = affine_dtype == MVUE_BF16;
    // four rows at a time where that leaves every SM a block's worth of them
    Plan q = plan(rows, cols, 4, dev.sm_count);
    const int at_once = q.wide || q.blocks >= dev.sm_count ? 4 : 1;
    if (at_once == 1) q = plan(rows, cols, 1, dev.sm_count);
    const int v = widest(widest(8, x, ldx, cols, rows, dtype), y, ldy, cols, rows, dtype);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const auto pick = [&](auto t) {
        using T = decltype(t);
        return v == 8 ? forward<T, 8>(q, at_once, p, st) : v == 2 ? forward<T, 2>(q, at_once, p, st) : forward<T, 1>(q, at_once, p, st);
    };
    const cudaError_t e = dtype == MVUE_BF16 ? pick(__nv_bfloat16()) : pick(float());
    if (e != cudaSuccess) { set_cuda_error(e, "mvue_layer_norm launch"); return MVUE_ERR_CUDA; }
    return MVUE_OK;
}

extern "C" int mvue_layer_norm_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, int dtype, int64_t rows, int64_t cols,
                                        const float* mean, const float* rstd, const void* gamma, int affine_dtype, void* dx, int64_t lddx,
                                        float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes, void* stream) {
    if (int s = check(x, dtype, rows, cols, affine_dtype, gamma, nullptr)) return s;
    if (ldx < cols || lddy < cols || lddx < cols) return MVUE_ERR_SHAPE;
    if (rows > 0 && (!dy || !dx || !mean || !rstd)) return MVUE_ERR_NULL;
    if (off(dy, size_of(dtype)) || off(dx, size_of(dtype)) || off(mean, 4) || off(rstd, 4) || off(dgamma, 4) || off(dbeta, 4)) return MVUE_ERR_ALIGN;
    DeviceInfo dev;
    if (int s = current_device_info(&dev)) return s;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const bool sums = dgamma || dbeta;
    if (rows == 0) {
        cudaError_t e = dgamma ? cudaMemsetAsync(dgamma, 0, cols * sizeof(float), st) : cudaSuccess;
        if (e == cudaSuccess && dbeta) e = cudaMemsetAsync(dbeta, 0, cols * sizeof(float), st);
        if (e != cudaSuccess) { set_cuda_error(e, "mvue_layer_norm_backward"); return MVUE_ERR_CUDA; }
        return MVUE_OK;
    }
    if (sums && (!workspace || off(workspace, 16) || workspace_bytes < workspace_bytes_of(rows, cols, dev.sm_count))) return MVUE_ERR_WORKSPACE;
    Params p = {};
    p.x = x; p.dy = dy; p.dx = dx; p.gamma = gamma; p.mean_in = mean; p.rstd_in = rstd; p.partial = static_cast<float*>(workspace);
    p.rows = rows; p.cols = cols; p.ldx = ldx; p.lddy = lddy; p.ldy = lddx;
    p.inv_cols = (float)(1.0 / (double)cols); p.affine_bf16 = affine_dtype == MVUE_BF16;
    const Plan q = plan(rows, cols, 2, dev.sm_count);
    const int v = widest(widest(widest(8, x, ldx, cols, rows, dtype), dy, lddy, cols, rows, dtype), dx, lddx, cols, rows, dtype);
    const auto pick = [&](auto t) {
        using T = decltype(t);
        return v == 8 ? backward<T, 8>(q, sums, p, st) : v == 2 ? backward<T, 2>(q, sums, p, st) : backward<T, 1>(q, sums, p, st);
    };
    cudaError_t e = dtype == MVUE_BF16 ? pick(__nv_bfloat16()) : pick(float());
    if (e == cudaSuccess && sums)
        e = launch_dependent(&join_kernel, dim3((unsigned)((2 * cols + 31) / 32)), dim3(256), 0, st, p.partial, q.parts, cols, dgamma, dbeta);
    if (e != cudaSuccess) { set_cuda_error(e, "mvue_layer_norm_backward launch"); return MVUE_ERR_CUDA; }
    return MVUE_OK;
}

extern "C" int mvue_layer_norm_workspace_bytes(int64_t rows, int64_t cols, size_t* bytes) {
    if (!bytes) return MVUE_ERR_NULL;
    if (rows < 0 || cols < 1 || cols > 0x7FFFFFFF || rows > 0x7FFFFFFFFFll) return MVUE_ERR_SHAPE;
    DeviceInfo dev;
    if (int s = current_device_info(&dev)) return s;
    *bytes = rows == 0 ? 0 : workspace_bytes_of(rows, cols, dev.sm_count);
    return MVUE_OK;
}
