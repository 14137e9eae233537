// The Muon step: momentum, the update's orthogonalisation by Newton-Schulz products, the param.
//
// With X the update over its norm, transposed where it has more rows than columns ([m x n], m <= n), a step of the iteration is
//   A = X X^T;  B = a I + b A + c A A;  X' = B X
// Products are binary16 on the tensor cores with fp32 accumulators: binary16 and not bf16, since the polynomial's slope of a = 3.4
// at zero multiplies what a rounding adds to small singular values by up to 485 in five steps (an update of sixteen large
// directions and noise a tenth as strong comes out 9 % off with bf16, 1 % with binary16).  The same update is 0.1 % off if, in all
// steps but the last two, a second binary16 beside the first (x = hi + lo 2^-11) adds a lo to B hi: what the roundings of B do lies in
// few directions, what that of X does in all.
// a I in binary16 with the rest of B, and not a X added in binary32, costs digits where a few directions dominate and gains some on noise (the two
// roundings, five steps in 64 bits, 512 x 1024: one direction and 0.01 noise 5.3e-4 -> 7.3e-4, m/16 directions and 0.1 noise 1.3e-3 -> 1.5e-3, noise
// 1.36e-3 -> 1.28e-3); the product then reads half as much or nothing beside its operands (24 of 1024 x 4096 orthogonalised 2.28 -> 2.07 ms).
// A and B are symmetric: only tiles on and above the diagonal are computed, and stored twice.
// X is stored times xs, A and B times S, powers of two near the root of n, so that entries of 1 / sqrt(n) stay normal numbers; xs is larger for
// an update far below eps.  The norm counts every update that binary32 can hold: an update of 5e-24 whose squares all came out as zero had X scaled
// as if it were nothing, and grew beyond binary16.
//
// Matrices of equal extents go through the products together.
//
// 24 of 4096 x 1024, binary32 gradients, bf16 params rounded at random, five steps: 2.3 ms, 2.5 ms in a long run under the power limit.
// Momentum 0.19, start 0.20 and param 0.17 ms run at 3.7 (param: the random numbers, and a matrix that is turned over) to 6.2 TB/s.
// The products' 1.7 TFLOP take 1.7 ms: B X 0.17 to 0.21 ms a step (1.0 to 1.2 PFLOP/s; a library product sustains 1.4), X X^T 0.12 ms, of
// which a fifth is what 240 tiles leave of four rounds of 74 pairs, B 0.04 ms, where 16 steps of 64 are too short for a tile's epilogue.
// 256 x 256: 64 us, fifteen dependent products in one launch, 4 us each, of which the tensor cores have work for a tenth.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/mvue_layer.h"
#include "mvue_dense.cuh"
#include "mvue_few.cuh"
#include "mvue_train.cuh"

namespace mvue {
namespace {

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr double kEps = 1e-7;
constexpr int kBatch = 64;                          // matrices that go together
constexpr int64_t kBatchElements = 1 << 27;         // unless they have more elements than this
constexpr int kMaxParts = 128;                      // blocks that share a matrix's norm
constexpr int kThreads = 256, kTile = 64;
constexpr float kLo = 2048.0f;                      // 2^11: lo holds what hi lost, times this
constexpr float kSquaresFrom = 7.88860905e-31f;     // 2^-100: what eight squares lose below 2^-149 is nothing beside such a sum

enum : uint32_t { kTransposed = 1, kGradBf16 = 2, kParamBf16 = 4, kWideIn = 8, kWideOut = 16 };

struct Matrix {
    const void* grad;
    float* momentum;            // NULL: orthogonalise grad itself
    void* param;                // or the output
    float* master;
    int64_t first_block;        // the call's 256-element blocks before this matrix
    uint32_t flags, pad;
};

struct Group {
    int count, m, n;            // m <= n
    int64_t ld_grad, ld_param;  // of a matrix as the caller holds it; momentum and master lie as the param does
    // workspace
    __half *hi, *lo;            // [count][m][n_pitch]
    int64_t n_pitch;
    double* parts;              // [count][n_parts]
    int n_parts;
    float* xs;                  // [count]
    float S, growth;            // growth: 3.4445^steps
    // the step
    float mu, one_mu, grad_scale, decay, size;      // size: lr times the scale of the update
    const float* dev_grad_scale;
    int nesterov, random;
    RoundKeys keys;
    Matrix matrix[kBatch];

    __device__ __forceinline__ int rows(const Matrix& t) const { return t.flags & kTransposed ? n : m; }
    __device__ __forceinline__ int cols(const Matrix& t) const { return t.flags & kTransposed ? m : n; }
    __device__ __forceinline__ float scale() const { return dev_grad_scale ? __fmul_rn(grad_scale, *dev_grad_scale) : grad_scale; }
};

__device__ __forceinline__ void load_grad(const Matrix& t, int64_t at, bool wide, int count, float gs, float (&g)[8]) {
    if (t.flags & kGradBf16) load8(static_cast<const __nv_bfloat16*>(t.grad) + at, wide, count, g);
    else load8(static_cast<const float*>(t.grad) + at, wide, count, g);
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] *= gs;
}

// The new momentum, and a share of the squared norm of the update.  Grid: n_parts x count.
__global__ void __launch_bounds__(kThreads) momentum_kernel(const __grid_constant__ Group q) {
    __shared__ double warps[kThreads / 32];
    grid_dependency_wait();
    const Matrix& t = q.matrix[blockIdx.y];
    const float gs = q.scale();
    const int cols = q.cols(t);
    // rows without gaps are one long row
    const bool dense = q.ld_grad == cols;
    const int64_t len = dense ? (int64_t)q.m * q.n : cols, pieces = (len + 8 * kThreads - 1) / (8 * kThreads), rows = dense ? 1 : q.rows(t);
    double sum = 0.0;
    for (int64_t w = blockIdx.x; w < rows * pieces; w += gridDim.x) {
        const int64_t row = w / pieces, i0 = (w - row * pieces) * 8 * kThreads + threadIdx.x * 8;
        const int count = (int)min((int64_t)8, len - i0);
        if (count <= 0) continue;
        const bool wide = (t.flags & kWideIn) && count == 8;
        float g[8], u[8];
        load_grad(t, row * q.ld_grad + i0, wide, count, gs, g);
        if (t.momentum) {
            load8(t.momentum + row * q.ld_param + i0, wide, count, u);
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i] = fmaf(q.mu, u[i], q.one_mu * g[i]);
            store8(t.momentum + row * q.ld_param + i0, wide, count, u);
            if (q.nesterov) {
#pragma unroll
                for (int i = 0; i < 8; ++i) u[i] = fmaf(q.mu, u[i], q.one_mu * g[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i] = g[i];
        }
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s = fmaf(u[i], u[i], s);
        if (s >= kSquaresFrom && s <= 3.402823466e38f) {
            sum += (double)s;
        } else {                                   // squares that binary32 loses or has no room for, and what is not finite
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += (double)u[i] * (double)u[i];
        }
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
    if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kThreads / 32; ++w) sum += warps[w];
        q.parts[(int64_t)blockIdx.y * q.n_parts + blockIdx.x] = sum;
    }
}

// hi and lo of eight values.
__device__ __forceinline__ void split8(const float (&x)[8], uint4* hi, uint4* lo) {
    uint32_t h[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 a = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
        const float2 f = __half22float2(a);
        const __half2 b = __floats2half2_rn((x[2 * i] - f.x) * kLo, (x[2 * i + 1] - f.y) * kLo);
        h[i] = *reinterpret_cast<const uint32_t*>(&a);
        l[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    *hi = make_uint4(h[0], h[1], h[2], h[3]);
    *lo = make_uint4(l[0], l[1], l[2], l[3]);
}

// X = update / (norm + eps) in tiles of 64 x 64 of the caller's matrix, which is turned over where it has more rows than columns.
// Eight neighbours a thread; n_pitch is a multiple of eight, so what is written in X's rows is whole pieces of it.
__global__ void __launch_bounds__(kThreads) start_kernel(const __grid_constant__ Group q) {
    __shared__ float tile[kTile][kTile + 1];
    __shared__ float factor[2];
    grid_dependency_wait();
    const int z = blockIdx.y;
    const Matrix& t = q.matrix[z];
    const int rows = q.rows(t), cols = q.cols(t);
    if (threadIdx.x < 32) {                        // every block adds the shares in the same order
        double s = 0.0;
        for (int i = threadIdx.x; i < q.n_parts; i += 32) s += q.parts[(int64_t)z * q.n_parts + i];
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
        if (threadIdx.x == 0) {
            const double norm = sqrt(s);
            // xs: S, or more where even the last X stays below one (eps outweighs the update): S 2^k, k at most 100, which brings the last X's
            // norm to 2^13 or above, so that the first, smaller by 3.4445^steps, is not lost
            const float last = fminf((float)(norm / (norm + kEps)) * q.growth, 1.25f);
            const float xs = last < 1.25f ? q.S * exp2f(fminf(floorf(log2f(16384.0f / (q.S * fmaxf(last, 1e-37f)))), 100.0f)) : q.S;
            // xs / (norm + eps) in two factors near its root, the first a power of two: the whole is beyond binary32 for the least updates and
            // subnormal for the largest
            const double whole = (double)xs / (norm + kEps);
            const int e = isfinite(norm) ? ((__double2hiint(whole) >> 20) - 1023) / 2 : 0;       // (whole is a normal number from 2^-148 to 2^134)
            factor[0] = __int_as_float((127 + e) << 23);
            factor[1] = isfinite(norm) ? (float)(whole * (double)__int_as_float((127 - e) << 23)) : __uint_as_float(0x7FFFFFFFu);
            if (blockIdx.x == 0) q.xs[z] = xs;
        }
    }
    __syncthreads();
    const float gs = q.scale(), f0 = factor[0], f1 = factor[1];
    const int tiles_x = (cols + kTile - 1) / kTile, tiles = tiles_x * ((rows + kTile - 1) / kTile);
    __half *hi = q.hi + (int64_t)z * q.m * q.n_pitch, *lo = q.lo + (int64_t)z * q.m * q.n_pitch;
    for (int w = blockIdx.x; w < tiles; w += gridDim.x) {
        const int row0 = w / tiles_x * kTile, col0 = w % tiles_x * kTile;
        const int c = (threadIdx.x & 7) * 8;
#pragma unroll
        for (int it = 0; it < 2; ++it) {
            const int r = (threadIdx.x >> 3) + 32 * it, row = row0 + r, col = col0 + c;
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = 0.0f;
            const int count = row < rows ? max(0, min(8, cols - col)) : 0;
            if (count > 0) {
                const bool wide = (t.flags & kWideIn) && count == 8;
                load_grad(t, (int64_t)row * q.ld_grad + col, wide, count, gs, x);
                if (t.momentum) {
                    float u[8];
                    load8(t.momentum + (int64_t)row * q.ld_param + col, wide, count, u);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = q.nesterov ? fmaf(q.mu, u[i], q.one_mu * x[i]) : u[i];
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = x[i] * f0 * f1;
            }
            if (t.flags & kTransposed) {
#pragma unroll
                for (int i = 0; i < 8; ++i) tile[r][c + i] = x[i];
            } else if (count > 0) {
                const int64_t at = (int64_t)row * q.n_pitch + col;
                split8(x, reinterpret_cast<uint4*>(hi + at), reinterpret_cast<uint4*>(lo + at));
            }
        }
        if (t.flags & kTransposed) {
            __syncthreads();
#pragma unroll
            for (int it = 0; it < 2; ++it) {
                const int r = (threadIdx.x >> 3) + 32 * it, row = col0 + r, col = row0 + c;       // of X
                if (row < q.m && col < q.n) {
                    float x[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = tile[c + i][r];
                    const int64_t at = (int64_t)row * q.n_pitch + col;
                    split8(x, reinterpret_cast<uint4*>(hi + at), reinterpret_cast<uint4*>(lo + at));
                }
            }
            __syncthreads();
        }
    }
}

// What comes of the last X (hi / xs): the output, or the param's step.  Tiles as above.  What a thread reads of a tile is on its way at
// once: of 24 matrices of 4096 x 1024 bf16 params, rounded at random, 165 us (222 us with each piece loaded before it is used).
enum { kOutput, kBf16Param, kFloatParam };
template <int kKind, bool kTurn>
__device__ __forceinline__ void finish_tiles(const Group& q, const Matrix& t, int z, float (*tile)[kTile + 1]) {
    constexpr int kWords = kKind == kOutput ? 1 : kKind == kBf16Param ? 4 : 8;
    const int rows = q.rows(t), cols = q.cols(t);
    const float inv = 1.0f / q.xs[z];
    const int tiles_x = (cols + kTile - 1) / kTile, tiles = tiles_x * ((rows + kTile - 1) / kTile);
    const __half* hi = q.hi + (int64_t)z * q.m * q.n_pitch;
    const float* from32 = t.master ? t.master : static_cast<const float*>(t.param);
    const __nv_bfloat16* from16 = static_cast<const __nv_bfloat16*>(t.param);
    const bool rounds = kKind == kBf16Param && q.random;
    const int c = (threadIdx.x & 7) * 8;
    for (int w = blockIdx.x; w < tiles; w += gridDim.x) {
        const int row0 = w / tiles_x * kTile, col0 = w % tiles_x * kTile;
        uint4 v[2];
        uint32_t held[2][kWords];
        int count[2];
        bool wide[2];
#pragma unroll
        for (int it = 0; it < 2; ++it) {
            const int r = (threadIdx.x >> 3) + 32 * it, row = row0 + r, col = col0 + c;
            count[it] = row < rows ? max(0, min(8, cols - col)) : 0;
            wide[it] = (t.flags & kWideOut) && count[it] == 8;
            const int x_row = kTurn ? col0 + r : row, x_col = kTurn ? row0 + c : col;
            v[it] = make_uint4(0u, 0u, 0u, 0u);
            if (x_row < q.m && x_col < q.n) v[it] = *reinterpret_cast<const uint4*>(hi + (int64_t)x_row * q.n_pitch + x_col);
            if (kKind != kOutput && wide[it]) {
                const int64_t at = (int64_t)row * q.ld_param + col;
                if constexpr (kKind == kBf16Param) {
                    const uint4 p = *reinterpret_cast<const uint4*>(from16 + at);
                    held[it][0] = p.x; held[it][1] = p.y; held[it][2] = p.z; held[it][3] = p.w;
                } else if constexpr (kKind == kFloatParam) {
                    ld256(from32 + at, held[it]);
                }
            }
        }
        float x[2][8];
#pragma unroll
        for (int it = 0; it < 2; ++it) {
            const uint32_t words[4] = {v[it].x, v[it].y, v[it].z, v[it].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&words[i]));
                x[it][2 * i] = f.x * inv;
                x[it][2 * i + 1] = f.y * inv;
            }
        }
        if (kTurn) {
            const int r = threadIdx.x >> 3;
            __syncthreads();                       // the last tile has been read
#pragma unroll
            for (int it = 0; it < 2; ++it)
#pragma unroll
                for (int i = 0; i < 8; ++i) tile[c + i][r + 32 * it] = x[it][i];
            __syncthreads();
#pragma unroll
            for (int it = 0; it < 2; ++it)
#pragma unroll
                for (int i = 0; i < 8; ++i) x[it][i] = tile[r + 32 * it][c + i];
        }
#pragma unroll
        for (int it = 0; it < 2; ++it) {
            if (count[it] == 0) continue;
            const int64_t at = (int64_t)(row0 + (threadIdx.x >> 3) + 32 * it) * q.ld_param + col0 + c;
            uint32_t random[4];
            if constexpr (kKind != kOutput) {
                float p[8];
                if (wide[it]) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        p[i] = kKind == kFloatParam ? __uint_as_float(held[it][i]) : i & 1 ? bf16_hi(held[it][i / 2]) : bf16_lo(held[it][i / 2]);
                } else if constexpr (kKind == kBf16Param) {
                    load8(from16 + at, false, count[it], p);
                } else {
                    load8(from32 + at, false, count[it], p);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) x[it][i] = fmaf(p[i], q.decay, -q.size * x[it][i]);
                if (t.master) store8(t.master + at, wide[it], count[it], x[it]);
                if (rounds) {
                    // elements 8u .. 8u + 7 of the padded list share a call; a piece that starts inside one takes two
                    const uint64_t first = (uint64_t)t.first_block * 256u + (uint64_t)at;
                    const int shift = (int)(first & 7u);
                    const uint4 a = philox4x32_10(first >> 3, q.keys, 2u);
                    random[0] = a.x; random[1] = a.y; random[2] = a.z; random[3] = a.w;
                    if (shift) {
                        const uint4 b = philox4x32_10((first >> 3) + 1u, q.keys, 2u);
                        const uint32_t words[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
#pragma unroll
                            for (int s = 1; s < 8; ++s)
                                if (s == shift)
                                    random[i] = s & 1 ? words[i + s / 2] >> 16 | words[i + s / 2 + 1] << 16 : words[i + s / 2];
                        }
                    }
                }
            }
            if (t.flags & kParamBf16) {
                uint32_t o[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (rounds) {
                        // (a NaN whose lower half is zero: random bits do not carry into its sign)
                        const float lo = x[it][2 * i] == x[it][2 * i] ? x[it][2 * i] : __uint_as_float(0x7FC00000u);
                        const float hi2 = x[it][2 * i + 1] == x[it][2 * i + 1] ? x[it][2 * i + 1] : __uint_as_float(0x7FC00000u);
                        o[i] = pack_out<true>(lo, hi2, random[i]);
                    } else {
                        o[i] = pack_bf16x2(x[it][2 * i], x[it][2 * i + 1]);
                    }
                }
                store8_words(static_cast<__nv_bfloat16*>(t.param) + at, wide[it], count[it], o);
            } else {
                store8(static_cast<float*>(t.param) + at, wide[it], count[it], x[it]);
            }
        }
    }
}
__global__ void __launch_bounds__(kThreads, 4) finish_kernel(const __grid_constant__ Group q) {
    __shared__ float tile[kTile][kTile + 1];
    grid_dependency_wait();
    const int z = blockIdx.y;
    const Matrix& t = q.matrix[z];
    const bool turn = t.flags & kTransposed;
    if (!t.momentum) turn ? finish_tiles<kOutput, true>(q, t, z, tile) : finish_tiles<kOutput, false>(q, t, z, tile);
    else if ((t.flags & kParamBf16) && !t.master) turn ? finish_tiles<kBf16Param, true>(q, t, z, tile) : finish_tiles<kBf16Param, false>(q, t, z, tile);
    else turn ? finish_tiles<kFloatParam, true>(q, t, z, tile) : finish_tiles<kFloatParam, false>(q, t, z, tile);
}

// ---- epilogues of the products -----------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t half_pair(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 halves(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
// A S = acc S / xs^2 (kPoly false; kAdd: added to what there is of a long sum), B S = a S on the diagonal + b (A S) + c acc / S (true); symmetric,
// the tile's mirror image is stored too.  diag: the column of these 32 that is the row's own, or -1.
template <bool kPoly, bool kAdd = false>
struct Symmetric {
    using Maps = dense::SlabMaps;
    static constexpr bool kSlabs = true, kMirror = true;
    static constexpr int kIn = kPoly || kAdd ? 1 : 0;
    const float* xs;
    float S;
    __device__ __forceinline__ bool two_out() const { return true; }
    __device__ __forceinline__ float values(int z) const { return kPoly ? kC / S : S / xs[z] / xs[z]; }
    __device__ __forceinline__ void compute(float alpha, const uint32_t (&v)[32], uint4 (&x)[2][4], int diag) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t w[4] = {x[0][i].x, x[0][i].y, x[0][i].z, x[0][i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float lo = __uint_as_float(v[8 * i + 2 * j]) * alpha, hi = __uint_as_float(v[8 * i + 2 * j + 1]) * alpha;
                if (kPoly) {
                    const float2 a = halves(w[j]);
                    lo = fmaf(kB, a.x, lo);
                    hi = fmaf(kB, a.y, hi);
                    if (diag >= 0) {                         // (a whole warp)
                        if (8 * i + 2 * j == diag) lo = fmaf(kA, S, lo);
                        if (8 * i + 2 * j + 1 == diag) hi = fmaf(kA, S, hi);
                    }
                }
                if (kAdd) {
                    const float2 a = halves(w[j]);
                    lo += a.x;
                    hi += a.y;
                }
                w[j] = half_pair(lo, hi);
            }
            x[0][i] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
};

// X' xs = acc / S, and with kWithLo a times the second half of X, which comes in x[0].
template <bool kWithLo>
struct Apply {
    using Maps = dense::SlabMaps;
    static constexpr bool kSlabs = true, kMirror = false;
    static constexpr int kIn = kWithLo ? 1 : 0;
    float inv_S;
    int write_lo;
    __device__ __forceinline__ bool two_out() const { return kWithLo && write_lo; }
    __device__ __forceinline__ float values(int) const { return inv_S; }
    __device__ __forceinline__ void compute(float scale, const uint32_t (&v)[32], uint4 (&x)[2][4], int) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t h[4], l[4] = {};
            if (kWithLo) { l[0] = x[0][i].x; l[1] = x[0][i].y; l[2] = x[0][i].z; l[3] = x[0][i].w; }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float a = __uint_as_float(v[8 * i + 2 * j]) * scale, b = __uint_as_float(v[8 * i + 2 * j + 1]) * scale;
                if (kWithLo) {
                    const float2 y = halves(l[j]);
                    a = fmaf(kA / kLo, y.x, a);
                    b = fmaf(kA / kLo, y.y, b);
                }
                h[j] = half_pair(a, b);
                if (kWithLo) {
                    const float2 r = halves(h[j]);
                    l[j] = half_pair((a - r.x) * kLo, (b - r.y) * kLo);
                }
            }
            x[0][i] = make_uint4(h[0], h[1], h[2], h[3]);
            if (kWithLo) x[1][i] = make_uint4(l[0], l[1], l[2], l[3]);
        }
    }
};

// ---- small matrices --------------------------------------------------------------------------------------------------------
// Tiles of 128 x 64, one thread block each; operands by TMA from L2, where the last product's results are.
// kCluster: a cluster of eight blocks per matrix goes through all products with a cluster barrier between them instead of a launch
// (fifteen dependent launches of a product that takes two microseconds cost nine each).  Else one product a launch, a block per tile:
// for matrices that pair tiles would leave most SMs without.
//   warps 0-3 epilogue      warp 4 TMA producer      warp 5 tensor-memory allocation, MMA issue
// A block has eight stages and an SM to itself where the blocks leave room for that, else four.
constexpr int kSmallBlocks = 8, kSmallThreads = 192;
constexpr int kSmallBox = 64 * 128, kSmallStage = 3 * kSmallBox;        // 128 rows of the first operand, 64 of the second
constexpr int small_smem(int stages) { return stages * kSmallStage + 256 + 1024; }
// What a cluster takes: up to 256 x 512 (256 x 256: 64 us, a launch a product 73 us; 24 of 256 x 512 117 us, 137 us), twice as long where
// there are few rows or many matrices (24 of 256 x 1024: 178 us, 193 us; one 112 us, 90 us).
constexpr int kSmallM = 256, kSmallN = 1024;
// One product a launch, in tiles of 128 x 64, while a product has no more than this many tiles of 256 x 256 in all matrices.
// B X: 512 x 512 94 us (pair tiles 165 us), 1024 x 1024 133 us (200 us).  X X^T and A A, of which pair tiles cover the upper half alone:
// 1024 x 4096, 10 tiles, 240 us (286 us), two of 321 x 3274 181 us (222 us), 12 of 308 x 2389, 36 tiles, 343 us (332 us).
// Up to 256 rows four times as many (14 of 197 x 3708 281 us, 318 us, but all in small tiles 373 us), and up to 128, where half of a pair
// tile would be empty, any number (24 of 128 x 4096 296 us, 353 us; 24 of 64 x 4096 200 us, 318 us).
constexpr int64_t kSmallPairTiles = 40, kSmallSquareTiles = 24;
// Terms that an accumulator adds up: what an addition has below the sum's last place is cut off, always downwards, so A shrinks with their
// number.  2 x n, five steps, at the worst of some: 1.5e-3 off at 2^15 terms, 1.8e-3 at 2^17, 6.3e-3 at 2^18, 2.3e-2 at 2^20, 1.2e-1 at 2^23.  X X^T of longer
// rows is split over a cluster, or in pair tiles summed up by several launches (A is rounded to binary16 in between).
constexpr int64_t kSumTerms = 1 << 17, kMostTerms = 8 * kSumTerms;

struct SmallParams {
    int m, n, steps;
    int blocks, first, last;                 // blocks (tiles, where the sum is split) of a matrix; phases (three a step)
    int split;                               // !kCluster, A = X X^T: blocks of a cluster that share the sum of a tile
    int64_t n_pitch, m_pitch;
    __half *X[2], *lo, *A, *B;
    float* xs;                               // [matrices]; NaN where a wait ran out, which finish_kernel hands on to the results
    float S;
    int* dev_status;
};
struct SmallMaps {
    CUtensorMap X[2], A, B;                  // boxes of 64 x 64
};

__device__ __forceinline__ void mma_half(uint32_t d, uint64_t a, uint64_t b, uint32_t instr, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(instr), "r"(accumulate) : "memory");
}
// 32 halves of a row from global memory; pieces of eight that do not begin before `left` are zero, or not written
__device__ __forceinline__ void load_row(const __half* from, int left, uint4 (&w)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = 8 * i < left ? *reinterpret_cast<const uint4*>(from + 8 * i) : make_uint4(0u, 0u, 0u, 0u);
}
__device__ __forceinline__ void store_row(__half* to, int left, const uint4 (&w)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (8 * i < left) *reinterpret_cast<uint4*>(to + 8 * i) = w[i];
}

template <int kSmallStages, bool kCluster>
__global__ void __launch_bounds__(kSmallThreads, kSmallStages == 4 ? 2 : 1)
small_kernel(const __grid_constant__ SmallMaps maps, const __grid_constant__ SmallParams p) {
    extern __shared__ uint8_t smem_raw[];
    constexpr int kSmallBars = kSmallStages * kSmallStage;
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem_gen = smem_raw + (smem_base - smem_u32(smem_raw));
    const uint32_t bar_base = smem_base + kSmallBars;
    const auto full_bar = [&](int s) { return bar_base + 8u * s; };
    const auto empty_bar = [&](int s) { return bar_base + 8u * (kSmallStages + s); };
    const auto acc_bar = [&](int b) { return bar_base + 8u * (2 * kSmallStages + b); };
    const auto free_bar = [&](int b) { return bar_base + 8u * (2 * kSmallStages + 2 + b); };
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem_gen + kSmallBars + 8 * (2 * kSmallStages + 4));
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, unit = blockIdx.x / p.split;
    const int part = blockIdx.x - unit * p.split, z = unit / p.blocks, rank = unit - z * p.blocks;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kSmallStages; ++s) {
            mbar_init(full_bar(s), 1);
            mbar_init(empty_bar(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(acc_bar(b), 1);
            mbar_init(free_bar(b), 4);
        }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 5) {
        tmem_alloc(smem_u32(tmem_slot), 128);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    grid_launch_dependents();
    grid_dependency_wait();

    const int64_t x0 = (int64_t)z * p.m * p.n_pitch, a0 = (int64_t)z * p.m * p.m_pitch;
    const float xs = p.xs[z];
    int s = 0, done = 0;                                     // stage, tiles of this block so far: each role counts for itself
    uint32_t parity = warp == 4 ? 1u : 0u;
    for (int phase = p.first; phase < p.last; ++phase) {
        const int k = phase / 3, what = phase - 3 * k;       // 0: A = X X^T, 1: B = a I + b A + c A A, 2: X' = B X
        const int N = what == 2 ? p.n : p.m, K = what == 0 ? p.n : p.m;
        const int tiles_n = (N + 63) / 64, tiles = (p.m + 127) / 128 * tiles_n;
        // this block's share of the sum
        const int all = (K + 63) / 64, share = (all + p.split - 1) / p.split, begin = part * share, steps = max(0, min(all - begin, share));
        if (warp == 4 && lane == 0) {
            asm volatile("fence.proxy.async.global;" ::: "memory");
            const CUtensorMap* first = what == 0 ? &maps.X[k & 1] : what == 1 ? &maps.A : &maps.B;
            const CUtensorMap* second = what == 1 ? &maps.A : &maps.X[k & 1];
            bool ok = true;
            for (int t = rank; t < tiles && ok; t += p.blocks) {
                const int m0 = t / tiles_n * 128, n0 = t % tiles_n * 64;
                for (int i = 0; i < steps; ++i) {
                    if (!(ok = mbar_wait(empty_bar(s), parity, abort_flag))) break;
                    const uint32_t to = smem_base + s * kSmallStage;
                    mbar_expect_tx(full_bar(s), kSmallStage);
                    const int at = 64 * (begin + i);
                    dense::tma_load_3d(to, first, at, m0, z, full_bar(s));
                    dense::tma_load_3d(to + kSmallBox, first, at, m0 + 64, z, full_bar(s));
                    dense::tma_load_3d(to + 2 * kSmallBox, second, what == 2 ? n0 : at, what == 2 ? at : n0, z, full_bar(s));
                    if (++s == kSmallStages) { s = 0; parity ^= 1u; }
                }
            }
        } else if (warp == 5 && lane == 0) {
            const uint32_t instr = (1u << 4) | (what == 2 ? 1u << 16 : 0u) | (64u >> 3 << 17) | (128u >> 4 << 24);
            const uint64_t da = make_smem_desc(smem_base, 16, 1024, kSwizzle128B), db = make_smem_desc(smem_base + 2 * kSmallBox, kSmallBox, 1024, kSwizzle128B);
            const int b_step = what == 2 ? 16 * 128 / 16 : 2;
            bool ok = true;
            for (int t = rank; t < tiles && ok; t += p.blocks, ++done) {
                if (done > 1) {
                    if (!(ok = mbar_wait(free_bar(done & 1), ((done >> 1) - 1) & 1u, abort_flag))) break;
                    tc_fence_after();
                }
                for (int i = 0; i < steps; ++i) {
                    if (!(ok = mbar_wait(full_bar(s), parity, abort_flag))) break;
                    tc_fence_after();
                    const uint64_t stage = (uint64_t)(s * (kSmallStage >> 4));
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        mma_half(tmem_base + 64u * (done & 1), da + stage + 2 * j, db + stage + j * b_step, instr, (i > 0 || j > 0) ? 1u : 0u);
                    tc_commit(empty_bar(s));
                    if (++s == kSmallStages) { s = 0; parity ^= 1u; }
                }
                if (!ok) break;
                tc_commit(acc_bar(done & 1));                // (a share of nothing: at once)
            }
        } else if (warp < 4) {
            const bool read_lo = what == 2 && k < p.steps - 2, write_lo = what == 2 && k + 1 < p.steps - 2;
            const float alpha = what == 0 ? p.S / xs / xs : what == 1 ? kC / p.S : 1.0f / p.S;
            for (int t = rank; t < tiles; t += p.blocks, ++done) {
                const int row = t / tiles_n * 128 + 32 * warp + lane, n0 = t % tiles_n * 64;
                const int64_t at = what == 2 ? x0 + row * p.n_pitch + n0 : a0 + row * p.m_pitch + n0;
                const bool there = row < p.m;
                // (read where other blocks wrote: from L2)
                uint4 x[2][2][4];
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int left = there ? N - n0 - 32 * c : 0;
                    if (what == 1) load_row(p.A + at + 32 * c, left, x[c][0]);
                    if (read_lo) load_row(p.lo + at + 32 * c, left, x[c][0]);
                }
                if (!__all_sync(0xFFFFFFFFu, mbar_wait(acc_bar(done & 1), (done >> 1) & 1u, abort_flag))) break;
                tc_fence_after();
                if (!kCluster && p.split > 1) {              // the sum of this block's share, [64 columns][128 rows]: the stages are done with
                    float* to = reinterpret_cast<float*>(smem_gen) + 32 * warp + lane;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        uint32_t v[32];
                        tmem_ld_32x32b_x32(tmem_base + ((uint32_t)(32 * warp) << 16) + 64u * (done & 1) + 32u * c, v);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 32; ++i) to[(32 * c + i) * 128] = steps > 0 ? __uint_as_float(v[i]) : 0.0f;
                    }
                    continue;
                }
                uint32_t v[2][32];
                tmem_ld_32x32b_x32(tmem_base + ((uint32_t)(32 * warp) << 16) + 64u * (done & 1), v[0]);
                tmem_ld_32x32b_x32(tmem_base + ((uint32_t)(32 * warp) << 16) + 64u * (done & 1) + 32u, v[1]);
                tmem_ld_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) dense::mbar_arrive(free_bar(done & 1));
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int left = there ? N - n0 - 32 * c : 0;
                    if (what == 0) Symmetric<false>{nullptr, p.S}.compute(alpha, v[c], x[c], -1);
                    else if (what == 1) Symmetric<true>{nullptr, p.S}.compute(alpha, v[c], x[c], row - lane == n0 + 32 * c ? lane : -1);
                    else if (read_lo) Apply<true>{0.0f, 0}.compute(alpha, v[c], x[c], -1);
                    else Apply<false>{0.0f, 0}.compute(alpha, v[c], x[c], -1);
                    store_row((what == 0 ? p.A : what == 1 ? p.B : p.X[(k + 1) & 1]) + at + 32 * c, left, x[c][0]);
                    if (write_lo) store_row(p.lo + at + 32 * c, left, x[c][1]);
                }
            }
            asm volatile("fence.proxy.async.global;" ::: "memory");
        }
        __syncwarp();
        if (kCluster) cluster_sync();        // the product is complete and seen by the cluster's copies
    }
    if (!kCluster && p.split > 1) {
        // Each block adds up a share of the tile's columns, in order of rank, and stores them where the tile's mirror image lies: A is
        // symmetric, and there the rows of a column are neighbours.
        const int tiles_n = (p.m + 63) / 64, m0 = rank / tiles_n * 128, n0 = rank % tiles_n * 64;
        tc_fence_before();
        __syncthreads();
        if (*abort_flag) {                   // its sum is a NaN for all that add it
            for (int i = threadIdx.x; i < 64 * 128; i += kSmallThreads) reinterpret_cast<float*>(smem_gen)[i] = __uint_as_float(0x7FFFFFFFu);
        }
        cluster_sync();
        const int share = 64 / p.split;
        const float alpha = p.S / xs / xs;
        for (int i = threadIdx.x; i < share * 16; i += kSmallThreads) {
            const int c = part * share + (i >> 4), r = (i & 15) * 8;
            if (n0 + c >= p.m || m0 + r >= p.m) continue;
            float x[8] = {};
            for (int q = 0; q < p.split; ++q) {
                const uint32_t from = map_to_cta(smem_base + (uint32_t)(c * 128 + r) * 4, q);
                const float4 a = dense::ld_cluster4(from), b = dense::ld_cluster4(from + 16);
                x[0] += a.x; x[1] += a.y; x[2] += a.z; x[3] += a.w;
                x[4] += b.x; x[5] += b.y; x[6] += b.z; x[7] += b.w;
            }
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = half_pair(x[2 * j] * alpha, x[2 * j + 1] * alpha);
            *reinterpret_cast<uint4*>(p.A + a0 + (int64_t)(n0 + c) * p.m_pitch + m0 + r) = make_uint4(w[0], w[1], w[2], w[3]);
        }
        cluster_sync();                      // no block leaves while another reads its sums
    }

    tc_fence_before();
    __syncthreads();
    if (*abort_flag && threadIdx.x == 0) {
        for (int i = 0; i < kSmallStages; ++i)
            for (uint32_t spin = 0; spin < 4096 && !mbar_try_wait(full_bar(i), 0) && !mbar_try_wait(full_bar(i), 1); ++spin) __nanosleep(64);
        p.xs[z] = __uint_as_float(0x7FFFFFFFu);
        if (p.dev_status) *p.dev_status = MVUE_ERR_DEVICE_TIMEOUT;
    }
    __syncthreads();
    if (warp == 5) {
        tc_fence_after();
        tmem_dealloc(tmem_base, 128);
    }
}

// ---- host ----------------------------------------------------------------------------------------------------------------
int64_t padded(int64_t bytes) { return (bytes + 255) / 256 * 256; }
int64_t pitch_of(int64_t n) { return (n + 7) / 8 * 8; }

// Bytes of a group's workspace, in the order X (two), lo, A, B, shares of the norms, xs.
int64_t group_bytes(int64_t count, int64_t m, int64_t n) {
    return 3 * padded(count * m * pitch_of(n) * 2) + 2 * padded(count * m * pitch_of(m) * 2) + padded(count * kMaxParts * 8) + padded(count * 4);
}
int64_t batch_of(int64_t m, int64_t n) { return std::max<int64_t>(1, std::min<int64_t>(kBatch, kBatchElements / (m * n))); }

bool extents_ok(int64_t rows, int64_t cols) {
    return rows >= 0 && cols >= 0 && std::min(rows, cols) <= kSumTerms && std::max(rows, cols) <= kMostTerms;
}

cudaLaunchConfig_t small_config(int64_t blocks, int stages, cudaLaunchAttribute (&attr)[2], int cluster, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(kSmallThreads);
    cfg.dynamicSmemBytes = (size_t)small_smem(stages);
    cfg.stream = stream;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cfg;
}

template <bool kCluster> cudaError_t launch_small(const SmallMaps& maps, const SmallParams& p, int count, int sm_count, cudaStream_t stream) {
    static PerDeviceOnce once;
    static int clusters[kMaxDevices];                        // of blocks with eight stages that run at once
    cudaLaunchAttribute attr[2];
    cudaError_t e = once_per_device(once, [&](int dev) {
        cudaError_t err = cudaFuncSetAttribute(small_kernel<4, kCluster>, cudaFuncAttributeMaxDynamicSharedMemorySize, small_smem(4));
        if (err == cudaSuccess) err = cudaFuncSetAttribute(small_kernel<8, kCluster>, cudaFuncAttributeMaxDynamicSharedMemorySize, small_smem(8));
        if (err == cudaSuccess && kCluster) {
            cudaLaunchConfig_t cfg = small_config(kSmallBlocks, 8, attr, kSmallBlocks, nullptr);
            int n = 0;
            if (cudaOccupancyMaxActiveClusters(&n, small_kernel<8, kCluster>, &cfg) == cudaSuccess) clusters[dev] = n;
            (void)cudaGetLastError();
        }
        return err;
    });
    int dev = 0;
    if (e == cudaSuccess) e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const int64_t blocks = (int64_t)p.blocks * p.split * count;
    // (18 matrices of 136 x 141: a cluster takes eight SMs of one part of the chip, and 16 of them fit)
    const int stages = (kCluster ? count <= clusters[dev] : blocks <= sm_count) ? 8 : 4;
    const cudaLaunchConfig_t cfg = small_config(blocks, stages, attr, kCluster ? kSmallBlocks : p.split, stream);
    return cudaLaunchKernelEx(&cfg, stages == 8 ? &small_kernel<8, kCluster> : &small_kernel<4, kCluster>, maps, p);
}

// The whole step of the q.count matrices of q, which have the extents q.m <= q.n.
cudaError_t run_group(Group& q, int steps, uint8_t* ws, int* dev_status, int sm_count, cudaStream_t st) {
    const int64_t m = q.m, n = q.n, mp = pitch_of(m);
    q.n_pitch = pitch_of(n);
    const int64_t x_bytes = padded(q.count * m * q.n_pitch * 2), a_bytes = padded(q.count * m * mp * 2);
    __half* X[2] = {reinterpret_cast<__half*>(ws), reinterpret_cast<__half*>(ws + x_bytes)};
    q.lo = reinterpret_cast<__half*>(ws + 2 * x_bytes);
    __half *A = reinterpret_cast<__half*>(ws + 3 * x_bytes), *B = reinterpret_cast<__half*>(ws + 3 * x_bytes + a_bytes);
    q.parts = reinterpret_cast<double*>(ws + 3 * x_bytes + 2 * a_bytes);
    q.xs = reinterpret_cast<float*>(ws + 3 * x_bytes + 2 * a_bytes + padded((int64_t)q.count * kMaxParts * 8));
    q.hi = X[0];
    q.S = (float)std::ldexp(1.0, (int)std::lround(0.5 * std::log2((double)n)));       // up to 2^10: 3.4445 S, B's largest entry, is a binary16
    q.growth = (float)std::pow((double)kA, (double)steps);
    const int64_t pieces = (m * n + 8 * kThreads - 1) / (8 * kThreads);
    q.n_parts = (int)std::min<int64_t>(pieces, kMaxParts);
    cudaError_t e = launch_dependent(&momentum_kernel, dim3(q.n_parts, q.count), dim3(kThreads), 0, st, q);
    const int64_t tiles = ((m + kTile - 1) / kTile) * ((n + kTile - 1) / kTile);
    const unsigned tile_blocks = (unsigned)std::min<int64_t>(tiles, std::max(1, 64 * sm_count / q.count));
    if (e == cudaSuccess) e = launch_dependent(&start_kernel, dim3(tile_blocks, q.count), dim3(kThreads), 0, st, q);
    const int64_t t = (m + 255) / 256, square_tiles = t * (t + 1) / 2 * q.count, rect_tiles = t * ((n + 255) / 256) * q.count;
    const bool cluster = m <= kSmallM && n <= kSmallN && (n <= kSmallN / 2 || m <= 128 || q.count >= 16);
    const bool small_square = m <= 128 || square_tiles <= (m <= kSmallM ? 4 : 1) * kSmallSquareTiles;
    const bool small_rect = m <= 128 || rect_tiles <= (m <= kSmallM ? 4 : 1) * kSmallPairTiles;
    const dense::Operand oa = {A, mp * 2, m * mp * 2}, ob = {B, mp * 2, m * mp * 2}, olo = {q.lo, q.n_pitch * 2, m * q.n_pitch * 2};
    const dense::Operand ox[2] = {{X[0], olo.pitch, olo.matrix}, {X[1], olo.pitch, olo.matrix}};
    SmallMaps maps;
    SmallParams small = {q.m, q.n, steps, kSmallBlocks, 0, 3 * steps, 1, q.n_pitch, mp, {X[0], X[1]}, q.lo, A, B, q.xs, q.S, dev_status};
    if (cluster || small_square || small_rect) {
        const auto map = [&](CUtensorMap* to, const dense::Operand& from, int64_t cols) {
            return dense::make_map_3d(to, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, from.base, cols, m, q.count, from.pitch, from.matrix, 64, 64, CU_TENSOR_MAP_SWIZZLE_128B);
        };
        if (!map(&maps.X[0], ox[0], n) || !map(&maps.X[1], ox[1], n) || !map(&maps.A, oa, m) || !map(&maps.B, ob, m)) return cudaErrorInvalidValue;
    }
    dense::SlabMaps gram, poly, apply[2];
    if (!cluster && !(small_square && small_rect)) {
        if (!dense::make_slab_map(&gram.out[0], oa, m, m, q.count, false) || !dense::make_slab_map(&gram.out[1], oa, m, m, q.count, true) ||
            !dense::make_slab_map(&poly.out[0], ob, m, m, q.count, false) || !dense::make_slab_map(&poly.out[1], ob, m, m, q.count, true) ||
            !dense::make_slab_map(&apply[0].out[0], ox[1], m, n, q.count, false) || !dense::make_slab_map(&apply[1].out[0], ox[0], m, n, q.count, false) ||
            !dense::make_slab_map(&apply[0].out[1], olo, m, n, q.count, false))
            return cudaErrorInvalidValue;
        gram.in = poly.in = gram.out[0];
        apply[0].in = apply[1].in = apply[1].out[1] = apply[0].out[1];
    }
    using KMajor = dense::Shape<false, false, 4>;
    using NMajor = dense::Shape<false, true, 4>;
    if (e == cudaSuccess && cluster) e = launch_small<true>(maps, small, q.count, sm_count, st);
    for (int phase = 0; phase < 3 * steps && e == cudaSuccess && !cluster; ++phase) {
        const int k = phase / 3, what = phase - 3 * k;
        if (what == 2 ? small_rect : small_square) {
            small.first = phase;
            small.last = phase + 1;
            small.blocks = (int)((m + 127) / 128 * (((what == 2 ? n : m) + 63) / 64));
            // as many shares as there are SMs for, of eight steps of 64 at least, or as a long sum needs.  So what goes beside a matrix decides in
            // what order its sums are added.  Shares that do not depend on it cost one side or the other: 512 x 14336 in one share 489 us instead of
            // 265, 24 of 512 x 4096 in two 1186 us instead of 776.
            small.split = 1;
            while (what == 0 && small.split < 8 &&
                   (n > kSumTerms * small.split || (2 * small.split * small.blocks * (int64_t)q.count <= sm_count && n >= 1024 * small.split)))
                small.split *= 2;
            e = launch_small<false>(maps, small, q.count, sm_count, st);
            continue;
        }
        dense::Params p = {};
        p.batch = q.count;
        p.lost = q.xs;
        p.dev_status = dev_status;
        p.M = q.m;
        p.N = what == 2 ? q.n : q.m;
        p.K = what == 0 ? q.n : q.m;
        p.symmetric = what != 2;
        const bool read_lo = k < steps - 2, write_lo = k + 1 < steps - 2;
        if (what == 0) {
            for (int64_t k0 = 0; k0 < n && e == cudaSuccess; k0 += kSumTerms) {
                p.K = (int)std::min(kSumTerms, n - k0);
                const dense::Operand part = {X[k & 1] + k0, olo.pitch, olo.matrix};
                e = k0 == 0 ? dense::launch_pair<KMajor>(p, part, part, gram, Symmetric<false>{q.xs, q.S}, st)
                            : dense::launch_pair<KMajor>(p, part, part, gram, Symmetric<false, true>{q.xs, q.S}, st);
            }
        } else if (what == 1) e = dense::launch_pair<KMajor>(p, oa, oa, poly, Symmetric<true>{q.xs, q.S}, st);
        else e = read_lo ? dense::launch_pair<NMajor>(p, ob, ox[k & 1], apply[k & 1], Apply<true>{1.0f / q.S, write_lo}, st)
                         : dense::launch_pair<NMajor>(p, ob, ox[k & 1], apply[k & 1], Apply<false>{1.0f / q.S, 0}, st);
    }
    q.hi = X[steps & 1];
    if (e == cudaSuccess) e = launch_dependent(&finish_kernel, dim3(tile_blocks, q.count), dim3(kThreads), 0, st, q);
    return e;
}

bool wide(const void* p, int64_t size, int64_t ld) { return !off(p, 8 * size) && ld % 8 == 0; }

}  // namespace
}  // namespace mvue

using namespace mvue;

extern "C" int mvue_muon_workspace_bytes(const mvue_muon_tensor* tensors, int64_t count, size_t* bytes) {
    if (!bytes || (count > 0 && !tensors)) return MVUE_ERR_NULL;
    if (count < 0) return MVUE_ERR_SHAPE;
    int64_t most = 0;
    for (int64_t i = 0; i < count; ++i) {
        if (!extents_ok(tensors[i].rows, tensors[i].cols)) return MVUE_ERR_SHAPE;
        const int64_t m = std::min(tensors[i].rows, tensors[i].cols), n = std::max(tensors[i].rows, tensors[i].cols);
        if (m == 0) continue;
        int64_t same = 0;
        for (int64_t j = 0; j < count; ++j) same += std::min(tensors[j].rows, tensors[j].cols) == m && std::max(tensors[j].rows, tensors[j].cols) == n;
        most = std::max(most, group_bytes(std::min(same, batch_of(m, n)), m, n));
    }
    *bytes = (size_t)most;
    return MVUE_OK;
}

extern "C" int mvue_muon_step(const mvue_muon_tensor* tensors, int64_t count, const mvue_muon_config* cfg, void* workspace,
                              size_t workspace_bytes, int* dev_status, void* stream) {
    if (!cfg || (count > 0 && !tensors)) return MVUE_ERR_NULL;
    if (count < 0 || cfg->ns_steps < 1 || cfg->ns_steps > 16) return MVUE_ERR_SHAPE;
    if (cfg->options & ~(uint32_t)(MVUE_OPT_STOCHASTIC_ROUNDING | MVUE_OPT_NESTEROV)) return MVUE_ERR_OPTION;
    if (cfg->scale_rule != MVUE_MUON_SCALE_RMS && cfg->scale_rule != MVUE_MUON_SCALE_SHAPE) return MVUE_ERR_OPTION;
    if (!(cfg->momentum >= 0.0 && cfg->momentum < 1.0)) return MVUE_ERR_OPTION;
    for (int64_t i = 0; i < count; ++i) {
        const mvue_muon_tensor& t = tensors[i];
        if (!extents_ok(t.rows, t.cols)) return MVUE_ERR_SHAPE;
        if ((t.param_dtype != MVUE_F32 && t.param_dtype != MVUE_BF16) || (t.grad_dtype != MVUE_F32 && t.grad_dtype != MVUE_BF16) ||
            (t.master && t.param_dtype != MVUE_BF16))
            return MVUE_ERR_DTYPE;
        if (t.rows == 0 || t.cols == 0) continue;
        if (!t.param || !t.grad || !t.momentum) return MVUE_ERR_NULL;
        if (off(t.param, size_of(t.param_dtype)) || off(t.grad, size_of(t.grad_dtype)) || off(t.master, 4) || off(t.momentum, 4)) return MVUE_ERR_ALIGN;
    }
    size_t need = 0;
    if (int s = mvue_muon_workspace_bytes(tensors, count, &need)) return s;
    if (need == 0) return MVUE_OK;
    if (!workspace || off(workspace, 256) || workspace_bytes < need) return MVUE_ERR_WORKSPACE;
    DeviceInfo dev;
    if (int s = current_device_info(&dev)) return s;

    Group q = {};
    q.mu = (float)cfg->momentum;
    q.one_mu = (float)(1.0 - cfg->momentum);
    q.grad_scale = (float)cfg->grad_scale;
    q.dev_grad_scale = cfg->dev_grad_scale;
    q.decay = (float)(1.0 - cfg->lr * cfg->weight_decay);
    q.nesterov = (cfg->options & MVUE_OPT_NESTEROV) != 0;
    q.random = (cfg->options & MVUE_OPT_STOCHASTIC_ROUNDING) != 0;
    q.keys = make_round_keys(cfg->seed);
    for (int64_t i = 0; i < count; ++i) {
        const int64_t rows = tensors[i].rows, cols = tensors[i].cols;
        if (rows == 0 || cols == 0) continue;
        bool seen = false;                                      // rows and cols both, since the scale rule may tell them apart
        for (int64_t j = 0; j < i && !seen; ++j) seen = tensors[j].rows == rows && tensors[j].cols == cols;
        if (seen) continue;
        const int64_t m = std::min(rows, cols), n = std::max(rows, cols), batch = batch_of(m, n);
        q.m = (int)m;
        q.n = (int)n;
        q.ld_grad = q.ld_param = cols;
        const double s = cfg->scale_rule == MVUE_MUON_SCALE_RMS ? 0.2 * std::sqrt((double)n) : std::sqrt(std::max(1.0, (double)rows / (double)cols));
        q.size = (float)(cfg->lr * s);
        q.count = 0;
        int64_t blocks = 0;
        for (int64_t j = 0; j < count; ++j) {
            const mvue_muon_tensor& t = tensors[j];
            const int64_t numel = t.rows * t.cols;
            if (t.rows == rows && t.cols == cols) {
                Matrix& x = q.matrix[q.count++];
                x = {t.grad, static_cast<float*>(t.momentum), t.param, static_cast<float*>(t.master), blocks, 0u, 0u};
                x.flags = (rows > cols ? kTransposed : 0u) | (t.grad_dtype == MVUE_BF16 ? kGradBf16 : 0u) | (t.param_dtype == MVUE_BF16 ? kParamBf16 : 0u);
                if (wide(t.grad, size_of(t.grad_dtype), cols) && wide(t.momentum, 4, cols)) x.flags |= kWideIn;
                if (wide(t.param, size_of(t.param_dtype), cols) && wide(t.master, 4, cols)) x.flags |= kWideOut;
            }
            blocks += (numel + 255) / 256;
            if (q.count == batch || (j + 1 == count && q.count > 0)) {
                const cudaError_t e = run_group(q, cfg->ns_steps, static_cast<uint8_t*>(workspace), dev_status, dev.sm_count, reinterpret_cast<cudaStream_t>(stream));
                if (e != cudaSuccess) { set_cuda_error(e, "mvue_muon_step launch"); return MVUE_ERR_CUDA; }
                q.count = 0;
            }
        }
    }
    return MVUE_OK;
}

extern "C" int mvue_orthogonalize_workspace_bytes(int64_t batch, int64_t rows, int64_t cols, size_t* bytes) {
    if (!bytes) return MVUE_ERR_NULL;
    if (batch < 0 || !extents_ok(rows, cols)) return MVUE_ERR_SHAPE;
    const int64_t m = std::min(rows, cols), n = std::max(rows, cols);
    *bytes = batch == 0 || m == 0 ? 0 : (size_t)group_bytes(std::min(batch, batch_of(m, n)), m, n);
    return MVUE_OK;
}

extern "C" int mvue_orthogonalize(const void* x, int dtype, int64_t batch, int64_t rows, int64_t cols, int64_t ldx, int64_t x_stride, int ns_steps,
                                  void* out, int out_dtype, int64_t ldo, int64_t out_stride, void* workspace, size_t workspace_bytes,
                                  int* dev_status, void* stream) {
    if ((dtype != MVUE_F32 && dtype != MVUE_BF16) || (out_dtype != MVUE_F32 && out_dtype != MVUE_BF16)) return MVUE_ERR_DTYPE;
    if (ns_steps < 1 || ns_steps > 16 || ldx < cols || ldo < cols || x_stride < 0 || out_stride < 0) return MVUE_ERR_SHAPE;
    size_t need = 0;
    if (int s = mvue_orthogonalize_workspace_bytes(batch, rows, cols, &need)) return s;
    // results one behind the other, or the rows of all matrices side by side
    if (batch > 1 && need > 0 && (rows - 1) * ldo + cols > out_stride && (out_stride < cols || (batch - 1) * out_stride + cols > ldo)) return MVUE_ERR_SHAPE;
    if (need == 0) return MVUE_OK;
    if (!x || !out) return MVUE_ERR_NULL;
    if (off(x, size_of(dtype)) || off(out, size_of(out_dtype))) return MVUE_ERR_ALIGN;
    if (!workspace || off(workspace, 256) || workspace_bytes < need) return MVUE_ERR_WORKSPACE;
    DeviceInfo dev;
    if (int s = current_device_info(&dev)) return s;
    Group q = {};
    q.m = (int)std::min(rows, cols);
    q.n = (int)std::max(rows, cols);
    q.ld_grad = ldx;
    q.ld_param = ldo;
    q.grad_scale = 1.0f;
    const int64_t most = batch_of(q.m, q.n);
    for (int64_t z = 0; z < batch;) {
        for (q.count = 0; q.count < most && z < batch; ++z) {
            Matrix& t = q.matrix[q.count++];
            t = {static_cast<const uint8_t*>(x) + z * x_stride * size_of(dtype), nullptr,
                 static_cast<uint8_t*>(out) + z * out_stride * size_of(out_dtype), nullptr, 0, 0u, 0u};
            t.flags = (rows > cols ? kTransposed : 0u) | (dtype == MVUE_BF16 ? kGradBf16 : 0u) | (out_dtype == MVUE_BF16 ? kParamBf16 : 0u);
            if (wide(t.grad, size_of(dtype), ldx)) t.flags |= kWideIn;
            if (wide(t.param, size_of(out_dtype), ldo)) t.flags |= kWideOut;
        }
        const cudaError_t e = run_group(q, ns_steps, static_cast<uint8_t*>(workspace), dev_status, dev.sm_count, reinterpret_cast<cudaStream_t>(stream));
        if (e != cudaSuccess) { set_cuda_error(e, "mvue_orthogonalize launch"); return MVUE_ERR_CUDA; }
    }
    return MVUE_OK;
}
