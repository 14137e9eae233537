// Layer normalisation over the columns of a matrix, forward and backward.
//
// Bytes bound it: the forward pass reads x and writes y, the backward pass reads x and dy and writes dx, all once.  A team of threads
// owns rows and holds them in registers until their sums are there; the next rows are on their way meanwhile.  Variances are
// taken about the mean.  Rows are taken several at a time, so that one barrier serves their sums, and in a warp the lanes fold (six
// shuffles for four sums instead of twenty).
// Weight and bias gradients: a thread keeps the sums of its columns for all of its rows, a block's teams join in shared memory,
// blocks leave one partial sum each, and a second launch adds those in order: equal inputs give equal bits.
//   forward8, backward8   accesses of eight elements and rows for all SMs; the weight in shared memory, packed pairs of binary32.
//                         16384 x 4096 bf16 forward 53 us (5.0 of 6.46 TB/s copy), 32768 x 1024 bf16 backward 43 us (4.7 TB/s):
//                         half of the issue slots are taken, and a barrier in three phases keeps 16 warps an SM from more.  4096 x 14336
//                         bf16 forward 59 to 70 us, by where the buffers lie
//   forward, backward     any alignment, up to 4096 columns, and few rows; the weight in registers (4097 x 1111 fp32 backward 17 us
//                         with the join, 8 x 4096 bf16 forward 2.1 us)
//   wide                  rows that do not fit a block's threads are gone over again, from L2; column sums in shared memory
//                         (4096 x 14344 bf16 forward 89 us, 4096 x 14336 backward 160 us: three and two times over the row, not bandwidth)
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <type_traits>

#include "../../include/mvue_layer.h"
#include "mvue_device.cuh"
#include "mvue_internal.h"
#include "mvue_train.cuh"

namespace mvue {
namespace {

constexpr int kMaxTeam = 512;                    // threads; eight columns each in the kernels for any alignment
constexpr int kWideThreads = 1024;
constexpr int64_t kWideSums = 24576;             // columns whose sums an SM's shared memory holds, eight bytes each
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

// bf16 rows that are not whole pieces of eight, or do not begin at one, still have aligned pieces inside.  A thread's eight neighbours begin
// at 8 lane - shift, where the row begins `shift` elements behind an aligned address: all pieces but the first and the last are accesses
// of eight.  Rows eight apart have the same shift, so a block that takes such rows has the same columns in a thread all along.
// 16384 x 1111: forward 29 us, backward 40 us (with accesses of single elements 55 and 78, of pairs for 1110 columns 47 and 54).  fp32 in
// single elements and pairs is as fast (16384 x 1110: 33 and 42 us; shifted 35 and 49).
constexpr int kShifted = 16;
template <int kVec> struct Place : Cols<kVec> {
    __device__ __forceinline__ Place(int64_t cols, int lane, int team, int) : Cols<kVec>(0, cols, lane, team) {}
    __device__ __forceinline__ bool has(int j) const { return j < this->count; }
};
template <> struct Place<kShifted> {
    int64_t first, second;                       // the second thread's first, of a whole piece
    int from, count;                             // of the eight, those in [from, count) exist
    __device__ __forceinline__ Place(int64_t cols, int lane, int, int shift) {
        first = 8 * (int64_t)lane - shift;
        second = 8 - shift;
        from = first < 0 ? (int)-first : 0;
        count = (int)min((int64_t)8, cols - first);
    }
    __device__ __forceinline__ bool whole() const { return from == 0 && count == 8; }
    __device__ __forceinline__ bool has(int j) const { return j >= from && j < count; }
    __device__ __forceinline__ int64_t at(int j) const { return first + j; }
    __device__ __forceinline__ void store(__nv_bfloat16* row, const float (&x)[8]) const {
        if (whole()) {
            Cols<8> c(0, 8, 0, 1);
            c.store(row + first, x);
        } else {
            const uint32_t own = bits();
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (own >> j & 1u) row[first + j] = __float2bfloat16_rn(x[j]);
        }
    }
    __device__ __forceinline__ uint32_t bits() const { return count <= 0 ? 0u : (0xFFu << from) & (0xFFu >> (8 - count)); }
};
// A thread's eight elements as they were read, so that nothing waits for them before they are used.
template <typename T, int kVec> struct Held {
    static constexpr bool kPairs = sizeof(T) == 2 && kVec != 1;
    uint32_t w[kPairs ? 4 : 8];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (uint32_t& x : w) x = 0u;
    }
    __device__ __forceinline__ void wide(const T* p) {
        if constexpr (sizeof(T) == 2) {
            const uint4 v = *reinterpret_cast<const uint4*>(p);
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        } else {
            ld256(p, w);
        }
    }
    // Row `row` of the `rows` at `base`; one that does not exist leaves what there is.  kShifted: without a choice between accesses, which would
    // wait for the elements.  A piece that is not all of its row's takes elements of the rows beside it too, or where there are none gives
    // way to the second piece (whole in sixteen columns).  All of a block's rows have its shift: an access begins at 8 elements.
    __device__ __forceinline__ void load(const Place<kVec>& c, const T* base, int64_t ld, int64_t row, int64_t rows) {
        if constexpr (kVec == kShifted) {
            if (row < rows) wide(base + row * ld + (c.whole() || (c.count > 0 && beside(row, rows)) ? c.first : c.second));
        } else {
            if (row >= rows || c.count <= 0) {
                clear();
                return;
            }
            const T* from = base + row * ld;
            if constexpr (kVec == 8) {
                wide(from + c.first);
            } else if constexpr (kVec == 2) {
                clear();
#pragma unroll
                for (int j = 0; j < 8; j += 2)
                    if (c.has(j)) {
                        if constexpr (sizeof(T) == 2) {
                            w[j / 2] = *reinterpret_cast<const uint32_t*>(from + c.at(j));
                        } else {
                            const uint2 v = *reinterpret_cast<const uint2*>(from + c.at(j));
                            w[j] = v.x;
                            w[j + 1] = v.y;
                        }
                    }
            } else {
                clear();
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c.has(j)) {
                        if constexpr (sizeof(T) == 2) w[j] = *reinterpret_cast<const unsigned short*>(from + c.at(j));
                        else w[j] = __float_as_uint(from[c.at(j)]);
                    }
            }
        }
    }
    static __device__ __forceinline__ bool beside(int64_t row, int64_t rows) { return row > 0 && row + 1 < rows; }
    // What a piece has of its own, without a comparison for each element of each row: a mask for the words, and one or zero for the mean.
    struct Own {
        uint32_t words[4];
        float one[8];
        __device__ __forceinline__ Own(const Place<kVec>& c) {
#pragma unroll
            for (int j = 0; j < 8; ++j) one[j] = c.has(j) ? 1.0f : 0.0f;
            if constexpr (kVec == kShifted) {
#pragma unroll
                for (int i = 0; i < 4; ++i) words[i] = (c.has(2 * i) ? 0xFFFFu : 0u) | (c.has(2 * i + 1) ? 0xFFFF0000u : 0u);
            }
        }
    };
    __device__ __forceinline__ void floats(const Place<kVec>& c, const Own& own, const T* base, int64_t ld, int64_t row, int64_t rows, float (&x)[8]) const {
        constexpr bool kShift = kVec == kShifted;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if constexpr (kPairs) {
                const uint32_t v = kShift ? w[j / 2] & own.words[j / 2] : w[j / 2];
                x[j] = j & 1 ? bf16_hi(v) : bf16_lo(v);
            } else {
                x[j] = __uint_as_float(sizeof(T) == 2 ? w[j] << 16 : w[j]);
            }
        }
        if constexpr (kShift) {
            if (!beside(row, rows)) {                        // (the first row, the last, and those that do not exist)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (row >= rows) x[j] = 0.0f;
                    else if (!c.whole() && c.has(j)) x[j] = __bfloat162float(base[row * ld + c.at(j)]);
            }
        }
    }
};

template <int kVec> __device__ __forceinline__ bool there(const Cols<kVec>& c, int j) { return j < c.count; }
__device__ __forceinline__ bool there(const Place<kShifted>& c, int j) { return c.has(j); }
// Eight columns of weight or bias; `none` where there is no such tensor.
template <typename C> __device__ __forceinline__ void load_affine(const C& c, const void* from, int bf16, float none, float (&v)[8]) {
    if (!from) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = none;
        return;
    }
    constexpr bool kEight = std::is_base_of<Cols<8>, C>::value;
    if (kEight && c.count == 8 && (reinterpret_cast<uintptr_t>(from) & 31u) == 0) {
        if (bf16) load8(static_cast<const __nv_bfloat16*>(from) + c.first, true, 8, v);
        else load8(static_cast<const float*>(from) + c.first, true, 8, v);
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
        v[j] = !there(c, j) ? 0.0f : bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(from)[c.at(j)]) : static_cast<const float*>(from)[c.at(j)];
}

__device__ __forceinline__ void team_barrier(int team, int threads) {
    if (threads == 32) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(threads) : "memory");
}

// Sums of kN (1, 2 or 4) values over a team.  Within a warp the lanes fold: each exchange leaves a lane with half of the values, and
// the last ones are added up (four values: six shuffles instead of twenty).  `sums`: the team's slots, four for each of its warps; not
// used again before another barrier of the team.
template <int kN>
__device__ __forceinline__ void team_sum(float (&v)[kN], float (*sums)[4], int team, int threads, int warp, int lane) {
    float t;
    if constexpr (kN == 4) {
        const bool b0 = lane & 1, b1 = lane & 2;
        const float p = (b0 ? v[2] : v[0]) + __shfl_xor_sync(0xFFFFFFFFu, b0 ? v[0] : v[2], 1);
        const float q = (b0 ? v[3] : v[1]) + __shfl_xor_sync(0xFFFFFFFFu, b0 ? v[1] : v[3], 1);
        t = (b1 ? q : p) + __shfl_xor_sync(0xFFFFFFFFu, b1 ? p : q, 2);             // value 2 (lane & 1) + (lane >> 1 & 1)
    } else if constexpr (kN == 2) {
        t = (lane & 1 ? v[1] : v[0]) + __shfl_xor_sync(0xFFFFFFFFu, lane & 1 ? v[0] : v[1], 1);
    } else {
        t = v[0];
    }
#pragma unroll
    for (int d = kN; d < 32; d <<= 1) t += __shfl_xor_sync(0xFFFFFFFFu, t, d);
    if (threads > 32) {
        if (lane < kN) sums[warp][lane] = t;
        team_barrier(team, threads);
        t = 0.0f;
        for (int w = lane / kN; w < (threads >> 5); w += 32 / kN) t += sums[w][lane % kN];
#pragma unroll
        for (int d = kN; d < 32; d <<= 1) t += __shfl_xor_sync(0xFFFFFFFFu, t, d);
    }
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = __shfl_sync(0xFFFFFFFFu, t, kN == 4 ? (i >> 1) | (i & 1) << 1 : i);
}

// Eight neighbours as they lie in memory.
template <typename T> struct Raw;
template <> struct Raw<__nv_bfloat16> {
    uint32_t w[4];
    __device__ __forceinline__ void load(const __nv_bfloat16* p) {
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    }
    __device__ __forceinline__ f2 two(int i) const { return pair(bf16_lo(w[i]), bf16_hi(w[i])); }          // elements 2i, 2i + 1
};
template <> struct Raw<float> {
    uint32_t w[8];
    __device__ __forceinline__ void load(const float* p) { ld256(p, w); }
    __device__ __forceinline__ f2 two(int i) const { return pair(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1])); }
};
__device__ __forceinline__ void floats_of(const f2 (&p)[4], float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) unpair(p[i], x[2 * i], x[2 * i + 1]);
}
__device__ __forceinline__ void store_eight(float* to, const f2 (&p)[4]) {
    float x[8];
    floats_of(p, x);
    store8(to, true, 8, x);
}
__device__ __forceinline__ void store_eight(__nv_bfloat16* to, const f2 (&p)[4]) {
    float x[8];
    floats_of(p, x);
    *reinterpret_cast<uint4*>(to) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}
__device__ __forceinline__ float both(f2 a) {
    float lo, hi;
    unpair(a, lo, hi);
    return lo + hi;
}
// Weight or bias in shared memory as binary32, in the order in which a team's threads read it without conflicts: the piece of eight columns
// with number i lies as two quarters of 16 bytes, `pieces` such quarters apart.
__device__ __forceinline__ void stage_quarters(float* to, const void* from, int bf16, float none, int cols) {
    const int pieces = cols >> 3;
    for (int i = threadIdx.y * blockDim.x + threadIdx.x; i < cols; i += blockDim.x * blockDim.y)
        to[((i >> 2 & 1) * pieces + (i >> 3)) * 4 + (i & 3)] =
            !from ? none : bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(from)[i]) : static_cast<const float*>(from)[i];
}
__device__ __forceinline__ void quarters_of(const float* from, int piece, int pieces, f2 (&x)[4]) {
    const float4 a = reinterpret_cast<const float4*>(from)[piece], b = reinterpret_cast<const float4*>(from)[pieces + piece];
    x[0] = pair(a.x, a.y);
    x[1] = pair(a.z, a.w);
    x[2] = pair(b.x, b.y);
    x[3] = pair(b.z, b.w);
}

// Means and sums of squares about them of kR rows over a team whose threads have `count` elements of each.  Equal counts n join as
// m = (m_a + m_b) / 2, M2 = M2_a + M2_b + (m_b - m_a)^2 n / 2; in a warp the lanes fold as in team_sum.
template <int kR>
__device__ __forceinline__ void team_moments(float (&mean)[kR], float (&m2)[kR], float2 (*slots)[kR], int team, int threads, int warp, int lane, float count) {
    const auto join = [](float& m, float& q, float om, float oq, float half_n) {
        const float delta = om - m;
        q = fmaf(delta * delta, half_n, q + oq);
        m = fmaf(0.5f, delta, m);
    };
    float m = mean[0], q = m2[0], half_n = 0.5f * count;
    int d = 1;
    if constexpr (kR == 4) {
        const bool up = lane & 1;
        float ma = up ? mean[2] : mean[0], qa = up ? m2[2] : m2[0], mb = up ? mean[3] : mean[1], qb = up ? m2[3] : m2[1];
        join(ma, qa, __shfl_xor_sync(0xFFFFFFFFu, up ? mean[0] : mean[2], 1), __shfl_xor_sync(0xFFFFFFFFu, up ? m2[0] : m2[2], 1), half_n);
        join(mb, qb, __shfl_xor_sync(0xFFFFFFFFu, up ? mean[1] : mean[3], 1), __shfl_xor_sync(0xFFFFFFFFu, up ? m2[1] : m2[3], 1), half_n);
        half_n *= 2.0f;
        const bool up2 = lane & 2;
        m = up2 ? mb : ma;
        q = up2 ? qb : qa;
        join(m, q, __shfl_xor_sync(0xFFFFFFFFu, up2 ? ma : mb, 2), __shfl_xor_sync(0xFFFFFFFFu, up2 ? qa : qb, 2), half_n);
        half_n *= 2.0f;
        d = 4;
    } else if constexpr (kR == 2) {
        const bool up = lane & 1;
        m = up ? mean[1] : mean[0];
        q = up ? m2[1] : m2[0];
        join(m, q, __shfl_xor_sync(0xFFFFFFFFu, up ? mean[0] : mean[1], 1), __shfl_xor_sync(0xFFFFFFFFu, up ? m2[0] : m2[1], 1), half_n);
        half_n *= 2.0f;
        d = 2;
    }
#pragma unroll
    for (; d < 32; d <<= 1) {
        join(m, q, __shfl_xor_sync(0xFFFFFFFFu, m, d), __shfl_xor_sync(0xFFFFFFFFu, q, d), half_n);
        half_n *= 2.0f;
    }
    if (threads > 32) {
        const int warps = threads >> 5;
        if (lane < kR) slots[warp][lane] = make_float2(m, q);
        team_barrier(team, threads);
        // lane r + kR w holds row r of warp w (several where there are more warps than that)
        float2 own[kR];
        float total = 0.0f;
#pragma unroll
        for (int i = 0; i < kR; ++i) {
            const int w = lane / kR + i * (32 / kR);
            own[i] = w < warps ? slots[w][lane % kR] : make_float2(0.0f, 0.0f);
            total += own[i].x;
        }
#pragma unroll
        for (int e = kR; e < 32; e <<= 1) total += __shfl_xor_sync(0xFFFFFFFFu, total, e);
        m = total / (float)warps;
        q = 0.0f;
#pragma unroll
        for (int i = 0; i < kR; ++i)
            if (lane / kR + i * (32 / kR) < warps) q += fmaf((own[i].x - m) * (own[i].x - m), 32.0f * count, own[i].y);
#pragma unroll
        for (int e = kR; e < 32; e <<= 1) q += __shfl_xor_sync(0xFFFFFFFFu, q, e);
    }
#pragma unroll
    for (int i = 0; i < kR; ++i) {
        const int from = kR == 4 ? (i >> 1) | (i & 1) << 1 : i;
        mean[i] = __shfl_sync(0xFFFFFFFFu, m, from);
        m2[i] = __shfl_sync(0xFFFFFFFFu, q, from);
    }
}

// Many rows that the team's threads cover exactly, kC pieces of eight columns each: a thread holds its pieces of kR rows while the next
// rows' are on their way; weight and bias wait in shared memory and are read once for the kR rows.  One barrier for the kR rows: each thread
// takes mean and squares about it of its own elements.
// 16384 x 4096 bf16: a row at a time, with the weight's pieces in their own order (bank conflicts), took 71 us.
constexpr int kEightThreads = 512;
template <typename T, int kC, int kR>
__global__ void __launch_bounds__(kEightThreads, 1) forward8_kernel(const __grid_constant__ Params p) {
    __shared__ float2 slots[2][kEightThreads / 32][kR];
    extern __shared__ __align__(16) float affine[];
    const int threads = blockDim.x, team = threadIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int cols = (int)p.cols, pieces = cols >> 3, step = threads * 8;
    const int64_t first = ((int64_t)blockIdx.x * blockDim.y + team) * kR, stride = (int64_t)gridDim.x * blockDim.y * kR;
    const T* from = static_cast<const T*>(p.x) + first * p.ldx + threadIdx.x * 8;
    T* to = static_cast<T*>(p.y) + first * p.ldy + threadIdx.x * 8;
    Raw<T> next[kR][kC];
    const auto fetch = [&](int64_t row) {                    // (rows beyond the last: the last, which nobody stores)
#pragma unroll
        for (int r = 0; r < kR; ++r) {
            const T* at = from + (row + r < p.rows ? r : p.rows - 1 - row) * p.ldx;
#pragma unroll
            for (int c = 0; c < kC; ++c) next[r][c].load(at + c * step);
        }
    };
    grid_dependency_wait();
    if (first < p.rows) fetch(first);
    stage_quarters(affine, p.gamma, p.affine_bf16, 1.0f, cols);
    stage_quarters(affine + cols, p.beta, p.affine_bf16, 0.0f, cols);
    __syncthreads();
    int turn = 0;
    for (int64_t row = first; row < p.rows; row += stride, turn ^= 1) {
        f2 v[kR][kC][4];
        float own[kR], mean[kR], m2[kR];
#pragma unroll
        for (int r = 0; r < kR; ++r) {
            f2 sum = pair(0.0f);
#pragma unroll
            for (int c = 0; c < kC; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    v[r][c][j] = next[r][c].two(j);
                    sum = add2(sum, v[r][c][j]);
                }
            own[r] = both(sum) * (1.0f / (8 * kC));
        }
        from += stride * p.ldx;
        if (row + stride < p.rows) fetch(row + stride);
#pragma unroll
        for (int r = 0; r < kR; ++r) {
            f2 sum = pair(0.0f);
#pragma unroll
            for (int c = 0; c < kC; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    v[r][c][j] = add2(v[r][c][j], pair(-own[r]));
                    sum = fma2(v[r][c][j], v[r][c][j], sum);
                }
            mean[r] = own[r];
            m2[r] = both(sum);
        }
        team_moments<kR>(mean, m2, slots[turn] + team * (threads >> 5), team, threads, warp, lane, (float)(8 * kC));
#pragma unroll
        for (int r = 0; r < kR; ++r) {
            m2[r] = rsqrtf(fmaf(m2[r], p.inv_cols, p.eps));
            if (threadIdx.x == 0 && row + r < p.rows) {
                if (p.mean) p.mean[row + r] = mean[r];
                if (p.rstd) p.rstd[row + r] = m2[r];
            }
        }
#pragma unroll
        for (int c = 0; c < kC; ++c) {
            f2 gamma[4], beta[4], o[4];
            quarters_of(affine, threadIdx.x + c * threads, pieces, gamma);
            quarters_of(affine + cols, threadIdx.x + c * threads, pieces, beta);
#pragma unroll
            for (int r = 0; r < kR; ++r) {
                if (row + r >= p.rows) break;
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = fma2(mul2(add2(v[r][c][j], pair(own[r] - mean[r])), pair(m2[r])), gamma[j], beta[j]);
                store_eight(to + r * p.ldy + c * step, o);
            }
        }
        to += stride * p.ldy;
    }
}

// The teams of a block add up their column sums in order, each thread its own places, and the block leaves its partial sum.
template <int kN>
__device__ __forceinline__ bool join_teams(float (&dgamma)[kN], float (&dbeta)[kN], float* joined, int team, int threads) {
    if (blockDim.y > 1) {
        float* at = joined + threadIdx.x;
        for (int t = 0; t < (int)blockDim.y; ++t) {
            if (t == team) {
#pragma unroll
                for (int j = 0; j < kN; ++j) {
                    at[2 * j * threads] = t == 0 ? dgamma[j] : at[2 * j * threads] + dgamma[j];
                    at[(2 * j + 1) * threads] = t == 0 ? dbeta[j] : at[(2 * j + 1) * threads] + dbeta[j];
                }
            }
            __syncthreads();
        }
        if (team != 0) return false;
#pragma unroll
        for (int j = 0; j < kN; ++j) {
            dgamma[j] = at[2 * j * threads];
            dbeta[j] = at[(2 * j + 1) * threads];
        }
    }
    return true;
}

// The same for the backward pass: kR rows, two sums each.  kFull: the team's threads cover a row exactly.
template <typename T, int kC, int kR, bool kSums, bool kFull>
__global__ void __launch_bounds__(kEightThreads, 1) backward8_kernel(const __grid_constant__ Params p) {
    __shared__ float slots[2][32][4];
    extern __shared__ __align__(16) float affine[];          // the weight; at the end the teams' sums
    const int threads = blockDim.x, team = threadIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int cols = (int)p.cols, pieces = cols >> 3, c0 = threadIdx.x * 8, step = threads * 8;
    const T *x = static_cast<const T*>(p.x), *dy = static_cast<const T*>(p.dy);
    T* dx = static_cast<T*>(p.dx);
    const int64_t stride = (int64_t)gridDim.x * blockDim.y * kR;
    int64_t row = ((int64_t)blockIdx.x * blockDim.y + team) * kR;
    Raw<T> next_x[kR][kC], next_g[kR][kC];
    float next_mean[kR], next_rstd[kR];
    f2 dgamma[4 * kC], dbeta[4 * kC];
#pragma unroll
    for (int j = 0; j < 4 * kC; ++j) dgamma[j] = dbeta[j] = pair(0.0f);
    const auto fetch = [&](int64_t from) {
#pragma unroll
        for (int r = 0; r < kR; ++r) {
            const bool there = from + r < p.rows;
            next_mean[r] = there ? p.mean_in[from + r] : 0.0f;
            next_rstd[r] = there ? p.rstd_in[from + r] : 0.0f;
#pragma unroll
            for (int c = 0; c < kC; ++c)
                if (there && (kFull || c0 + c * step < cols)) {
                    next_x[r][c].load(x + (from + r) * p.ldx + c0 + c * step);
                    next_g[r][c].load(dy + (from + r) * p.lddy + c0 + c * step);
                } else {
#pragma unroll
                    for (uint32_t& w : next_x[r][c].w) w = 0u;
#pragma unroll
                    for (uint32_t& w : next_g[r][c].w) w = 0u;
                }
        }
    };
    grid_dependency_wait();
    fetch(row);
    stage_quarters(affine, p.gamma, p.affine_bf16, 1.0f, cols);
    __syncthreads();
    int turn = 0;
    for (; row < p.rows; row += stride, turn ^= 1) {
        f2 xh[kR][kC][4], w[kR][kC][4];
        float rstd[kR], s[2 * kR];
#pragma unroll
        for (int r = 0; r < kR; ++r) {
            rstd[r] = next_rstd[r];
            const f2 minus = pair(-next_mean[r]), scale = pair(rstd[r]);
#pragma unroll
            for (int c = 0; c < kC; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    xh[r][c][j] = mul2(add2(next_x[r][c].two(j), minus), scale);
                    w[r][c][j] = next_g[r][c].two(j);
                }
        }
        fetch(row + stride);
        f2 s0[kR], s1[kR];
#pragma unroll
        for (int r = 0; r < kR; ++r) s0[r] = s1[r] = pair(0.0f);
#pragma unroll
        for (int c = 0; c < kC; ++c) {
            if (!kFull && c0 + c * step >= cols) break;
            f2 gamma[4];
            quarters_of(affine, threadIdx.x + c * threads, pieces, gamma);
#pragma unroll
            for (int r = 0; r < kR; ++r) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (kSums) {
                        dgamma[4 * c + j] = fma2(w[r][c][j], xh[r][c][j], dgamma[4 * c + j]);
                        dbeta[4 * c + j] = add2(dbeta[4 * c + j], w[r][c][j]);
                    }
                    w[r][c][j] = mul2(w[r][c][j], gamma[j]);
                    s0[r] = add2(s0[r], w[r][c][j]);
                    s1[r] = fma2(w[r][c][j], xh[r][c][j], s1[r]);
                }
            }
        }
#pragma unroll
        for (int r = 0; r < kR; ++r) {
            s[2 * r] = both(s0[r]);
            s[2 * r + 1] = both(s1[r]);
        }
        team_sum<2 * kR>(s, slots[turn] + team * (threads >> 5), team, threads, warp, lane);
#pragma unroll
        for (int c = 0; c < kC; ++c) {
            if (!kFull && c0 + c * step >= cols) break;
#pragma unroll
            for (int r = 0; r < kR; ++r) {
                if (row + r >= p.rows) break;
                const f2 m0 = pair(-s[2 * r] * p.inv_cols), m1 = pair(-s[2 * r + 1] * p.inv_cols), scale = pair(rstd[r]);
                f2 o[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = mul2(scale, add2(w[r][c][j], fma2(xh[r][c][j], m1, m0)));
                store_eight(dx + (row + r) * p.ldy + c0 + c * step, o);
            }
        }
    }
    if constexpr (kSums) {
        float a[8 * kC], b[8 * kC];
#pragma unroll
        for (int j = 0; j < 4 * kC; ++j) {
            unpair(dgamma[j], a[2 * j], a[2 * j + 1]);
            unpair(dbeta[j], b[2 * j], b[2 * j + 1]);
        }
        __syncthreads();
        if (!join_teams(a, b, affine, team, threads)) return;
        float* out = p.partial + (int64_t)blockIdx.x * 2 * p.cols;
#pragma unroll
        for (int c = 0; c < kC; ++c) {
            if (c0 + c * step >= cols) break;
            float4 *to_a = reinterpret_cast<float4*>(out + c0 + c * step), *to_b = reinterpret_cast<float4*>(out + p.cols + c0 + c * step);
#pragma unroll
            for (int h = 0; h < 2; ++h) {                    // (the workspace is aligned to 16 bytes)
                to_a[h] = make_float4(a[8 * c + 4 * h], a[8 * c + 4 * h + 1], a[8 * c + 4 * h + 2], a[8 * c + 4 * h + 3]);
                to_b[h] = make_float4(b[8 * c + 4 * h], b[8 * c + 4 * h + 1], b[8 * c + 4 * h + 2], b[8 * c + 4 * h + 3]);
            }
        }
    }
}

// Block: blockDim.x threads a team, blockDim.y teams.  kR rows at a time: 4, or 1 where there are few.  kShifted: a block's rows lie eight
// apart, and there are a multiple of eight blocks.
template <typename T, int kVec>
struct Rows {
    static constexpr int kGap = kVec == kShifted ? 8 : 1;
    int shift;
    int64_t first, stride;
    __device__ __forceinline__ Rows(const void* base, int64_t ld, int at_once) {
        const int64_t block = kGap == 8 ? blockIdx.x >> 3 : blockIdx.x, rest = kGap == 8 ? blockIdx.x & 7 : 0;
        shift = (int)((reinterpret_cast<uintptr_t>(base) / sizeof(T) + (uint64_t)(rest * ld)) & 7u);
        first = rest + kGap * ((block * blockDim.y + threadIdx.y) * at_once);
        stride = (int64_t)gridDim.x * blockDim.y * at_once;
    }
};
template <typename T, int kVec, int kR>
__global__ void __launch_bounds__(kMaxTeam) forward_kernel(const __grid_constant__ Params p) {
    __shared__ float slots[2][32][4];
    grid_dependency_wait();
    const int threads = blockDim.x, team = threadIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float(*sums0)[4] = slots[0] + team * (threads >> 5);
    float(*sums1)[4] = slots[1] + team * (threads >> 5);
    const Rows<T, kVec> rows(p.x, p.ldx, kR);
    constexpr int kGap = Rows<T, kVec>::kGap;
    const Place<kVec> c(p.cols, threadIdx.x, threads, rows.shift);
    float gamma[8], beta[8];
    load_affine(c, p.gamma, p.affine_bf16, 1.0f, gamma);
    load_affine(c, p.beta, p.affine_bf16, 0.0f, beta);
    const T* x = static_cast<const T*>(p.x);
    T* y = static_cast<T*>(p.y);
    const bool mine = c.count > 0;
    const typename Held<T, kVec>::Own own(c);
    const int64_t stride = rows.stride;
    int64_t row = rows.first;
    Held<T, kVec> next[kR];                                  // the rows to come, on their way while these are worked on
#pragma unroll
    for (Held<T, kVec>& h : next) h.clear();
    const auto fetch = [&](int64_t from) {
#pragma unroll
        for (int r = 0; r < kR; ++r) next[r].load(c, x, p.ldx, from + r * kGap, p.rows);
    };
    fetch(row);
    for (; row < p.rows; row += stride) {
        float v[kR][8], s[kR];
#pragma unroll
        for (int r = 0; r < kR; ++r) next[r].floats(c, own, x, p.ldx, row + r * kGap, p.rows, v[r]);
        fetch(row + stride);
#pragma unroll
        for (int r = 0; r < kR; ++r) s[r] = ((v[r][0] + v[r][1]) + (v[r][2] + v[r][3])) + ((v[r][4] + v[r][5]) + (v[r][6] + v[r][7]));
        team_sum<kR>(s, sums0, team, threads, warp, lane);
        float mean[kR];
#pragma unroll
        for (int r = 0; r < kR; ++r) {
            mean[r] = s[r] * p.inv_cols;
            s[r] = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[r][j] = fmaf(-mean[r], own.one[j], v[r][j]);
                s[r] = fmaf(v[r][j], v[r][j], s[r]);
            }
        }
        team_sum<kR>(s, sums1, team, threads, warp, lane);
#pragma unroll
        for (int r = 0; r < kR; ++r) {
            const int64_t at = row + r * kGap;
            if (at >= p.rows) break;
            const float rstd = rsqrtf(fmaf(s[r], p.inv_cols, p.eps));
            if (threadIdx.x == 0) {
                if (p.mean) p.mean[at] = mean[r];
                if (p.rstd) p.rstd[at] = rstd;
            }
            if (mine) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[r][j] = fmaf(v[r][j] * rstd, gamma[j], beta[j]);
                c.store(y + at * p.ldy, v[r]);
            }
        }
    }
}

// Two rows at a time.  kSums: the column sums are wanted too.
template <typename T, int kVec, bool kSums>
__global__ void __launch_bounds__(kMaxTeam) backward_kernel(const __grid_constant__ Params p) {
    __shared__ float slots[2][32][4];
    extern __shared__ float joined[];                       // [2][blockDim.x * 8] where there are several teams
    grid_dependency_wait();
    const int threads = blockDim.x, team = threadIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Rows<T, kVec> rows(p.x, p.ldx, 2);
    constexpr int kGap = Rows<T, kVec>::kGap;
    const Place<kVec> c(p.cols, threadIdx.x, threads, rows.shift);
    float gamma[8], dgamma[8], dbeta[8];
    load_affine(c, p.gamma, p.affine_bf16, 1.0f, gamma);
#pragma unroll
    for (int j = 0; j < 8; ++j) dgamma[j] = dbeta[j] = 0.0f;
    const T *x = static_cast<const T*>(p.x), *dy = static_cast<const T*>(p.dy);
    T* dx = static_cast<T*>(p.dx);
    const bool mine = c.count > 0;
    const typename Held<T, kVec>::Own own(c);
    const int64_t stride = rows.stride;
    int64_t row = rows.first;
    Held<T, kVec> next_x[2], next_g[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        next_x[r].clear();
        next_g[r].clear();
    }
    float next_mean[2], next_rstd[2];
    const auto fetch = [&](int64_t from) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int64_t at = from + r * kGap;
            const bool there = at < p.rows;
            next_mean[r] = there ? p.mean_in[at] : 0.0f;
            next_rstd[r] = there ? p.rstd_in[at] : 0.0f;
            next_x[r].load(c, x, p.ldx, at, p.rows);
            next_g[r].load(c, dy, p.lddy, at, p.rows);
        }
    };
    fetch(row);
    int turn = 0;
    for (; row < p.rows; row += stride, turn ^= 1) {
        float xh[2][8], g[2][8], s[4], rstd[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            rstd[r] = next_rstd[r];
            next_x[r].floats(c, own, x, p.ldx, row + r * kGap, p.rows, xh[r]);
            next_g[r].floats(c, own, dy, p.lddy, row + r * kGap, p.rows, g[r]);
#pragma unroll
            for (int j = 0; j < 8; ++j) xh[r][j] = fmaf(-next_mean[r], own.one[j], xh[r][j]) * rstd[r];
        }
        fetch(row + stride);
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            s[2 * r] = s[2 * r + 1] = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (kSums) {
                    dgamma[j] = fmaf(g[r][j], xh[r][j], dgamma[j]);
                    dbeta[j] += g[r][j];
                }
                g[r][j] *= gamma[j];
                s[2 * r] += g[r][j];
                s[2 * r + 1] = fmaf(g[r][j], xh[r][j], s[2 * r + 1]);
            }
        }
        team_sum<4>(s, slots[turn] + team * (threads >> 5), team, threads, warp, lane);
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            if (row + r * kGap >= p.rows || !mine) break;
            const float m0 = s[2 * r] * p.inv_cols, m1 = s[2 * r + 1] * p.inv_cols;
#pragma unroll
            for (int j = 0; j < 8; ++j) g[r][j] = rstd[r] * (g[r][j] - fmaf(xh[r][j], m1, m0));
            c.store(dx + (row + r * kGap) * p.ldy, g[r]);
        }
    }
    if constexpr (kSums) {
        float* out = p.partial + (int64_t)blockIdx.x * 2 * p.cols;
        if (!join_teams(dgamma, dbeta, joined, team, threads)) return;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c.has(j)) {
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
    v = lane < (int)(blockDim.x >> 5) ? slots[lane] : 0.0f;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    __syncthreads();
    return v;
}

template <typename T, int kVec>
__global__ void __launch_bounds__(kWideThreads) wide_forward_kernel(const __grid_constant__ Params p) {
    __shared__ float slots[32];
    const int threads = blockDim.x;
    grid_dependency_wait();
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(p.x) + row * p.ldx;
        T* y = static_cast<T*>(p.y) + row * p.ldy;
        float s = 0.0f, v[8];
        for (int64_t c0 = 0; c0 < p.cols; c0 += 8 * threads) {
            const Cols<kVec> c(c0, p.cols, threadIdx.x, threads);
            if (c.count == 0) break;
            c.load(x, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) s += j < c.count ? v[j] : 0.0f;
        }
        const float mean = block_sum(s, slots) * p.inv_cols;
        s = 0.0f;
        for (int64_t c0 = 0; c0 < p.cols; c0 += 8 * threads) {
            const Cols<kVec> c(c0, p.cols, threadIdx.x, threads);
            if (c.count == 0) break;
            c.load(x, v);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < c.count) s = fmaf(v[j] - mean, v[j] - mean, s);
        }
        const float rstd = rsqrtf(fmaf(block_sum(s, slots), p.inv_cols, p.eps));
        for (int64_t c0 = 0; c0 < p.cols; c0 += 8 * threads) {
            const Cols<kVec> c(c0, p.cols, threadIdx.x, threads);
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

// kSums: the column sums too, in shared memory, a thread's sixteen of each slab (eight columns a thread) as four quarters that lie a
// block's threads apart.
template <typename T, int kVec, bool kSums>
__global__ void __launch_bounds__(kWideThreads) wide_backward_kernel(const __grid_constant__ Params p) {
    __shared__ float slots[32];
    extern __shared__ float4 wide_sums[];
    const int threads = blockDim.x;
    grid_dependency_wait();
    if (kSums) {
        for (int64_t c0 = 0, q = 0; c0 < p.cols; c0 += 8 * threads)
            for (int i = 0; i < 4; ++i, ++q) wide_sums[q * threads + threadIdx.x] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const T *x = static_cast<const T*>(p.x) + row * p.ldx, *dy = static_cast<const T*>(p.dy) + row * p.lddy;
        T* dx = static_cast<T*>(p.dx) + row * p.ldy;
        const float mean = p.mean_in[row], rstd = p.rstd_in[row];
        float s0 = 0.0f, s1 = 0.0f, v[8], g[8], gamma[8];
        const auto take = [&](const Cols<kVec>& c, float4* sums) {
            c.load(x, v);
            c.load(dy, g);
            load_affine(c, p.gamma, p.affine_bf16, 1.0f, gamma);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = j < c.count ? (v[j] - mean) * rstd : 0.0f;
            if (kSums && sums) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float4 &a = sums[h * threads], &b = sums[(2 + h) * threads];
                    a = make_float4(fmaf(g[4 * h], v[4 * h], a.x), fmaf(g[4 * h + 1], v[4 * h + 1], a.y), fmaf(g[4 * h + 2], v[4 * h + 2], a.z),
                                    fmaf(g[4 * h + 3], v[4 * h + 3], a.w));
                    b = make_float4(b.x + g[4 * h], b.y + g[4 * h + 1], b.z + g[4 * h + 2], b.w + g[4 * h + 3]);
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] *= gamma[j];
        };
        int64_t slab = 0;
        for (int64_t c0 = 0; c0 < p.cols; c0 += 8 * threads, ++slab) {
            const Cols<kVec> c(c0, p.cols, threadIdx.x, threads);
            if (c.count == 0) break;
            take(c, wide_sums + slab * 4 * threads + threadIdx.x);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < c.count) {
                    s0 += g[j];
                    s1 = fmaf(g[j], v[j], s1);
                }
        }
        const float m0 = block_sum(s0, slots) * p.inv_cols, m1 = block_sum(s1, slots) * p.inv_cols;
        for (int64_t c0 = 0; c0 < p.cols; c0 += 8 * threads) {
            const Cols<kVec> c(c0, p.cols, threadIdx.x, threads);
            if (c.count == 0) break;
            take(c, nullptr);
#pragma unroll
            for (int j = 0; j < 8; ++j) g[j] = rstd * (g[j] - fmaf(v[j], m1, m0));
            c.store(dx, g);
        }
    }
    if (kSums) {
        float* out = p.partial + (int64_t)blockIdx.x * 2 * p.cols;
        int64_t slab = 0;
        for (int64_t c0 = 0; c0 < p.cols; c0 += 8 * threads, ++slab) {
            const Cols<kVec> c(c0, p.cols, threadIdx.x, threads);
            if (c.count == 0) break;
            const float4* sums = wide_sums + slab * 4 * threads + threadIdx.x;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float4 a = sums[h * threads], b = sums[(2 + h) * threads];
                const float x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (4 * h + j < c.count) {
                        out[c.at(4 * h + j)] = x[j];
                        out[p.cols + c.at(4 * h + j)] = y[j];
                    }
            }
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
// Which kernel: `eight` where every access is of eight elements (forward: and a row whole pieces of a team) and there are rows enough to
// fill the device with them; wide where a row does not fit the threads of a block; else the one for any alignment.
struct Plan {
    enum Kind { kAny, kEight, kWide } kind;
    bool full;                                // kEight, backward: the team covers a row exactly
    int pieces, at_once;                      // kEight: pieces of eight columns per thread; rows at once
    int team, teams, blocks;                  // kWide: blocks of rows
    int parts;                                // partial sums of the backward pass
    dim3 columns;                             // kWide: grid of the column sums
};
int round_up(int64_t x, int to) { return (int)((x + to - 1) / to * to); }

Plan plan(bool backward, int64_t rows, int64_t cols, int dtype, int vec, int sm_count) {
    Plan q = {};
    if (vec == 8 && !backward && cols % 256 == 0 && cols <= 32 * kEightThreads) {
        // bf16 two rows of two pieces of eight, fp32 two rows of one, where the columns allow it
        const int64_t eights = cols / 256, most = kEightThreads / 32;
        const int room = dtype == MVUE_BF16 ? 4 : 2;
        q.pieces = eights <= most && (room == 2 || eights % 2 != 0) ? 1 : eights <= 2 * most ? 2 : 4;
        q.at_once = std::max(1, room / q.pieces);
        q.team = (int)(eights / q.pieces * 32);
        q.teams = std::max(1, 512 / q.team);
        const int64_t per_block = (int64_t)q.teams * q.at_once, blocks = (rows + per_block - 1) / per_block;
        if (eights % q.pieces == 0 && blocks >= sm_count) {
            q.kind = Plan::kEight;
            q.blocks = (int)std::min<int64_t>(blocks, (int64_t)sm_count);
            return q;
        }
    }
    if (vec == 8 && backward && cols <= 16 * kEightThreads) {
        const int room = dtype == MVUE_BF16 ? 2 : 1;                       // pieces of two tensors that the registers have room for
        q.pieces = cols > 8 * kEightThreads || (room == 2 && cols > 2048 && cols % 512 == 0) ? 2 : 1;
        q.at_once = std::max(1, room / q.pieces);
        q.team = round_up((cols + 8 * q.pieces - 1) / (8 * q.pieces), 32);
        q.teams = std::max(1, 512 / q.team);
        q.full = (int64_t)q.team * 8 * q.pieces == cols;
        const int64_t per_block = (int64_t)q.teams * q.at_once, blocks = (rows + per_block - 1) / per_block;
        if (blocks >= sm_count) {
            q.kind = Plan::kEight;
            q.blocks = q.parts = sm_count;
            return q;
        }
    }
    if (cols > 8 * kMaxTeam) {
        q.kind = Plan::kWide;
        // blocks of 256 threads, eight an SM: several rows on their way at once (3387 x 4984 bf16 forward: 55 us with two of 1024)
        q.team = 256;
        q.blocks = (int)std::min<int64_t>(rows, 8 * (int64_t)sm_count);
        if (backward && cols <= kWideSums) {
            // as many blocks as have room for their sums
            const int fit = std::min(8, (int)(kWideSums / round_up(cols, 2048)));
            q.team = fit >= 4 ? 256 : fit >= 2 ? 512 : 1024;
            q.blocks = q.parts = (int)std::min<int64_t>(rows, (int64_t)fit * sm_count);
            return q;
        }
        const int64_t slabs = (cols + 255) / 256;
        q.parts = (int)std::max<int64_t>(1, std::min<int64_t>((rows + 4 * kColumnRows - 1) / (4 * kColumnRows), 8 * (int64_t)sm_count / slabs));
        q.columns = dim3((unsigned)slabs, (unsigned)q.parts);
        return q;
    }
    q.kind = Plan::kAny;
    q.team = round_up((cols + (vec == kShifted ? 14 : 7)) / 8, 32);
    q.teams = std::max(1, 512 / q.team);
    q.at_once = backward ? 2 : rows >= (int64_t)4 * q.teams * sm_count ? 4 : 1;
    if (q.at_once == 1) q.teams = 1;
    const int64_t per_block = (int64_t)q.teams * q.at_once;
    const int64_t most = (int64_t)sm_count * std::max(1, (backward ? 512 : 1024) / (q.team * q.teams));
    if (vec == kShifted) q.blocks = (int)(8 * std::min<int64_t>((rows + 8 * per_block - 1) / (8 * per_block), std::max<int64_t>(1, most / 8)));
    else q.blocks = (int)std::min<int64_t>((rows + per_block - 1) / per_block, most);
    q.parts = q.blocks;
    return q;
}

template <typename K> cudaError_t roomy(PerDeviceOnce& once, K kernel) {
    return once_per_device(once, [&](int) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 8 * kEightThreads * 4 * 8); });
}
template <typename T, int kC, int kR> cudaError_t forward8(const Plan& q, const Params& p, cudaStream_t st) {
    static PerDeviceOnce once;
    if (cudaError_t e = roomy(once, &forward8_kernel<T, kC, kR>)) return e;
    return launch_dependent(&forward8_kernel<T, kC, kR>, dim3(q.blocks), dim3(q.team, q.teams), (size_t)p.cols * 8, st, p);
}
template <typename T, int kC, int kR, bool kSums, bool kFull> cudaError_t backward8(const Plan& q, const Params& p, cudaStream_t st) {
    static PerDeviceOnce once;
    if (cudaError_t e = roomy(once, &backward8_kernel<T, kC, kR, kSums, kFull>)) return e;
    const size_t joined = kSums && q.teams > 1 ? (size_t)q.team * 16 * kC * 4 : 0;
    return launch_dependent(&backward8_kernel<T, kC, kR, kSums, kFull>, dim3(q.blocks), dim3(q.team, q.teams), std::max((size_t)p.cols * 4, joined), st, p);
}

template <typename T, int kVec> cudaError_t forward(const Plan& q, const Params& p, cudaStream_t st) {
    if constexpr (kVec == 8) {
        if (q.kind == Plan::kEight) {
            constexpr int kRoom = sizeof(T) == 2 ? 4 : 2;
            return q.pieces == 1   ? forward8<T, 1, kRoom>(q, p, st)
                   : q.pieces == 2 ? forward8<T, 2, kRoom / 2>(q, p, st)
                                   : forward8<T, 4, 1>(q, p, st);
        }
    }
    if constexpr (kVec != kShifted)
        if (q.kind == Plan::kWide) return launch_dependent(&wide_forward_kernel<T, kVec>, dim3(q.blocks), dim3(q.team), 0, st, p);
    const dim3 block(q.team, q.teams);
    if (q.at_once == 4) return launch_dependent(&forward_kernel<T, kVec, 4>, dim3(q.blocks), block, 0, st, p);
    return launch_dependent(&forward_kernel<T, kVec, 1>, dim3(q.blocks), block, 0, st, p);
}
template <typename T, int kVec, bool kSums> cudaError_t backward(const Plan& q, const Params& p, cudaStream_t st) {
    if constexpr (kVec == 8) {
        if (q.kind == Plan::kEight) {
            constexpr int kRoom = sizeof(T) == 2 ? 2 : 1;
            if (q.full) return q.pieces == 1 ? backward8<T, 1, kRoom, kSums, true>(q, p, st) : backward8<T, 2, 1, kSums, true>(q, p, st);
            return q.pieces == 1 ? backward8<T, 1, kRoom, kSums, false>(q, p, st) : backward8<T, 2, 1, kSums, false>(q, p, st);
        }
    }
    if constexpr (kVec != kShifted) {
    if (q.kind == Plan::kWide) {
        if (kSums && p.cols <= kWideSums) {
            static PerDeviceOnce once;
            const cudaError_t e = once_per_device(once, [](int) {
                return cudaFuncSetAttribute(&wide_backward_kernel<T, kVec, kSums>, cudaFuncAttributeMaxDynamicSharedMemorySize, 8 * kWideSums);
            });
            if (e != cudaSuccess) return e;
            return launch_dependent(&wide_backward_kernel<T, kVec, kSums>, dim3(q.blocks), dim3(q.team), (size_t)round_up(p.cols, 8 * q.team) * 8, st, p);
        }
        cudaError_t e = cudaSuccess;
        if (kSums) e = launch_dependent(&wide_column_kernel<T, kVec>, q.columns, dim3(32, kColumnRows), 0, st, p);
        if (e != cudaSuccess) return e;
        return launch_dependent(&wide_backward_kernel<T, kVec, false>, dim3(q.blocks), dim3(q.team), 0, st, p);
    }
    }
    return launch_dependent(&backward_kernel<T, kVec, kSums>, dim3(q.blocks), dim3(q.team, q.teams), kSums && q.teams > 1 ? q.team * 64 : 0, st, p);
}
// whether the rows of all tensors begin at the same distance from an aligned address, and the pieces fit a block's threads
bool shifts_alike(const void* a, int64_t lda, const void* b, int64_t ldb, int64_t rows, int dtype) {
    const uint64_t size = (uint64_t)size_of(dtype), pa = reinterpret_cast<uintptr_t>(a) / size, pb = reinterpret_cast<uintptr_t>(b) / size;
    return (pa - pb) % 8 == 0 && (rows == 1 || (lda - ldb) % 8 == 0);
}
bool shifted_fits(int64_t cols, int dtype) { return dtype == MVUE_BF16 && cols >= 16 && (cols + 14) / 8 <= kMaxTeam; }
int widest(int v, const void* p, int64_t ld, int64_t cols, int64_t rows, int dtype) { return std::min(v, row_vector(p, rows > 1 ? ld : cols, cols, dtype)); }

// enough for any alignment and type
size_t workspace_bytes_of(int64_t rows, int64_t cols, int sm_count) {
    int parts = 0;
    for (const int dtype : {MVUE_F32, MVUE_BF16})
        for (const int vec : {8, 1, kShifted})
            if (vec != kShifted || shifted_fits(cols, dtype)) parts = std::max(parts, plan(true, rows, cols, dtype, vec, sm_count).parts);
    return (size_t)parts * 2 * (size_t)cols * sizeof(float);
}

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
    int v = widest(widest(8, x, ldx, cols, rows, dtype), y, ldy, cols, rows, dtype);
    if (v < 8 && shifted_fits(cols, dtype) && shifts_alike(x, ldx, y, ldy, rows, dtype)) v = kShifted;
    const Plan q = plan(false, rows, cols, dtype, v, dev.sm_count);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const auto pick = [&](auto t) {
        using T = decltype(t);
        if constexpr (std::is_same<T, __nv_bfloat16>::value)
            if (v == kShifted) return forward<T, kShifted>(q, p, st);
        return v == 8 ? forward<T, 8>(q, p, st) : v == 2 ? forward<T, 2>(q, p, st) : forward<T, 1>(q, p, st);
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
    int v = widest(widest(widest(8, x, ldx, cols, rows, dtype), dy, lddy, cols, rows, dtype), dx, lddx, cols, rows, dtype);
    if (v < 8 && shifted_fits(cols, dtype) && shifts_alike(x, ldx, dy, lddy, rows, dtype) && shifts_alike(x, ldx, dx, lddx, rows, dtype)) v = kShifted;
    const Plan q = plan(true, rows, cols, dtype, v, dev.sm_count);
    const auto pick = [&](auto t) {
        using T = decltype(t);
        const auto go = [&](auto s) {
            constexpr bool kSums = decltype(s)::value;
            if constexpr (std::is_same<T, __nv_bfloat16>::value)
                if (v == kShifted) return backward<T, kShifted, kSums>(q, p, st);
            return v == 8 ? backward<T, 8, kSums>(q, p, st) : v == 2 ? backward<T, 2, kSums>(q, p, st) : backward<T, 1, kSums>(q, p, st);
        };
        return sums ? go(std::true_type()) : go(std::false_type());
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
