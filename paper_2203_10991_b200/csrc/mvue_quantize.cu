// e4m3 codes with a power-of-two scale for each block of 1 x 128 or 128 x 128 elements: what the products of mvue_scaled.cu take.
//
// Bytes: one pass, the input read once and one byte per element written; a block's elements wait in registers for its largest
// magnitude.  Sixteen lanes of eight neighbours each hold 128 columns.  The scale is a power of two, so dividing by it is
// exact and both roundings act on the element itself.
// Rounding at random: the element over its scale, times 2^-120, has its binary32 subnormals where e4m3 has its own, so the
// code is the upper bits of the bit pattern for subnormal, normal and zero alike; adding a random number to the 16 bits below
// them carries into them as often as the element is nearer to its upper neighbour.
// 16384 x 14336 bf16: to the nearest 117 us (6.0 of 6.46 TB/s copy), at random 197 to 202 us: the generator's ten rounds for every eight elements
// (74 us alone) and the rounding fill the issue slots (71 %), not memory.  14336 x 4096 in blocks of 128 x 128: 29 us (6.0 TB/s).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "../../include/mvue_layer.h"
#include "mvue_device.cuh"
#include "mvue_internal.h"
#include "mvue_train.cuh"

namespace mvue {
namespace {

constexpr int kThreads = 256;
constexpr int kRowsPerWarp = 4;                       // 1 x 128: rows of a warp, two blocks each
constexpr uint32_t kInf = 0x7F800000u;

struct Params {
    const void* x;
    int64_t rows, cols, ldx;
    uint8_t* codes;
    int64_t ldq;
    uint8_t* scales;
    int64_t scale_pitch;       // 1 x 128: bytes from one block of columns to the next (rows); 128 x 128: from one block of rows
    int64_t units;             // ceil(cols / 8): generator calls of a row
    bool wide_x, wide_q;       // eight elements, eight codes in one access
    int64_t tiles_x;
    RoundKeys keys;
};

// Eight elements of a lane as they were read.
template <typename T> struct Eight;
template <> struct Eight<__nv_bfloat16> {
    uint32_t w[4];
    __device__ __forceinline__ void load(const __nv_bfloat16* p, bool wide, int count) {
        if (wide && count == 8) {
            const uint4 v = *reinterpret_cast<const uint4*>(p);
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        } else {
            const unsigned short* q = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[i] = (2 * i < count ? (uint32_t)q[2 * i] : 0u) | (2 * i + 1 < count ? (uint32_t)q[2 * i + 1] << 16 : 0u);
        }
    }
    __device__ __forceinline__ float at(int i) const { return i & 1 ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]); }
    // upper halves of the magnitudes, two neighbours' largest in each half of the word
    __device__ __forceinline__ uint32_t tops() const {
        uint32_t m = w[0] & 0x7FFF7FFFu;
#pragma unroll
        for (int i = 1; i < 4; ++i) m = __vmaxu2(m, w[i] & 0x7FFF7FFFu);
        return m;
    }
    // bit pattern of the largest magnitude (as binary32); an infinity or a NaN is above all others
    __device__ __forceinline__ uint32_t top() const {
        const uint32_t m = tops();
        return max(m << 16, m & 0xFFFF0000u);
    }
    __device__ __forceinline__ uint32_t signs(int h) const { return __byte_perm(w[2 * h], w[2 * h + 1], 0x7531); }      // bit 7 of each byte
};
template <> struct Eight<float> {
    uint32_t w[8];
    __device__ __forceinline__ void load(const float* p, bool wide, int count) {
        if (wide && count == 8) {
            ld256(p, w);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = i < count ? __float_as_uint(p[i]) : 0u;
        }
    }
    __device__ __forceinline__ float at(int i) const { return __uint_as_float(w[i]); }
    __device__ __forceinline__ uint32_t top() const {
        uint32_t m = 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, w[i] & 0x7FFFFFFFu);
        return m;
    }
    __device__ __forceinline__ uint32_t signs(int h) const {
        return __byte_perm(__byte_perm(w[4 * h], w[4 * h + 1], 0x0073), __byte_perm(w[4 * h + 2], w[4 * h + 3], 0x0073), 0x5410);
    }
};

// The largest magnitudes of the blocks that kRows rows have in a lane's sixteen lanes.  bf16: two rows share a word.
template <typename T, int kRows>
__device__ __forceinline__ void block_tops(const Eight<T> (&x)[kRows], uint32_t (&top)[kRows]) {
    if constexpr (sizeof(T) == 2 && kRows % 2 == 0) {
#pragma unroll
        for (int r = 0; r < kRows; r += 2) {
            const uint32_t a = x[r].tops(), b = x[r + 1].tops();
            uint32_t m = __vmaxu2(__byte_perm(a, b, 0x5410), __byte_perm(a, b, 0x7632));
#pragma unroll
            for (int d = 8; d > 0; d >>= 1) m = __vmaxu2(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
            top[r] = m << 16;
            top[r + 1] = m & 0xFFFF0000u;
        }
    } else {
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            top[r] = x[r].top();
#pragma unroll
            for (int d = 8; d > 0; d >>= 1) top[r] = max(top[r], __shfl_xor_sync(0xFFFFFFFFu, top[r], d));
        }
    }
}

// the largest finite magnitude: where top() met something else
template <typename T> __device__ __forceinline__ uint32_t finite_top(const Eight<T>& x) {
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t b = __float_as_uint(x.at(i)) & 0x7FFFFFFFu;
        if (b < kInf) m = max(m, b);
    }
    return m;
}

// Exponent byte of the least power of two, 2^-126 or above, that brings the magnitude with these bits to 448 = 1.75 2^8 or less.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    return (uint32_t)max((int)(top >> 23) - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0), 1);
}

// NaN codes for elements that have none other.
template <typename T> __device__ __forceinline__ void put_nan(const Eight<T>& x, uint2& v) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t bits = __float_as_uint(x.at(i)), at = 8 * (i & 3);
        uint32_t& w = i < 4 ? v.x : v.y;
        if ((bits & 0x7FFFFFFFu) >= kInf) w = (w & ~(0xFFu << at)) | ((0x7Fu | bits >> 24 & 0x80u) << at);
    }
}

// Four codes rounded at random: y = the elements over their scale, times 2^-120.  The code fills the highest byte of the bits four
// places up, the sign falls out, the random number is below it.
__device__ __forceinline__ uint32_t random_codes(f2 y0, f2 y1, uint32_t r0, uint32_t r1) {
    float y[4];
    unpair(y0, y[0], y[1]);
    unpair(y1, y[2], y[3]);
    const uint32_t t0 = (__float_as_uint(y[0]) << 4) + __byte_perm(r0, 0u, 0x4104), t1 = (__float_as_uint(y[1]) << 4) + __byte_perm(r0, 0u, 0x4324);
    const uint32_t t2 = (__float_as_uint(y[2]) << 4) + __byte_perm(r1, 0u, 0x4104), t3 = (__float_as_uint(y[3]) << 4) + __byte_perm(r1, 0u, 0x4324);
    return __byte_perm(__byte_perm(t0, t1, 0x0073), __byte_perm(t2, t3, 0x0073), 0x5410);
}

template <typename T, bool kRandom>
__device__ __forceinline__ uint2 encode(const Eight<T>& x, uint32_t byte, uint4 random) {
    uint32_t out[2];
    if constexpr (kRandom) {
        const uint32_t rw[4] = {random.x, random.y, random.z, random.w};
        // 2^(7 - byte) in one product where that is a normal number (blocks of magnitudes up to 2^14), else in two
        const bool one = byte <= 133u;
        const f2 first = pair(__uint_as_float(one ? (134u - byte) << 23 : (254u - byte) << 23)), second = pair(7.52316384526264005e-37f);       // 2^-120
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            f2 y0 = mul2(pair(x.at(4 * h), x.at(4 * h + 1)), first), y1 = mul2(pair(x.at(4 * h + 2), x.at(4 * h + 3)), first);
            if (!one) {
                y0 = mul2(y0, second);
                y1 = mul2(y1, second);
            }
            out[h] = random_codes(y0, y1, rw[2 * h], rw[2 * h + 1]) | (x.signs(h) & 0x80808080u);
        }
    } else {
        const f2 factor = pair(__uint_as_float((254u - byte) << 23));          // 2^(127 - byte)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t half[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float lo, hi;
                unpair(mul2(pair(x.at(4 * h + 2 * j), x.at(4 * h + 2 * j + 1)), factor), lo, hi);
                asm("{\n\t.reg .b16 c;\n\tcvt.rn.satfinite.e4m3x2.f32 c, %1, %2;\n\tcvt.u32.u16 %0, c;\n\t}" : "=r"(half[j]) : "f"(hi), "f"(lo));
            }
            out[h] = __byte_perm(half[0], half[1], 0x5410);
        }
    }
    return make_uint2(out[0], out[1]);
}

__device__ __forceinline__ void store_codes(uint8_t* to, bool wide, int count, uint2 v) {
    if (wide && count == 8) {
        *reinterpret_cast<uint2*>(to) = v;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < count) to[i] = (uint8_t)((i < 4 ? v.x : v.y) >> (8 * (i & 3)));
    }
}

// 1 x 128: a warp takes two blocks (256 columns) of kRowsPerWarp rows, a thread block 32 rows.  16384 x 14336 at random: 197 us; two rows
// a warp 214 us, eight 246 us, four with four blocks an SM instead of five 203 us.
template <typename T, bool kRandom>
__global__ void __launch_bounds__(kThreads, 5) quantize_rows_kernel(const __grid_constant__ Params p) {
    grid_dependency_wait();
    const int lane = threadIdx.x & 31;
    const int64_t tile_y = blockIdx.x / p.tiles_x, tile_x = blockIdx.x - tile_y * p.tiles_x;
    const int64_t row0 = (tile_y * (kThreads / 32) + (threadIdx.x >> 5)) * kRowsPerWarp, col = tile_x * 256 + lane * 8;
    const int count = (int)min((int64_t)8, max((int64_t)0, p.cols - col));
    Eight<T> x[kRowsPerWarp];
#pragma unroll
    for (int r = 0; r < kRowsPerWarp; ++r)
        x[r].load(static_cast<const T*>(p.x) + (row0 + r) * p.ldx + col, p.wide_x, row0 + r < p.rows ? count : 0);
    uint32_t top[kRowsPerWarp];
    block_tops(x, top);
    uint8_t* to = p.codes + row0 * p.ldq + col;
    uint8_t* scale = p.scales + (col >> 7) * p.scale_pitch + row0;
    uint64_t unit = (uint64_t)(row0 * p.units + (col >> 3));
#pragma unroll
    for (int r = 0; r < kRowsPerWarp; ++r, to += p.ldq, unit += (uint64_t)p.units) {
        if (row0 + r >= p.rows) return;                                       // a whole warp
        const bool finite = __all_sync(0xFFFFFFFFu, top[r] < kInf);           // (the branches below are the warp's, and rarely taken)
        if (!finite) {
            top[r] = finite_top(x[r]);
#pragma unroll
            for (int d = 8; d > 0; d >>= 1) top[r] = max(top[r], __shfl_xor_sync(0xFFFFFFFFu, top[r], d));
        }
        const uint32_t byte = scale_byte(top[r]);
        uint4 random = make_uint4(0u, 0u, 0u, 0u);
        if (kRandom) random = philox4x32_10(unit, p.keys, 3u);
        uint2 v = encode<T, kRandom>(x[r], byte, random);
        if (!finite) put_nan(x[r], v);
        store_codes(to, p.wide_q, count, v);
        if ((lane & 15) == 0 && count > 0) scale[r] = (uint8_t)byte;
    }
}

// 128 x 128: a thread block takes one, a thread eight rows of eight columns.
template <typename T, bool kRandom>
__global__ void __launch_bounds__(kThreads) quantize_tiles_kernel(const __grid_constant__ Params p) {
    grid_dependency_wait();
    __shared__ uint32_t tops[kThreads / 32];
    const int64_t tile_y = blockIdx.x / p.tiles_x, tile_x = blockIdx.x - tile_y * p.tiles_x;
    const int64_t row0 = tile_y * 128 + (threadIdx.x >> 4), col = tile_x * 128 + (threadIdx.x & 15) * 8;
    const int count = (int)min((int64_t)8, max((int64_t)0, p.cols - col));
    Eight<T> x[8];
#pragma unroll
    for (int r = 0; r < 8; ++r)
        x[r].load(static_cast<const T*>(p.x) + (row0 + 16 * r) * p.ldx + col, p.wide_x, row0 + 16 * r < p.rows ? count : 0);
    uint32_t top = 0u;
#pragma unroll
    for (int r = 0; r < 8; ++r) top = max(top, x[r].top());
    top = __reduce_max_sync(0xFFFFFFFFu, top);
    const bool finite = top < kInf;                                           // of the warp
    if (!finite) {
        top = 0u;
#pragma unroll
        for (int r = 0; r < 8; ++r) top = max(top, finite_top(x[r]));
        top = __reduce_max_sync(0xFFFFFFFFu, top);
    }
    if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kThreads / 32; ++i) top = max(top, tops[i]);
    const uint32_t byte = scale_byte(top);
    uint8_t* to = p.codes + row0 * p.ldq + col;
    uint64_t unit = (uint64_t)(row0 * p.units + (col >> 3));
#pragma unroll
    for (int r = 0; r < 8; ++r, to += 16 * p.ldq, unit += 16 * (uint64_t)p.units) {
        if (row0 + 16 * r >= p.rows) break;
        uint4 random = make_uint4(0u, 0u, 0u, 0u);
        if (kRandom) random = philox4x32_10(unit, p.keys, 3u);
        uint2 v = encode<T, kRandom>(x[r], byte, random);
        if (!finite) put_nan(x[r], v);
        store_codes(to, p.wide_q, count, v);
    }
    if (threadIdx.x == 0) p.scales[tile_y * p.scale_pitch + tile_x] = (uint8_t)byte;
}

}  // namespace
}  // namespace mvue

using namespace mvue;

extern "C" int mvue_quantize_e4m3(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ldx, int block_rows, unsigned options,
                                  uint64_t seed, void* codes, int64_t ldq, void* scales, void* stream) {
    if (dtype != MVUE_F32 && dtype != MVUE_BF16) return MVUE_ERR_DTYPE;
    if (options & ~(unsigned)MVUE_OPT_STOCHASTIC_ROUNDING) return MVUE_ERR_OPTION;
    if ((block_rows != 1 && block_rows != MVUE_SCALE_BLOCK) || rows < 0 || cols < 0 || ldx < cols || ldq < cols) return MVUE_ERR_SHAPE;
    if (rows == 0 || cols == 0) return MVUE_OK;
    if (!x || !codes || !scales) return MVUE_ERR_NULL;
    if (off(x, size_of(dtype))) return MVUE_ERR_ALIGN;
    const bool random = (options & MVUE_OPT_STOCHASTIC_ROUNDING) != 0;
    Params p;
    p.x = x; p.rows = rows; p.cols = cols; p.ldx = ldx;
    p.codes = static_cast<uint8_t*>(codes); p.ldq = ldq;
    p.scales = static_cast<uint8_t*>(scales);
    p.units = (cols + 7) / 8;
    p.wide_x = !off(x, 8 * size_of(dtype)) && (ldx % 8 == 0 || rows == 1);
    p.wide_q = !off(codes, 8) && (ldq % 8 == 0 || rows == 1);
    p.keys = make_round_keys(seed);
    const int width = block_rows == 1 ? 256 : 128, height = block_rows == 1 ? kThreads / 32 * kRowsPerWarp : 128;
    p.tiles_x = (cols + width - 1) / width;
    p.scale_pitch = block_rows == 1 ? rows : p.tiles_x;
    const int64_t tiles_y = (rows + height - 1) / height;
    if (tiles_y > 0x7FFFFFFF / p.tiles_x) return MVUE_ERR_SHAPE;
    DeviceInfo dev;
    if (int s = current_device_info(&dev)) return s;
    using Kernel = void (*)(Params);
    const Kernel kernels[2][2][2] = {{{quantize_rows_kernel<float, false>, quantize_rows_kernel<float, true>},
                                      {quantize_rows_kernel<__nv_bfloat16, false>, quantize_rows_kernel<__nv_bfloat16, true>}},
                                     {{quantize_tiles_kernel<float, false>, quantize_tiles_kernel<float, true>},
                                      {quantize_tiles_kernel<__nv_bfloat16, false>, quantize_tiles_kernel<__nv_bfloat16, true>}}};
    const cudaError_t e = launch_dependent(kernels[block_rows != 1][dtype == MVUE_BF16][random], dim3((unsigned)(tiles_y * p.tiles_x)), dim3(kThreads),
                                           0, reinterpret_cast<cudaStream_t>(stream), p);
    if (e != cudaSuccess) { set_cuda_error(e, "mvue_quantize_e4m3 launch"); return MVUE_ERR_CUDA; }
    return MVUE_OK;
}
