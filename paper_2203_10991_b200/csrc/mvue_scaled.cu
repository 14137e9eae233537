// Dense products in 8-bit floating point with block scales: the forward product of a layer, C = x W^T, and its backward
// product, C = g W.
//
// 16384 x 14336 x 4096 bf16 out: 0.80 ms in a short run, 2.4 PFLOP/s, and 0.92 ms, 2.1 PFLOP/s, in a long one, where the power limit holds: 1.44
// and 1.48 times the rate of a large bf16 library product in the same state.  The tensor pipe is active 63 % of the time and waits for
// operands from L2: a pair's 256 x 256 tiles want 9 TB/s of them.  Stores take 6 %, the hand-over between tiles 1 %.
// 32768 x 1024 from 4096 outs, backward: 0.12 and 0.14 ms, 2.3 and 2.0 PFLOP/s.
// 8 x 14336 x 4096: 13.3 us in a graph, the weights at 4.4 TB/s; 14.0 to 14.4 us by calls from Python.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "../../include/mvue_layer.h"
#include "mvue_dense.cuh"
#include "mvue_few.cuh"
#include "mvue_train.cuh"

namespace mvue {
namespace {

// A 32 x 32 block of words turned over among the lanes: word i of lane l becomes word l of lane i.
__device__ __forceinline__ void turn_over(uint32_t (&v)[32], int lane) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        const bool up = (lane & d) != 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            if (i & d) continue;
            const uint32_t got = __shfl_xor_sync(0xFFFFFFFFu, up ? v[i] : v[i + d], d);
            if (up) v[i] = got;
            else v[i + d] = got;
        }
    }
}

// 32 consecutive results of a row; rows that do not allow wide accesses are turned over first, so that a warp's stores are neighbours.
template <bool kBf16>
struct Store {
    void* C;
    int64_t ldc;
    int vec;                                 // bytes that one access may take: 32, 16, or an element
    using Maps = dense::NoMaps;
    static constexpr bool kSlabs = false;
    __device__ __forceinline__ void store(const dense::Params& p, int row, int col, const uint32_t (&v)[32]) const {
        if (col >= p.N) return;                              // (a whole warp)
        const int left = p.N - col;
        if (vec < 16 || left < 32) {
            const int lane = threadIdx.x & 31, rows = p.M - (row - lane);
            uint32_t w[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) w[i] = v[i];
            turn_over(w, lane);
            if (lane >= left) return;
            const int64_t at = (int64_t)(row - lane) * ldc + col + lane;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                if (i >= rows) break;
                if constexpr (kBf16) static_cast<__nv_bfloat16*>(C)[at + i * ldc] = __float2bfloat16_rn(__uint_as_float(w[i]));
                else static_cast<float*>(C)[at + i * ldc] = __uint_as_float(w[i]);
            }
            return;
        }
        if (row >= p.M) return;
        if constexpr (kBf16) {
            __nv_bfloat16* to = static_cast<__nv_bfloat16*>(C) + (int64_t)row * ldc + col;
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = pack_bf16x2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1]));
            if (vec == 32) {
                store8_b32(to, w);
                store8_b32(to + 16, w + 8);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) reinterpret_cast<uint4*>(to)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
            }
        } else {
            float* to = static_cast<float*>(C) + (int64_t)row * ldc + col;
#pragma unroll
            for (int i = 0; i < 32; i += 8) store8_b32(to + i, v + i);
        }
    }
};

template <bool kBf16>
cudaError_t launch(const dense::Params& p, const dense::Operand& a, const dense::Operand& b, bool n_major, const Store<kBf16>& out, cudaStream_t stream) {
    if (n_major) return dense::launch_pair<dense::Shape<true, true, 6>>(p, a, b, {}, out, stream);
    return dense::launch_pair<dense::Shape<true, false, 6>>(p, a, b, {}, out, stream);
}

template <int kTN> cudaError_t launch_few(const dense::FewParams& p, const dense::Operand& t, const dense::Operand& w, bool n_major, cudaStream_t stream) {
    return n_major ? dense::launch_few<dense::FewShape<true, kTN>>(p, t, w, stream) : dense::launch_few<dense::FewShape<false, kTN>>(p, t, w, stream);
}

// Tiles of 128 outs and a cluster along the reduction where a token tile of the pair kernel would be half empty or its tiles would leave
// most SMs without work (256 x 4096 x 4096: 16 us against 20 us, 300 x 700 x 9000: 18 us against 68 us; 1000 x 4096 x 4096 22 us
// against 21 us, which stays with the pairs).
bool few(int64_t tokens, int64_t pair_tiles, int sm_count) { return tokens <= 128 || 8 * pair_tiles < 3 * sm_count; }

int scaled_gemm(const void* a, int64_t M, int64_t K, int64_t lda, const void* a_scales, const void* w, int64_t N, int64_t ldw,
                const void* w_scales, bool n_major, void* C, int c_dtype, int64_t ldc, int* dev_status, void* stream) {
    if (c_dtype != MVUE_F32 && c_dtype != MVUE_BF16) return MVUE_ERR_DTYPE;
    if (M < 0 || N <= 0 || K <= 0 || M > 0x7FFFFF00 || N > 0x7FFFFF00 || K > 0x7FFFFF00) return MVUE_ERR_SHAPE;
    if (lda < K || ldw < (n_major ? N : K) || ldc < N) return MVUE_ERR_SHAPE;
    if (!w || !w_scales || (M > 0 && (!a || !a_scales || !C))) return MVUE_ERR_NULL;
    if (off(a, 16) || off(w, 16) || lda % 16 != 0 || ldw % 16 != 0 || off(C, size_of(c_dtype))) return MVUE_ERR_ALIGN;
    if (M == 0) return MVUE_OK;
    DeviceInfo dev;
    if (int s = current_device_info(&dev)) return s;
    const dense::Operand oa = {a, lda, lda * M}, ob = {w, ldw, ldw * (n_major ? K : N)};
    const int64_t pitch = ldc * size_of(c_dtype);
    const int vec = !off(C, 32) && pitch % 32 == 0 ? 32 : !off(C, 16) && pitch % 16 == 0 ? 16 : (int)size_of(c_dtype);
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const int64_t blocks_n = (N + 127) / 128, blocks_k = (K + 127) / 128;
    const int64_t scales_n = n_major ? 1 : blocks_k, scales_k = n_major ? blocks_n : 1;
    const uint8_t *as = static_cast<const uint8_t*>(a_scales), *ws = static_cast<const uint8_t*>(w_scales);
    cudaError_t e;
    const int64_t pair_tiles = ((M + 255) / 256) * ((N + 255) / 256);
    if (few(M, pair_tiles, dev.sm_count)) {
        dense::FewParams p = {};
        p.tokens = (int)M; p.outs = (int)N; p.K = (int)K;
        p.tiles_o = (int)blocks_n;
        p.t_scales = as; p.w_scales = ws; p.w_scales_o = scales_n; p.w_scales_k = scales_k;
        p.C = C; p.ldc = ldc; p.bf16 = c_dtype == MVUE_BF16; p.vec = vec >= 16 ? 16 : 1;
        p.dev_status = dev_status;
        const int tn = M <= 16 ? 16 : M <= 64 ? 64 : 128;
        const int64_t tiles = blocks_n * ((M + tn - 1) / tn);
        // as many parts as two blocks an SM have room for, of eight steps at least (128 x 4096 x 4096: 11 us, 18 us with parts of four)
        p.split = 1;
        while (p.split < dense::kMaxSplit && tiles * p.split * 2 <= 2 * (int64_t)dev.sm_count && blocks_k >= 16 * p.split) p.split *= 2;
        p.steps_per_part = (int)((blocks_k + p.split - 1) / p.split);
        e = tn == 16 ? launch_few<16>(p, oa, ob, n_major, st) : tn == 64 ? launch_few<64>(p, oa, ob, n_major, st) : launch_few<128>(p, oa, ob, n_major, st);
    } else {
        dense::Params p = {};
        p.M = (int)M; p.N = (int)N; p.K = (int)K; p.batch = 1;
        p.a_scales = as; p.b_scales = ws; p.b_scales_n = scales_n; p.b_scales_k = scales_k;
        p.dev_status = dev_status;
        e = c_dtype == MVUE_BF16 ? launch(p, oa, ob, n_major, Store<true>{C, ldc, vec}, st) : launch(p, oa, ob, n_major, Store<false>{C, ldc, vec}, st);
    }
    if (e != cudaSuccess) { set_cuda_error(e, "scaled product launch"); return MVUE_ERR_CUDA; }
    return MVUE_OK;
}

}  // namespace
}  // namespace mvue

using namespace mvue;

extern "C" int mvue_scaled_forward_gemm(const void* x, const void* x_scales, int64_t tokens, int64_t in, int64_t ldx, const void* W,
                                        const void* W_scales, int64_t out, int64_t ldW, void* C, int c_dtype, int64_t ldc, int* dev_status,
                                        void* stream) {
    return scaled_gemm(x, tokens, in, ldx, x_scales, W, out, ldW, W_scales, false, C, c_dtype, ldc, dev_status, stream);
}

extern "C" int mvue_scaled_backward_gemm(const void* g, const void* g_scales, int64_t tokens, int64_t out, int64_t ldg, const void* W,
                                         const void* W_scales, int64_t in, int64_t ldW, void* C, int c_dtype, int64_t ldc, int* dev_status,
                                         void* stream) {
    return scaled_gemm(g, tokens, out, ldg, g_scales, W, in, ldW, W_scales, true, C, c_dtype, ldc, dev_status, stream);
}
