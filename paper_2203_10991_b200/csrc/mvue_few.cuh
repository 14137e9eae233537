// Products of few tokens, or of few output tiles: C[tokens x outs] from e4m3 codes with block scales, a single thread block's tensor core per
// tile and the reduction split over a cluster.
//
// The weights take the 128 rows of the instruction and the tokens its kTN columns, so that a handful of tokens costs shared memory for a
// handful: nearly all bytes in flight are weights.  A cluster of 1, 2, 4 or 8 blocks shares one tile, each a part of the reduction; the
// partial sums go to the blocks' own shared memory, and each block adds up a share of the tokens over the cluster in order of rank.
//   warps 0-3   warp 0: scales to shared memory in tensor-core order during the loop; then all: results
//   warp 4      TMA producer        warp 5   tensor-memory allocation, MMA issue
// Two blocks fit an SM.  8 x 14336 x 4096: 13.3 us in a graph, of which the weights' 58.7 MB take 9.1 us at the rate of a copy (9.3 us where they are
// in L2).
#pragma once
#include "mvue_dense.cuh"
#include "mvue_train.cuh"

namespace mvue {
namespace dense {

constexpr int kFewThreads = 192, kMaxSplit = 8;

template <bool kMMajorT, int kTNT>
struct FewShape {
    static constexpr bool kMMajor = kMMajorT;                            // the weights lie along the output axis, not along the reduction
    static constexpr int kTN = kTNT;
    static constexpr int kStages = kTN == 16 ? 5 : kTN == 64 ? 4 : 3;
    static constexpr int kWBytes = 128 * kLine, kStageBytes = kWBytes + kTN * kLine;
    static constexpr int kGroup = 4, kGroups = 3, kGroupBytes = 1024;    // scales: 512 bytes for the weights, 512 for the tokens
    static constexpr int kScaleBase = kStages * kStageBytes, kBars = kScaleBase + kGroups * kGroupBytes;
    static constexpr int kSmem = kBars + 256 + 1024;
    static constexpr uint32_t kCols = kTN == 16 ? 64 : kTN == 64 ? 128 : 256, kTmemScale = kTN;
    static constexpr uint32_t kInstr = (1u << 23) | ((kMMajor ? 1u : 0u) << 15) | ((uint32_t)(kTN >> 3) << 17) | ((128u >> 4) << 24);
    static_assert(kTmemScale + 8 * kGroups <= kCols && kTN * 128 * 4 <= kStages * kStageBytes && kWBytes % 1024 == 0, "does not fit");
};

struct FewParams {
    int tokens, outs, K;
    int tiles_o;                             // tiles of 128 outs
    int split, steps_per_part;
    const uint8_t *t_scales, *w_scales;      // exponent bytes [ceil(K / 128), tokens]; of the 128 x 128 blocks
    int64_t w_scales_o, w_scales_k;          // bytes from one block to the next along the outs, along K
    void* C;
    int64_t ldc;
    int bf16, vec;                           // vec: bytes that one access of C may take: 16, or an element
    int* dev_status;
};

__device__ __forceinline__ void mma_scaled(uint32_t d, uint64_t a, uint64_t b, uint32_t instr, uint32_t sa, uint32_t sb, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(instr), "r"(sa), "r"(sb), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void scales_to_tmem(uint32_t tmem, uint32_t smem) {
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(make_smem_desc(smem, 16, 128, kSwizzleNone)) : "memory");
}
__device__ __forceinline__ float ld_cluster1(uint32_t addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}

template <class S>
__global__ void __launch_bounds__(kFewThreads, 2)
few_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_t, const __grid_constant__ FewParams p) {
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem_gen = smem_raw + (smem_base - smem_u32(smem_raw));
    const uint32_t bar_base = smem_base + S::kBars;
    const auto full_bar = [&](int s) { return bar_base + 8u * s; };
    const auto empty_bar = [&](int s) { return bar_base + 8u * (S::kStages + s); };
    const auto scale_full_bar = [&](int s) { return bar_base + 8u * (2 * S::kStages + s); };
    const auto scale_empty_bar = [&](int s) { return bar_base + 8u * (2 * S::kStages + S::kGroups + s); };
    const uint32_t done_bar = bar_base + 8u * (2 * S::kStages + 2 * S::kGroups);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem_gen + S::kBars + 8 * (2 * S::kStages + 2 * S::kGroups + 1));
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int tile = blockIdx.x / p.split;
    const int out0 = tile % p.tiles_o * 128, token0 = tile / p.tiles_o * S::kTN;
    const int steps = (p.K + 127) / 128, begin = (int)rank * p.steps_per_part, count = max(0, min(steps - begin, p.steps_per_part));

    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) {
            mbar_init(full_bar(s), 1);
            mbar_init(empty_bar(s), 1);
        }
        for (int s = 0; s < S::kGroups; ++s) {
            mbar_init(scale_full_bar(s), 1);
            mbar_init(scale_empty_bar(s), 1);
        }
        mbar_init(done_bar, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 5) {
        tmem_alloc(smem_u32(tmem_slot), S::kCols);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    grid_dependency_wait();

    if (warp == 4) {
        if (lane == 0) {
            int s = 0;
            uint32_t parity = 1u;
            for (int i = 0; i < count; ++i) {
                if (!mbar_wait(empty_bar(s), parity, abort_flag)) break;
                const uint32_t w = smem_base + s * S::kStageBytes;
                const int k = (begin + i) * 128;
                mbar_expect_tx(full_bar(s), S::kStageBytes);
                tma_load_2d(w, &map_w, S::kMMajor ? out0 : k, S::kMMajor ? k : out0, full_bar(s));
                tma_load_2d(w + S::kWBytes, &map_t, k, token0, full_bar(s));
                if (++s == S::kStages) { s = 0; parity ^= 1u; }
            }
        }
    } else if (warp == 5) {
        if (lane == 0 && count > 0) {
            const uint64_t w0 = S::kMMajor ? make_smem_desc(smem_base, S::kWBytes, 1024, kSwizzle128B) : make_smem_desc(smem_base, 16, 1024, kSwizzle128B);
            const uint64_t t0 = make_smem_desc(smem_base + S::kWBytes, 16, 1024, kSwizzle128B);
            constexpr int kWStep = S::kMMajor ? 32 * kLine / 16 : 2;
            int s = 0, slot = 0;
            uint32_t parity = 0u, slot_parity = 0u;
            bool ok = true;
            for (int i = 0; i < count; ++i) {
                const uint32_t sw = tmem_base + S::kTmemScale + 8 * slot;
                if (i % S::kGroup == 0) {
                    if (!(ok = mbar_wait(scale_full_bar(slot), slot_parity, abort_flag))) break;
                    tc_fence_after();
                    scales_to_tmem(sw, smem_base + S::kScaleBase + slot * S::kGroupBytes);
                    scales_to_tmem(sw + 4, smem_base + S::kScaleBase + slot * S::kGroupBytes + 512);
                }
                if (!(ok = mbar_wait(full_bar(s), parity, abort_flag))) break;
                tc_fence_after();
                const uint64_t stage = (uint64_t)(s * (S::kStageBytes >> 4));
                const uint32_t id = (uint32_t)(i % S::kGroup);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    mma_scaled(tmem_base, w0 + stage + k * kWStep, t0 + stage + k * kAStep, S::kInstr | id << 4 | id << 29, sw, sw + 4, (i > 0 || k > 0) ? 1u : 0u);
                tc_commit(empty_bar(s));
                if (++s == S::kStages) { s = 0; parity ^= 1u; }
                if (i % S::kGroup == S::kGroup - 1 || i == count - 1) {
                    tc_commit(scale_empty_bar(slot));
                    if (++slot == S::kGroups) { slot = 0; slot_parity ^= 1u; }
                }
            }
            if (ok) tc_commit(done_bar);
        }
    } else if (warp == 0) {
        int slot = 0;
        uint32_t parity = 1u;
        const uint8_t* t_at[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) t_at[j] = p.t_scales + min(token0 + lane + 32 * j, p.tokens - 1);       // tokens that do not exist are zeros: any scale
        const uint8_t* w_at = p.w_scales + (out0 >> 7) * p.w_scales_o;
        for (int i0 = 0; i0 < count; i0 += S::kGroup) {
            uint32_t t[4] = {}, w = 0;
#pragma unroll
            for (int u = 0; u < S::kGroup; ++u) {
                const int64_t i = begin + min(i0 + u, count - 1);
#pragma unroll
                for (int j = 0; j < (S::kTN + 31) / 32; ++j) t[j] |= (uint32_t)__ldg(t_at[j] + i * p.tokens) << (8 * u);
                w |= (uint32_t)__ldg(w_at + i * p.w_scales_k) << (8 * u);
            }
            if (!__all_sync(0xFFFFFFFFu, mbar_wait(scale_empty_bar(slot), parity, abort_flag))) break;
            uint4* to = reinterpret_cast<uint4*>(smem_gen + S::kScaleBase + slot * S::kGroupBytes) + lane;
            to[0] = make_uint4(w, w, w, w);
            to[32] = make_uint4(t[0], t[1], t[2], t[3]);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(scale_full_bar(slot));
            if (++slot == S::kGroups) { slot = 0; parity ^= 1u; }
        }
    }
    __syncwarp();

    // the accumulator, row = out, to shared memory as [token][128 outs]: the stages are done with
    float* part = reinterpret_cast<float*>(smem_gen);
    if (warp < 4) {
        if (count > 0 && __all_sync(0xFFFFFFFFu, mbar_wait(done_bar, 0u, abort_flag))) {
            tc_fence_after();
            for (int c = 0; c < S::kTN; c += 16) {
                uint32_t v[16];
                asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                             : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
                               "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
                             : "r"(tmem_base + ((uint32_t)(32 * warp) << 16) + (uint32_t)c) : "memory");
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 16; ++i) part[(c + i) * 128 + 32 * warp + lane] = __uint_as_float(v[i]);
            }
        } else if (count == 0) {
            for (int c = 0; c < S::kTN; ++c) part[c * 128 + 32 * warp + lane] = 0.0f;
        }
    }
    tc_fence_before();
    __syncthreads();
    const bool failed = *abort_flag != 0;
    if (failed) {
        if (threadIdx.x == 0) {
            // copies that may still be in flight get a bounded chance to land
            for (int s = 0; s < S::kStages; ++s)
                for (uint32_t spin = 0; spin < 4096 && !mbar_try_wait(full_bar(s), 0) && !mbar_try_wait(full_bar(s), 1); ++spin) __nanosleep(64);
            if (p.dev_status) *p.dev_status = MVUE_ERR_DEVICE_TIMEOUT;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < S::kTN * 128; i += kFewThreads) part[i] = __uint_as_float(0x7FFFFFFFu);       // for all that add it
        __syncthreads();
    }
    if (p.split > 1) cluster_sync();         // every part is in shared memory

    // The next kernel is set up while this one adds up (8 x 14336 x 4096 one behind the other in a graph: 14.5 us without, 13.3 us; by calls from
    // Python 14.6 and 14.0; from the start on, its blocks took shared memory that this kernel's own wait for).
    grid_launch_dependents();
    // this block's share of the tokens, eight outs a thread: neighbours, or where rows do not allow wide accesses every sixteenth
    const int share = S::kTN / p.split, first = (int)rank * share;           // (split divides kTN)
    if (p.vec < 16) {
        for (int i = threadIdx.x; i < share * 16; i += kFewThreads) {
            const int token = first + (i >> 4), o = i & 15;
            if (token0 + token >= p.tokens) continue;
            const uint32_t at = smem_base + (uint32_t)(token * 128 + o) * 4;
            float x[8] = {};
            for (int r = 0; r < p.split; ++r) {
                const uint32_t from = map_to_cta(at, r);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] += ld_cluster1(from + 64 * j);
            }
            const int64_t to = (int64_t)(token0 + token) * p.ldc + out0 + o;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (out0 + o + 16 * j >= p.outs) break;
                if (p.bf16) static_cast<__nv_bfloat16*>(p.C)[to + 16 * j] = __float2bfloat16_rn(x[j]);
                else static_cast<float*>(p.C)[to + 16 * j] = x[j];
            }
        }
    } else
    for (int i = threadIdx.x; i < share * 16; i += kFewThreads) {
        const int token = first + (i >> 4), o = (i & 15) * 8;
        if (token0 + token >= p.tokens || out0 + o >= p.outs) continue;
        const uint32_t at = smem_base + (uint32_t)(token * 128 + o) * 4;
        float4 a[kMaxSplit], b[kMaxSplit];                   // all parts on their way at once
#pragma unroll
        for (int r = 0; r < kMaxSplit; ++r) {
            a[r] = b[r] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (r < p.split) {
                const uint32_t from = map_to_cta(at, r);
                a[r] = ld_cluster4(from);
                b[r] = ld_cluster4(from + 16);
            }
        }
        float x[8] = {};
#pragma unroll
        for (int r = 0; r < kMaxSplit; ++r) {
            x[0] += a[r].x; x[1] += a[r].y; x[2] += a[r].z; x[3] += a[r].w;
            x[4] += b[r].x; x[5] += b[r].y; x[6] += b[r].z; x[7] += b[r].w;
        }
        const int left = p.outs - out0 - o;
        const int64_t to = (int64_t)(token0 + token) * p.ldc + out0 + o;
        if (p.bf16) {
            const uint32_t w[4] = {pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
            store8_words(static_cast<__nv_bfloat16*>(p.C) + to, p.vec == 16 && left >= 8, left, w);
        } else {
            float* out = static_cast<float*>(p.C) + to;
            if (p.vec == 16 && left >= 8) {
                reinterpret_cast<float4*>(out)[0] = make_float4(x[0], x[1], x[2], x[3]);
                reinterpret_cast<float4*>(out)[1] = make_float4(x[4], x[5], x[6], x[7]);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < left) out[j] = x[j];
            }
        }
    }
    if (p.split > 1) cluster_sync();         // no block leaves while another reads its sums
    if (warp == 5) {
        tc_fence_after();
        tmem_dealloc(tmem_base, S::kCols);
    }
}

// tokens and weights as rows of bytes; n_major: the weights are [K x outs].
template <class S>
cudaError_t launch_few(FewParams p, const Operand& t, const Operand& w, cudaStream_t stream) {
    static PerDeviceOnce once;
    cudaError_t e = once_per_device(once, [](int) {
        return cudaFuncSetAttribute(few_kernel<S>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
    });
    if (e != cudaSuccess) return e;
    CUtensorMap map_w, map_t;
    if (!make_map_2d(&map_w, CU_TENSOR_MAP_DATA_TYPE_UINT8, w.base, S::kMMajor ? p.outs : p.K, S::kMMajor ? p.K : p.outs, w.pitch, 128, 128, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !make_map_2d(&map_t, CU_TENSOR_MAP_DATA_TYPE_UINT8, t.base, p.K, p.tokens, t.pitch, 128, S::kTN, CU_TENSOR_MAP_SWIZZLE_128B))
        return cudaErrorInvalidValue;
    const int tiles = p.tiles_o * ((p.tokens + S::kTN - 1) / S::kTN);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles * p.split));
    cfg.blockDim = dim3(kFewThreads);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)p.split;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, few_kernel<S>, map_w, map_t, p);
}

}  // namespace dense
}  // namespace mvue
