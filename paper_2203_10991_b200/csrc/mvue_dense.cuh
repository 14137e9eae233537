// Dense products on the 5th-generation tensor cores (tcgen05.mma), sm_100a: C[M x N] = A[M x K] . B, one or many matrices.
//   Half     A, B binary16, fp32 accumulators (kind::f16)
//   Scaled   A, B e4m3 with a power-of-two scale for each row of A and block of 128 along K, and for each 128 x 128 of B:
//            kind::mxf8f6f4 multiplies by the scales inside the tensor core (a scale byte there belongs to the 32 elements
//            along K of one instruction; four instructions take the same one), so no partial sum leaves the accumulator early
// A is K-major; B is K-major ([N x K] in memory) or N-major ([K x N]).
//
// Pair kernel: a cluster of two thread blocks computes one 256 x 256 tile with cta_group::2; block r loads its own 128 rows
// of A and its own half of B's columns, 128 bytes along K per stage.  Persistent: a pair walks the tiles.
//   warp 0      TMA producer (both blocks)          warp 1   MMA issue (leader)
//   warps 2, 3  tensor-memory allocation; Scaled: the scales from global to shared memory in tensor-core order
//   warps 4-11  epilogue
// Half keeps two accumulators of 256 columns.  Scaled needs tensor memory for scales beside them: its two accumulators
// overlap, and the epilogue drains the shared columns first, after which the next tile starts.
#pragma once
#include <cuda.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/mvue.h"
#include "mvue_device.cuh"
#include "mvue_internal.h"
#include "mvue_tc.cuh"
#include "mvue_tma.h"

namespace mvue {
namespace dense {

constexpr int kRowsA = 128;                  // rows of A per thread block
constexpr int kBN = 256;                     // columns of a pair's tile
constexpr int kLine = 128;                   // bytes along K per stage: 64 binary16 or 128 e4m3
constexpr int kPairThreads = 384;
constexpr int kEpiWarps = 8;
constexpr int kBand = 8;                     // row tiles per band of the tile order

// Epilogues.  Direct ones (kSlabs false) are handed 32 consecutive results of a row and store them themselves.  The others
// read and write matrices of binary16 in slabs of 128 rows x 64 columns, which an own warp moves by TMA through a ring in shared
// memory while the main loop runs: a thread owns a row, and its accesses to global memory would touch as many lines as there are lanes.
constexpr int kSlabBufs = 3;
constexpr int kSlabBytes = kRowsA * 64 * 2;  // 16 KiB; two matrices in a buffer

// How a product's operands lie and what its stages hold.  Scaled products have direct epilogues, the others slabs.
template <bool kScaledT, bool kNMajorT, int kStagesT>
struct Shape {
    static constexpr bool kScaled = kScaledT, kNMajor = kNMajorT;
    static constexpr int kBK = kScaled ? 128 : 64;                       // elements along K per stage
    static constexpr int kMmaK = kScaled ? 32 : 16;                      // elements along K per instruction: 32 bytes
    static constexpr int kABytes = kRowsA * kLine;                       // 16 KiB
    static constexpr int kHalfN = kBN / 2;                               // columns that one block of the pair loads
    static constexpr int kBBytes = kHalfN * kLine;                       // either order
    static constexpr int kColsBox = kScaled ? 128 : 64;                  // columns of an N-major box: a line of 128 bytes
    static constexpr int kBoxes = kNMajor ? kHalfN / kColsBox : 1;
    static constexpr int kBoxBytes = kBBytes / kBoxes;
    static constexpr int kBStep = (kNMajor ? kMmaK * kLine : 32) / 16;   // from one instruction's B to the next, in 16 bytes
    static constexpr int kStageBytes = kABytes + kBBytes;
    static constexpr int kStages = kStagesT;
    static constexpr int kSlabBase = kScaled ? 0 : kSlabBufs * 2 * kSlabBytes;        // bytes of that ring
    // Scales of kGroup stages travel together, four bytes of a row in a word, through rings of kGroups in shared and tensor memory.
    static constexpr int kGroup = 4, kGroups = kScaled ? 3 : 0;
    static constexpr int kScaleParts = 1 + kBN / 128;                                 // 128 rows of A, the columns of B
    static constexpr int kGroupBytes = 512 * kScaleParts;
    static constexpr int kScaleCols = 4 * kScaleParts;                                // tensor-memory columns of a group
    static constexpr int kTmemScale = 512 - kGroups * kScaleCols;
    static constexpr int kAcc1 = kScaled ? kTmemScale - kBN : kBN;                    // first column of the second accumulator
    static constexpr int kShared = kBN - kAcc1;                                       // columns that the accumulators share
    static constexpr int kSmem = kStages * kStageBytes + kGroups * kGroupBytes + kSlabBase + 1024 /*alignment*/ + 256 /*barriers*/;
    static constexpr uint32_t kInstr = (kScaled ? (1u << 23) /*scales: powers of two*/ : (1u << 4) /*D = f32*/) |
                                       ((kNMajor ? 1u : 0u) << 16) | ((uint32_t)(kBN >> 3) << 17);      // + M >> 4 at bit 24
    static_assert(kSmem <= 227 * 1024 && kStageBytes % 1024 == 0 && kAcc1 + kBN <= kTmemScale && kShared <= 64, "does not fit");
};

// Descriptors of a stage's operands; an address in one counts 16 bytes, so a stage's or an instruction's are sums.
constexpr int kAStep = 2;                    // 32 bytes along K per instruction
__device__ __forceinline__ uint64_t a_desc(uint32_t addr) { return make_smem_desc(addr, 16, 1024, kSwizzle128B); }
template <class S> __device__ __forceinline__ uint64_t b_desc(uint32_t addr) {
    if (!S::kNMajor) return make_smem_desc(addr, 16, 1024, kSwizzle128B);
    // groups of eight lines 1024 bytes apart, columns beyond a line in the next box
    return make_smem_desc(addr, S::kBoxBytes, 8 * kLine, kSwizzle128B);
}

__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t leader_bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(leader_bar) : "memory");
}
template <bool kScaled>
__device__ __forceinline__ void mma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t instr, uint32_t sa, uint32_t sb, uint32_t accumulate) {
    if constexpr (kScaled) {
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
            ::"r"(d), "l"(a), "l"(b), "r"(instr), "r"(sa), "r"(sb), "r"(accumulate) : "memory");
    } else {
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
            ::"r"(d), "l"(a), "l"(b), "r"(instr), "r"(accumulate) : "memory");
    }
}
// 32 lanes of 16 bytes to four columns of tensor memory, the same in each quarter of the lanes.
__device__ __forceinline__ void scales_to_tmem_pair(uint32_t tmem, uint32_t smem) {
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(make_smem_desc(smem, 16, 128, kSwizzleNone)) : "memory");
}

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, int x, int y, int z, uint32_t src) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(x), "r"(y), "r"(z), "r"(src) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }

// The matrices of a slab epilogue: one read, two written (the second may be the mirror image of the first).
struct SlabMaps {
    CUtensorMap in, out[2];
};
struct NoMaps {};

struct Params {
    int M, N, K, batch;
    int tiles_m, tiles_n;                    // of one matrix
    int tiles;                               // tiles of one matrix that are computed
    int symmetric;                           // M = N: only tiles on and above the diagonal
    int64_t n_work;
    const uint8_t* a_scales;                 // Scaled: exponent bytes [ceil(K / 128), M]
    const uint8_t* b_scales;                 // exponent bytes of the 128 x 128 blocks
    int64_t b_scales_n, b_scales_k;          // bytes from one block to the next along N, along K
    float* lost;                             // a number of each matrix that becomes NaN if a wait runs out: the caller hands it on to the results
    int* dev_status;
};

struct Tile {
    int m, n, z;                             // first row and column of the pair's tile, matrix
};
__device__ __forceinline__ Tile tile_at(const Params& p, int64_t w, int bn) {
    const int z = (int)(w / p.tiles);
    int t = (int)(w - (int64_t)z * p.tiles);
    if (p.symmetric) {
        int i = 0;
        while (t >= p.tiles_n - i) t -= p.tiles_n - i++;
        return {i * 2 * kRowsA, (i + t) * bn, z};
    }
    // bands of kBand row tiles, row tile fastest: the pairs at work share their operands in L2
    const int band = t / (kBand * p.tiles_n), h = min(kBand, p.tiles_m - band * kBand), in_band = t - band * kBand * p.tiles_n;
    return {(band * kBand + in_band % h) * 2 * kRowsA, in_band / h * bn, z};
}

template <class S, class Epilogue>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1)
pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ Params p,
            const __grid_constant__ typename Epilogue::Maps maps, const __grid_constant__ Epilogue epi) {
    static_assert(S::kScaled != Epilogue::kSlabs, "scaled products store directly, the others through slabs");
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem_gen = smem_raw + (smem_base - smem_u32(smem_raw));
    constexpr int kSlabs = S::kStages * S::kStageBytes, kScaleBase = kSlabs + S::kSlabBase, kBars = kScaleBase + S::kGroups * S::kGroupBytes;
    const uint32_t bar_base = smem_base + kBars;
    const auto full_bar = [&](int s) { return bar_base + 8u * s; };                // used in the leader only
    const auto empty_bar = [&](int s) { return bar_base + 8u * (S::kStages + s); };
    const auto acc_bar = [&](int b) { return bar_base + 8u * (2 * S::kStages + b); };          // accumulator complete (both blocks)
    const auto free_bar = [&](int b) { return bar_base + 8u * (2 * S::kStages + 2 + b); };     // accumulator drained (leader only)
    const auto scale_full_bar = [&](int s) { return bar_base + 8u * (2 * S::kStages + 4 + s); };                 // leader only
    const auto scale_empty_bar = [&](int s) { return bar_base + 8u * (2 * S::kStages + 4 + S::kGroups + s); };
    const auto slab_in_bar = [&](int b) { return bar_base + 8u * (2 * S::kStages + 4 + 2 * S::kGroups + b); };       // free, and its matrices read
    const auto slab_out_bar = [&](int b) { return bar_base + 8u * (2 * S::kStages + 4 + 2 * S::kGroups + kSlabBufs + b); };
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem_gen + kBars + 8 * (2 * S::kStages + 4 + 2 * S::kGroups + 2 * kSlabBufs));
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const int64_t n_pairs = gridDim.x >> 1, first = blockIdx.x >> 1;
    const int steps = (p.K + S::kBK - 1) / S::kBK;

    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) {
            mbar_init(full_bar(s), 1);       // the leader's producer arrives once, expecting both blocks' bytes
            mbar_init(empty_bar(s), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(acc_bar(b), 1);
            mbar_init(free_bar(b), 2 * kEpiWarps);
        }
        for (int s = 0; s < S::kGroups; ++s) {
            mbar_init(scale_full_bar(s), 2);                 // both blocks' scales
            mbar_init(scale_empty_bar(s), 1);
        }
        for (int b = 0; b < kSlabBufs; ++b) {
            mbar_init(slab_in_bar(b), 1);
            mbar_init(slab_out_bar(b), kEpiWarps);
        }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();                          // the peer's barriers exist before anyone signals them
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    grid_launch_dependents();
    grid_dependency_wait();                  // nothing above touches global memory

    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer (both blocks)
        if (lane == 0) {
            int s = 0;
            uint32_t parity = 1u;                            // of the stage's last release (a fresh barrier passes at parity 1)
            bool ok = true;
            for (int64_t w = first; w < p.n_work && ok; w += n_pairs) {
                const Tile t = tile_at(p, w, kBN);
                const int m = t.m + (int)rank * kRowsA, n = t.n + (int)rank * S::kHalfN;
                for (int i = 0; i < steps; ++i) {
                    if (!(ok = mbar_wait(empty_bar(s), parity, abort_flag))) break;
                    const uint32_t a_dst = smem_base + s * S::kStageBytes, b_dst = a_dst + S::kABytes;
                    const uint32_t leader_full = map_to_cta(full_bar(s), 0);
                    const int k = i * S::kBK;
                    if (rank == 0) mbar_expect_tx(full_bar(s), 2 * S::kStageBytes);
                    tma_load_3d_pair(a_dst, &map_a, k, m, t.z, leader_full);       // what lies outside a matrix reads as zeros
                    if (S::kNMajor) {
#pragma unroll
                        for (int j = 0; j < S::kBoxes; ++j)
                            tma_load_3d_pair(b_dst + j * S::kBoxBytes, &map_b, n + j * S::kColsBox, k, t.z, leader_full);
                    } else {
                        tma_load_3d_pair(b_dst, &map_b, k, n, t.z, leader_full);
                    }
                    if (++s == S::kStages) { s = 0; parity ^= 1u; }
                }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ MMA issue (leader)
        if (rank == 0 && lane == 0) {
            constexpr uint32_t instr = S::kInstr | ((2u * kRowsA >> 4) << 24);
            const uint64_t a0 = a_desc(smem_base), b0 = b_desc<S>(smem_base + S::kABytes);
            int s = 0, slot = 0;                             // stage; group of scales
            uint32_t parity = 0u, slot_parity = 0u, done = 0;
            bool ok = true;
            for (int64_t w = first; w < p.n_work && ok; w += n_pairs, ++done) {
                // Half: this accumulator's last tile is drained.  Scaled: the last tile's shared columns are.
                if (S::kScaled ? done > 0 : done > 1) {
                    ok = S::kScaled ? mbar_wait_cluster(free_bar(0), (done - 1) & 1u, abort_flag)
                                     : mbar_wait_cluster(free_bar(done & 1), ((done >> 1) - 1) & 1u, abort_flag);
                    if (!ok) break;
                    tc_fence_after();
                }
                const uint32_t acc = tmem_base + ((done & 1) ? S::kAcc1 : 0);
                for (int i = 0; i < steps; ++i) {
                    const uint32_t sa = tmem_base + S::kTmemScale + slot * S::kScaleCols;
                    if (S::kScaled && i % S::kGroup == 0) {
                        if (!(ok = mbar_wait_cluster(scale_full_bar(slot), slot_parity, abort_flag))) break;
                        tc_fence_after();
#pragma unroll
                        for (int j = 0; j < S::kScaleParts; ++j)
                            scales_to_tmem_pair(sa + 4 * j, smem_base + kScaleBase + slot * S::kGroupBytes + 512 * j);
                    }
                    if (!(ok = mbar_wait(full_bar(s), parity, abort_flag))) break;
                    tc_fence_after();
                    const uint64_t stage = (uint64_t)(s * (S::kStageBytes >> 4));
                    // the byte of the scales' words that this stage takes
                    const uint32_t id = S::kScaled ? (uint32_t)(i % S::kGroup) : 0u;
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        mma_pair<S::kScaled>(acc, a0 + stage + k * kAStep, b0 + stage + k * S::kBStep, instr | id << 4 | id << 29, sa, sa + 4,
                                             (i > 0 || k > 0) ? 1u : 0u);
                    tc_commit_pair(empty_bar(s));            // frees the stage in both blocks when the MMAs retire
                    if (++s == S::kStages) { s = 0; parity ^= 1u; }
                    if (S::kScaled && (i % S::kGroup == S::kGroup - 1 || i == steps - 1)) {
                        tc_commit_pair(scale_empty_bar(slot));
                        if (++slot == S::kGroups) { slot = 0; slot_parity ^= 1u; }
                    }
                }
                if (!ok) break;
                tc_commit_pair(acc_bar(done & 1));
            }
        }
    } else if (warp < 4 && S::kScaled) {
        // ------------------------------------------------------------ scales (both blocks): own rows of A, all columns of B
        // Two warps take groups of four stages in turn: a release at cluster scope takes longer than the tensor cores take for a
        // stage (one release per stage halved the rate of a 16384 x 14336 x 4096 product).
        // Lane l's words: rows l, l + 32, l + 64, l + 96 of 128, a byte for each of four stages.
        int slot = 0;
        uint32_t parity = 1u, group = 0;
        bool ok = true;
        const int blocks_n = (p.N + 127) >> 7;
        for (int64_t w = first; w < p.n_work && ok; w += n_pairs) {
            const Tile t = tile_at(p, w, kBN);
            const int row0 = t.m + (int)rank * kRowsA + lane;
            const uint8_t* a_at[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) a_at[j] = p.a_scales + min(row0 + 32 * j, p.M - 1);        // rows that do not exist are zeros: any scale
            for (int i0 = 0; i0 < steps; i0 += S::kGroup, ++group) {
                if (((group ^ warp) & 1u) == 0u) {
                    uint32_t a[4] = {}, b[kBN / 128] = {};
#pragma unroll
                    for (int u = 0; u < S::kGroup; ++u) {                          // all loads before the wait
                        const int64_t i = min(i0 + u, steps - 1);
#pragma unroll
                        for (int j = 0; j < 4; ++j) a[j] |= (uint32_t)__ldg(a_at[j] + i * p.M) << (8 * u);
#pragma unroll
                        for (int j = 0; j < kBN / 128; ++j)
                            b[j] |= (uint32_t)__ldg(p.b_scales + min((t.n >> 7) + j, blocks_n - 1) * p.b_scales_n + i * p.b_scales_k) << (8 * u);
                    }
                    if (!(ok = __all_sync(0xFFFFFFFFu, mbar_wait(scale_empty_bar(slot), parity, abort_flag)))) break;
                    uint4* to = reinterpret_cast<uint4*>(smem_gen + kScaleBase + slot * S::kGroupBytes) + lane;
                    to[0] = make_uint4(a[0], a[1], a[2], a[3]);
#pragma unroll
                    for (int j = 0; j < kBN / 128; ++j) to[32 * (1 + j)] = make_uint4(b[j], b[j], b[j], b[j]);
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the tensor cores read what the lanes wrote
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(map_to_cta(scale_full_bar(slot), 0));
                }
                if (++slot == S::kGroups) { slot = 0; parity ^= 1u; }
            }
        }
    } else if (Epilogue::kSlabs && warp == 3) {
        // ------------------------------------------------------------ slabs of the epilogue (both blocks, own rows)
        if constexpr (Epilogue::kSlabs) {
            if (lane == 0) {
                constexpr int kPer = kBN / 64;                // slabs of a tile
                // reads run a ring less one slab ahead of writes; a buffer is free when the write before the last has been taken from it
                int64_t w_in = first, w_out = first;
                int at_in = 0, at_out = 0, buf_in = 0, buf_out = 0;
                uint32_t parity = 0u;
                const auto read = [&] {
                    if (w_in >= p.n_work) return;
                    if (Epilogue::kIn > 0) {
                        const Tile t = tile_at(p, w_in, kBN);
                        const uint32_t to = smem_base + kSlabs + buf_in * 2 * kSlabBytes;
                        mbar_expect_tx(slab_in_bar(buf_in), kSlabBytes);
                        tma_load_3d(to, &maps.in, t.n + 64 * at_in, t.m + (int)rank * kRowsA, t.z, slab_in_bar(buf_in));
                    } else {
                        mbar_arrive(slab_in_bar(buf_in));
                    }
                    if (++buf_in == kSlabBufs) buf_in = 0;
                    if (++at_in == kPer) { at_in = 0; w_in += n_pairs; }
                };
                for (int i = 1; i < kSlabBufs; ++i) read();
                while (w_out < p.n_work) {
                    if (!mbar_wait(slab_out_bar(buf_out), parity, abort_flag)) break;
                    const Tile t = tile_at(p, w_out, kBN);
                    const int m = t.m + (int)rank * kRowsA, n = t.n + 64 * at_out;
                    const uint32_t from = smem_base + kSlabs + buf_out * 2 * kSlabBytes;
                    if (m < p.M && n < p.N) {
                        tma_store_3d(&maps.out[0], n, m, t.z, from);
                        if (Epilogue::kMirror) {
                            if (t.m != t.n) tma_store_3d(&maps.out[1], m, n, t.z, from + kSlabBytes);
                        } else if (epi.two_out()) {
                            tma_store_3d(&maps.out[1], n, m, t.z, from + kSlabBytes);
                        }
                    }
                    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
                    read();
                    if (++buf_out == kSlabBufs) { buf_out = 0; parity ^= 1u; }
                    if (++at_out == kPer) { at_out = 0; w_out += n_pairs; }
                }
                asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
            }
        }
    } else if (Epilogue::kSlabs && warp >= 4) {
        // ------------------------------------------------------------ epilogue in slabs: a warp 32 rows and 32 of the 64 columns
        if constexpr (Epilogue::kSlabs) {
            const int q = warp & 3, half = (warp - 4) >> 2, row = 32 * q + lane;
            const uint32_t rows_at = (uint32_t)(32 * q) << 16;
            const uint32_t leader_free[2] = {map_to_cta(free_bar(0), 0), map_to_cta(free_bar(1), 0)};
            uint32_t done = 0, parity = 0u;
            int buf = 0;
            bool ok = true;
            for (int64_t w = first; w < p.n_work && ok; w += n_pairs, ++done) {
                const Tile t = tile_at(p, w, kBN);
                const auto values = epi.values(t.z);
                const int par = done & 1;
                if (!__all_sync(0xFFFFFFFFu, mbar_wait(acc_bar(par), (done >> 1) & 1u, abort_flag))) break;
                tc_fence_after();
                const uint32_t acc = tmem_base + rows_at + (par ? S::kAcc1 : 0) + 32 * half;
                for (int c = 0; c < kBN / 64; ++c) {
                    uint32_t v[32];
                    tmem_ld_32x32b_x32(acc + 64 * c, v);
                    if (!(ok = __all_sync(0xFFFFFFFFu, mbar_wait(slab_in_bar(buf), parity, abort_flag)))) break;
                    uint8_t* slab = smem_gen + kSlabs + buf * 2 * kSlabBytes;
                    uint4 x[2][4];
                    const auto piece = [&](int i) { return reinterpret_cast<uint4*>(slab + row * 128 + (((4 * half + i) ^ (row & 7)) << 4)); };
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (Epilogue::kIn > 0) x[0][i] = *piece(i);
                    }
                    tmem_ld_wait();
                    if (c == kBN / 64 - 1) {                  // the accumulator is in registers: it may be overwritten
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0)
                            asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(leader_free[par]) : "memory");
                    }
                    epi.compute(values, v, x, t.m + (int)rank * kRowsA + 32 * q == t.n + 64 * c + 32 * half ? lane : -1);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        *piece(i) = x[0][i];
                        if (!Epilogue::kMirror && epi.two_out()) *(piece(i) + kSlabBytes / 16) = x[1][i];
                    }
                    if (Epilogue::kMirror && t.m != t.n) {       // [64 columns][128 rows]
                        unsigned short* to = reinterpret_cast<unsigned short*>(slab + kSlabBytes) + 32 * half * kRowsA + row;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t word[4] = {x[0][i].x, x[0][i].y, x[0][i].z, x[0][i].w};
#pragma unroll
                            for (int j = 0; j < 8; ++j) to[(8 * i + j) * kRowsA] = (unsigned short)(word[j >> 1] >> (16 * (j & 1)));
                        }
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(slab_out_bar(buf));
                    if (++buf == kSlabBufs) { buf = 0; parity ^= 1u; }
                }
            }
        }
    } else if (!Epilogue::kSlabs && warp >= 4) {
        if constexpr (!Epilogue::kSlabs) {
        // ------------------------------------------------------------ epilogue (both blocks, own rows)
        const int q = warp & 3, half = (warp - 4) >> 2;          // a quarter of the lanes, half of the columns
        const uint32_t rows_at = (uint32_t)(32 * q) << 16;
        const uint32_t leader_free = map_to_cta(free_bar(0), 0);
        constexpr int kChunks = kBN / 64, kFirst = kChunks / 2;
        // (relaxed: what is handed back was read by tcgen05.wait::ld; a release would wait for earlier stores to global memory)
        const auto arrive = [&] {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(leader_free) : "memory");
        };
        uint32_t done = 0;
        for (int64_t w = first; w < p.n_work; w += n_pairs, ++done) {
            const Tile t = tile_at(p, w, kBN);
            const int row = t.m + (int)rank * kRowsA + 32 * q + lane, par = done & 1;
            if (!__all_sync(0xFFFFFFFFu, mbar_wait(acc_bar(par), (done >> 1) & 1u, abort_flag))) {
                // a wait ran out: this tile and the ones to come are NaN, not what the output held before
                uint32_t nan[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) nan[i] = 0x7FFFFFFFu;
                for (; w < p.n_work; w += n_pairs) {
                    const Tile rest = tile_at(p, w, kBN);
                    for (int c = half * kChunks; c < (half + 1) * kChunks; ++c) epi.store(p, rest.m + (int)rank * kRowsA + 32 * q + lane, rest.n + 32 * c, nan);
                }
                break;
            }
            tc_fence_after();
            // the columns that this accumulator shares with the other one are among this half's first two chunks
            const bool shares = half != par;
            if (!shares) arrive();
            const uint32_t acc = tmem_base + rows_at + (par ? S::kAcc1 : 0);
            const auto chunk_at = [&](int c) { return half ? kBN - 32 * (c + 1) : 32 * c; };       // upper half: from the end
            {
                uint32_t v[kFirst][32];
#pragma unroll
                for (int c = 0; c < kFirst; ++c) tmem_ld_32x32b_x32(acc + chunk_at(c), v[c]);
                tmem_ld_wait();
                if (shares) arrive();
#pragma unroll
                for (int c = 0; c < kFirst; ++c) epi.store(p, row, t.n + chunk_at(c), v[c]);
            }
            {
                uint32_t v[kFirst][32];
#pragma unroll
                for (int c = 0; c < kFirst; ++c) tmem_ld_32x32b_x32(acc + chunk_at(kFirst + c), v[c]);
                tmem_ld_wait();
#pragma unroll
                for (int c = 0; c < kFirst; ++c) epi.store(p, row, t.n + chunk_at(kFirst + c), v[c]);
            }
        }
        }
    }

    tc_fence_before();
    __syncthreads();
    if (*abort_flag && threadIdx.x == 0) {
        // copies that may still be in flight get a bounded chance to land before the pair exits
        for (int s = 0; s < S::kStages; ++s)
            for (uint32_t spin = 0; spin < 4096 && !mbar_try_wait(full_bar(s), 0) && !mbar_try_wait(full_bar(s), 1); ++spin) __nanosleep(64);
        for (int b = 0; b < (Epilogue::kSlabs ? kSlabBufs : 0); ++b)
            for (uint32_t spin = 0; spin < 4096 && !mbar_try_wait(slab_in_bar(b), 0) && !mbar_try_wait(slab_in_bar(b), 1); ++spin) __nanosleep(64);
        if (p.lost)
            for (int z = 0; z < p.batch; ++z) p.lost[z] = __uint_as_float(0x7FFFFFFFu);
        if (p.dev_status) *p.dev_status = MVUE_ERR_DEVICE_TIMEOUT;
    }
    cluster_sync();                          // neither block leaves while the other may still touch it
    if (warp == 2) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------
// `batch` row-major matrices of `outer` rows x `inner` elements; a box is box_inner x box_outer elements of one.
inline bool make_map_3d(CUtensorMap* map, CUtensorMapDataType dtype, const void* base, int64_t inner, int64_t outer, int64_t batch,
                        int64_t pitch_bytes, int64_t matrix_bytes, uint32_t box_inner, uint32_t box_outer, CUtensorMapSwizzle swizzle) {
    auto fn = tensor_map_encoder();
    if (!fn) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)inner, (cuuint64_t)outer, (cuuint64_t)batch};
    const cuuint64_t strides[2] = {(cuuint64_t)pitch_bytes, (cuuint64_t)matrix_bytes};
    const cuuint32_t box[3] = {box_inner, box_outer, 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, dtype, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Operand {
    const void* base;
    int64_t pitch, matrix;                   // bytes from row to row, from matrix to matrix (multiples of 16)
};

// A slab's map of binary16 matrices [rows x cols]; the mirror image of a slab is 128 columns of 64 rows, as it lies.
inline bool make_slab_map(CUtensorMap* map, const Operand& x, int64_t rows, int64_t cols, int64_t batch, bool mirror) {
    return make_map_3d(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, x.base, cols, rows, batch, x.pitch, x.matrix, mirror ? kRowsA : 64, mirror ? 64 : kRowsA,
                       mirror ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B);
}

template <class S, class Epilogue>
struct PairSetup {
    PerDeviceOnce once;
    int max_pairs[kMaxDevices] = {};
};

// Launches the pair kernel for p (M, N, K, batch, scales and symmetric set; the rest is filled in here).
template <class S, class Epilogue>
cudaError_t launch_pair(Params p, const Operand& a, const Operand& b, const typename Epilogue::Maps& maps, const Epilogue& epi, cudaStream_t stream) {
    static PairSetup<S, Epilogue> st;
    cudaError_t e = once_per_device(st.once, [](int dev) {
        const cudaError_t err = cudaFuncSetAttribute(pair_kernel<S, Epilogue>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(2, 1, 1);
        cfg.blockDim = dim3(kPairThreads, 1, 1);
        cfg.dynamicSmemBytes = S::kSmem;
        int n = 0;
        if (err == cudaSuccess && cudaOccupancyMaxActiveClusters(&n, pair_kernel<S, Epilogue>, &cfg) == cudaSuccess) st.max_pairs[dev] = n;
        (void)cudaGetLastError();
        return err;
    });
    if (e != cudaSuccess) return e;
    int dev = 0;
    if ((e = cudaGetDevice(&dev)) != cudaSuccess) return e;
    p.tiles_m = (p.M + 2 * kRowsA - 1) / (2 * kRowsA);
    p.tiles_n = (p.N + kBN - 1) / kBN;
    p.tiles = p.symmetric ? p.tiles_n * (p.tiles_n + 1) / 2 : p.tiles_m * p.tiles_n;
    p.n_work = (int64_t)p.tiles * p.batch;
    const CUtensorMapDataType dt = S::kScaled ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    CUtensorMap map_a, map_b;
    if (!make_map_3d(&map_a, dt, a.base, p.K, p.M, p.batch, a.pitch, a.matrix, S::kBK, kRowsA, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !(S::kNMajor ? make_map_3d(&map_b, dt, b.base, p.N, p.K, p.batch, b.pitch, b.matrix, S::kColsBox, S::kBK, CU_TENSOR_MAP_SWIZZLE_128B)
                     : make_map_3d(&map_b, dt, b.base, p.K, p.N, p.batch, b.pitch, b.matrix, S::kBK, S::kHalfN, CU_TENSOR_MAP_SWIZZLE_128B)))
        return cudaErrorInvalidValue;
    int64_t pairs = st.max_pairs[dev] > 0 ? st.max_pairs[dev] : 1;
    if (pairs > p.n_work) pairs = p.n_work;
    return launch_dependent(&pair_kernel<S, Epilogue>, dim3((unsigned)(2 * pairs)), dim3(kPairThreads), S::kSmem, stream, map_a, map_b, p, maps, epi);
}

}  // namespace dense
}  // namespace mvue
