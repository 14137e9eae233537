// Embedding lookup with scaling, and its gradient by sorted tokens.
//
// Both move rows and are bound by HBM.  Lookup: a row in, a row out, a team of threads per row.  Gradient: (1) one
// cluster of eight thread blocks sorts the tokens by id (stable radix sort, digits of up to nine bits, histograms exchanged
// through distributed shared memory); (2) beside it the other SMs fill the rows of dW that no token names with zeros -- each
// block marks the ids of its own rows in a bitmap by reading the whole token list, which costs two microseconds of L2 reads at
// 32768 tokens and saves a dependent launch; (3) the sorted tokens are cut into chunks of equal length, a team adds the
// rows of a chunk in token order and writes the sums of the ids that begin and end in it; what crosses a chunk's edge goes to
// the workspace as a partial sum; (4) those are added in chunk order.  No atomics on data: equal inputs give equal bits.
//
// Measured (B200, HBM copy 6.55 TB/s).  Lookup of 16384 rows of 4096 bf16 out of 131072: 36 us against 29 us of HBM time
// (6915 rows differ); four pieces in flight for two gave 37 us: bound by the mix of gathered reads and writes.  Gradient of
// 32768 x 1024 bf16 into 65536 rows: 75 us against 51 us: fill 43 us (216 MB, 5 TB/s; a plain memset of as much takes 32 us;
// bulk stores from shared memory gave the same), beside it the sort 29 us, sums 24 us (5 TB/s), joins 11 us (each launch by itself).  8192 x 768 into
// 50257 rows: 39 us against 26 us.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "../../include/mvue_train.h"
#include "mvue_device.cuh"
#include "mvue_internal.h"
#include "mvue_train.cuh"

namespace mvue {
namespace {

namespace cg = cooperative_groups;

constexpr int kSortCtas = 8, kSortThreads = 1024, kSortWarps = kSortThreads / 32, kKeysPerThread = 4;
constexpr int kMaxDigitBits = 9, kMaxBins = 1 << kMaxDigitBits, kTileKeys = kSortThreads * kKeysPerThread;
constexpr int kWindowRows = 65536;              // rows of dW that one pass over the tokens marks (an 8 KB bitmap)
constexpr int kMaxChunk = 32;                   // sorted tokens a team adds at most
constexpr int kSlab = 1024;                     // columns of a team at most: 128 threads of eight

struct Ids {
    const void* p;
    bool is64;
    __device__ __forceinline__ int64_t at(int64_t i) const {
        return is64 ? __ldg(static_cast<const long long*>(p) + i) : (int64_t)__ldg(static_cast<const int*>(p) + i);
    }
};

// ---- lookup ----------------------------------------------------------------------------------------------------------
template <typename TW, typename TO, int kVec>
__global__ void __launch_bounds__(256) embed_kernel(Ids ids, int64_t tokens, const TW* __restrict__ w, int64_t vocab, int64_t cols,
                                                    int64_t ldw, float scale, TO* __restrict__ out, int64_t ldo, int* dev_status) {
    grid_dependency_wait();
    const int team = blockDim.x;
    const int64_t t = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    if (t >= tokens) return;
    const int64_t id = ids.at(t);
    const bool known = id >= 0 && id < vocab;
    if (!known && threadIdx.x == 0 && blockIdx.y == 0 && dev_status) *dev_status = MVUE_ERR_INDEX;
    w += known ? id * ldw : 0;
    out += t * ldo;
    // two pieces at a time: both loads are out before the first is used
    for (int64_t c0 = (int64_t)blockIdx.y * team * 16; c0 < cols; c0 += (int64_t)gridDim.y * team * 16) {
        const Cols<kVec> a(c0, cols, threadIdx.x, team), b(c0 + team * 8, cols, threadIdx.x, team);
        float x[8] = {}, y[8] = {};
        if (known && a.count) a.load(w, x);
        if (known && b.count) b.load(w, y);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[j] *= scale;
            y[j] *= scale;
        }
        if (a.count) a.store(out, x);
        if (b.count) b.store(out, y);
    }
}

// ---- gradient, first launch: sort and fill ---------------------------------------------------------------------------
struct SortArgs {
    Ids ids;
    int64_t tokens, vocab, padding;
    uint32_t *key[2], *pos[2];       // pass p reads [p & 1 ^ 1] (the first one the ids) and writes [p & 1]
    int passes, digit_bits;
    void* dw;
    int64_t cols, lddw;
    int elem_bytes, wide;
    int* dev_status;
};

__device__ __forceinline__ uint32_t key_of(const SortArgs& a, int64_t i) {
    const int64_t id = a.ids.at(i);
    if (id < 0 || id >= a.vocab) {
        if (a.dev_status) *a.dev_status = MVUE_ERR_INDEX;
        return (uint32_t)a.vocab;
    }
    return id == a.padding ? (uint32_t)a.vocab : (uint32_t)id;     // behind all rows
}

struct SortShared {
    uint32_t hist[kMaxBins];                        // this block's digits
    uint32_t base[kMaxBins];                        // where the block's next key of each digit goes
    uint16_t of_warp[kSortWarps][kMaxBins];
    uint32_t scan[kSortWarps];
};

__device__ void sort_tokens(const SortArgs& a, SortShared& s) {
    cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = (int)cluster.block_rank();
    const int bins = 1 << a.digit_bits;
    // consecutive tokens for each block
    const int64_t each = (a.tokens + kSortCtas - 1) / kSortCtas;
    const int64_t begin = min(a.tokens, each * rank), end = min(a.tokens, begin + each);
    for (int p = 0; p < a.passes; ++p) {
        const uint32_t* in_key = p ? a.key[(p & 1) ^ 1] : nullptr;
        const uint32_t* in_pos = p ? a.pos[(p & 1) ^ 1] : nullptr;
        const int shift = p * a.digit_bits;
        const uint32_t mask = bins - 1;
        for (int d = tid; d < kMaxBins; d += kSortThreads) s.hist[d] = 0u;
        __syncthreads();
        for (int64_t i = begin + tid; i < end; i += kSortThreads)
            atomicAdd(&s.hist[((p ? __ldcg(in_key + i) : key_of(a, i)) >> shift) & mask], 1u);
        cluster.sync();
        // keys of smaller digits anywhere, and of the same digit in earlier blocks, come first
        uint32_t total = 0u, before = 0u;
        if (tid < bins)
            for (int c = 0; c < kSortCtas; ++c) {
                const uint32_t h = cluster.map_shared_rank(s.hist, c)[tid];
                total += h;
                before += c < rank ? h : 0u;
            }
        uint32_t incl = total;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t up = __shfl_up_sync(0xFFFFFFFFu, incl, o);
            incl += lane >= o ? up : 0u;
        }
        if (lane == 31) s.scan[warp] = incl;
        __syncthreads();
        uint32_t front = 0u;
        for (int w = 0; w < warp && w < kMaxBins / 32; ++w) front += s.scan[w];
        if (tid < bins) s.base[tid] = front + incl - total + before;

        for (int64_t tile = begin; tile < end; tile += kTileKeys) {
            uint32_t* counts = reinterpret_cast<uint32_t*>(s.of_warp);
            for (int i = tid; i < kSortWarps * kMaxBins / 2; i += kSortThreads) counts[i] = 0u;
            __syncthreads();
            // ranks within the warp's 128 consecutive keys, in their order
            uint32_t key[kKeysPerThread], pos[kKeysPerThread], at[kKeysPerThread];
            const int64_t first = tile + (int64_t)warp * 32 * kKeysPerThread + lane;
#pragma unroll
            for (int k = 0; k < kKeysPerThread; ++k) {
                const int64_t i = first + k * 32;
                const bool in = i < end;
                key[k] = in ? (p ? __ldcg(in_key + i) : key_of(a, i)) : 0u;
                pos[k] = in ? (p ? __ldcg(in_pos + i) : (uint32_t)i) : 0u;
            }
#pragma unroll
            for (int k = 0; k < kKeysPerThread; ++k) {
                const bool in = first + k * 32 < end;
                const uint32_t d = in ? (key[k] >> shift) & mask : 0xFFFFFFFFu;
                const uint32_t same = __match_any_sync(0xFFFFFFFFu, d);
                const uint32_t lower = __popc(same & ((1u << lane) - 1u));
                uint32_t seen = 0u;
                if (in) seen = s.of_warp[warp][d];
                __syncwarp();
                if (in && lower == 0u) s.of_warp[warp][d] = (uint16_t)(seen + __popc(same));
                __syncwarp();
                at[k] = seen + lower;
            }
            __syncthreads();
            uint32_t sum = 0u, base = 0u;
            if (tid < bins) {
                base = s.base[tid];
#pragma unroll
                for (int w = 0; w < kSortWarps; ++w) {
                    const uint32_t n = s.of_warp[w][tid];
                    s.of_warp[w][tid] = (uint16_t)sum;
                    sum += n;
                }
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kKeysPerThread; ++k)
                if (first + k * 32 < end) {
                    const uint32_t d = (key[k] >> shift) & mask;
                    const uint32_t to = s.base[d] + s.of_warp[warp][d] + at[k];
                    a.key[p & 1][to] = key[k];
                    a.pos[p & 1][to] = pos[k];
                }
            __syncthreads();
            if (tid < bins) s.base[tid] = base + sum;
        }
        cluster.sync();          // the next pass reads what other blocks wrote, and their histograms have been read
    }
}

// zeros into this block's share of the rows that no token names; `mark(f)` calls f with every token's key
template <typename M>
__device__ __forceinline__ void fill_rows(const SortArgs& a, uint32_t* bitmap, int part, int parts, M mark) {
    const int tid = threadIdx.x;
    const int64_t row_bytes = a.cols * a.elem_bytes;
    const int64_t each = (a.vocab + parts - 1) / parts;
    const int64_t begin = min(a.vocab, each * part), end = min(a.vocab, begin + each);
    for (int64_t r0 = begin; r0 < end; r0 += kWindowRows) {
        const int64_t rows = min((int64_t)kWindowRows, end - r0);
        for (int i = tid; i < (rows + 31) / 32; i += kSortThreads) bitmap[i] = 0u;
        __syncthreads();
        mark([&](int64_t id) {
            const int64_t r = id - r0;
            if (r >= 0 && r < rows && id != a.padding) atomicOr(&bitmap[r >> 5], 1u << (r & 31));
        });
        __syncthreads();
        const uint32_t zero[8] = {};
        for (int64_t r = tid >> 5; r < rows; r += kSortWarps) {
            if (bitmap[r >> 5] >> (r & 31) & 1u) continue;
            char* row = static_cast<char*>(a.dw) + (r0 + r) * a.lddw * a.elem_bytes;
            if (a.wide)
                for (int64_t b = (tid & 31) * 32; b < row_bytes; b += 1024) st256(row + b, zero);
            else if (a.elem_bytes == 4)
                for (int64_t c = tid & 31; c < a.cols; c += 32) reinterpret_cast<uint32_t*>(row)[c] = 0u;
            else
                for (int64_t c = tid & 31; c < a.cols; c += 32) reinterpret_cast<uint16_t*>(row)[c] = 0;
        }
        __syncthreads();
    }
}

// One cluster.  What follows on the stream may start at once (the fill, which needs nothing of this kernel, and waits for
// it at its end so that the launch behind it has both).
__global__ void __launch_bounds__(kSortThreads, 1) embed_sort_kernel(const __grid_constant__ SortArgs a) {
    grid_dependency_wait();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ SortShared s;
    sort_tokens(a, s);
}
// Launched behind the sort: by the time its blocks run, every kernel before the sort has completed (the sort waited for
// them before it let this one start), so the ids may be read and dW written.
__global__ void __launch_bounds__(kSortThreads, 1) embed_fill_kernel(const __grid_constant__ SortArgs a) {
    __shared__ uint32_t bitmap[kWindowRows / 32];
    fill_rows(a, bitmap, blockIdx.x, gridDim.x, [&](auto f) {
#pragma unroll 4
        for (int64_t i = threadIdx.x; i < a.tokens; i += kSortThreads) f(a.ids.at(i));
    });
    grid_dependency_wait();
}

// Few tokens: every block holds all keys, a warp finds a token's place by counting those before it, and the same launch
// fills.  4096^2 comparisons are a microsecond on 148 SMs, where the sort in a cluster and a launch for it take fifteen; 8192^2
// would be four, which the fill hides less well than the sort beside it.
constexpr int kRankTokens = 4096;
__global__ void __launch_bounds__(kSortThreads, 1) embed_rank_kernel(const __grid_constant__ SortArgs a, int fill) {
    grid_dependency_wait();
    __shared__ __align__(16) uint32_t s_key[kRankTokens];
    __shared__ uint32_t bitmap[kWindowRows / 32];
    const int tokens = (int)a.tokens, padded = (tokens + 127) / 128 * 128, lane = threadIdx.x & 31;
    for (int i = threadIdx.x; i < padded; i += kSortThreads) s_key[i] = i < tokens ? key_of(a, i) : 0xFFFFFFFFu;
    __syncthreads();
    for (int t = (threadIdx.x >> 5) * gridDim.x + blockIdx.x; t < tokens; t += gridDim.x * kSortWarps) {
        const uint32_t key = s_key[t];
        uint32_t before = 0u;
        for (int j = lane * 4; j < padded; j += 128) {
            const uint4 k = *reinterpret_cast<const uint4*>(s_key + j);
            before += (k.x < key + (j < t)) + (k.y < key + (j + 1 < t)) + (k.z < key + (j + 2 < t)) + (k.w < key + (j + 3 < t));
        }
        before = __reduce_add_sync(0xFFFFFFFFu, before);
        if (lane == 0) {
            a.key[0][before] = key;
            a.pos[0][before] = (uint32_t)t;
        }
    }
    if (fill)
        fill_rows(a, bitmap, blockIdx.x, gridDim.x, [&](auto f) {
            for (int i = threadIdx.x; i < tokens; i += kSortThreads) f((int64_t)s_key[i] < a.vocab ? (int64_t)s_key[i] : -1);
        });
}

// ---- gradient, second launch: sums of chunks ---------------------------------------------------------------------------
struct SumArgs {
    const uint32_t *key, *pos;       // sorted
    int64_t tokens, vocab, chunks;
    int chunk;                       // sorted tokens of a team
    const void* dy;
    int64_t cols, lddy;
    float scale;
    void* dw;
    int64_t lddw;
    int accumulate;
    float* partial;                  // [chunks][2][ld_partial]: the id that came in over the chunk's front edge, the one that leaves
    int64_t ld_partial;
};

template <typename TD, int kVec>
__device__ __forceinline__ void put_row(const SumArgs& a, const Cols<kVec>& c, uint32_t id, float (&x)[8]) {
    TD* row = static_cast<TD*>(a.dw) + (int64_t)id * a.lddw;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] *= a.scale;
    if (a.accumulate) {              // fp32 only
        float old[8];
        c.load(row, old);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] += old[j];
    }
    c.store(row, x);
}

// Eight elements of a row as they lie in memory: what is in flight costs half the registers for bf16.
template <typename T, int kVec>
struct RawRow {
    static constexpr int kWords = kVec < 8 || sizeof(T) == 4 ? 8 : 4;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const Cols<kVec>& c, const T* row) {
        if constexpr (kVec < 8) {
            float x[8];
            c.load(row, x);
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(x[j]);
        } else if constexpr (sizeof(T) == 4) {
            ld256(row + c.first, w);
        } else {
            const uint4 q = *reinterpret_cast<const uint4*>(row + c.first);
            w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
        }
    }
    __device__ __forceinline__ void add_to(f2 (&acc)[4]) const {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            acc[j] = add2(acc[j], kWords == 4 ? pair(bf16_lo(w[j]), bf16_hi(w[j]))
                                              : pair(__uint_as_float(w[2 * j % kWords]), __uint_as_float(w[(2 * j + 1) % kWords])));
    }
};

template <typename TY, typename TD, int kVec>
__global__ void __launch_bounds__(128, kVec == 8 ? 6 : 4) embed_sum_kernel(const __grid_constant__ SumArgs a) {
    grid_dependency_wait();
    __shared__ uint32_t s_key[4][kMaxChunk + 2], s_pos[4][kMaxChunk];
    const int team = blockDim.x, ty = threadIdx.y;
    const int64_t chunk = (int64_t)blockIdx.x * blockDim.y + ty;
    const int64_t i0 = chunk * a.chunk;
    const int n = chunk < a.chunks ? (int)min((int64_t)a.chunk, a.tokens - i0) : 0;
    // keys of the chunk and of its neighbours on both sides (no id where there is none)
    for (int i = threadIdx.x; i < a.chunk + 2; i += team) {
        const int64_t at = i0 - 1 + i;
        s_key[ty][i] = n && at >= 0 && at < a.tokens ? a.key[at] : 0xFFFFFFFFu;
        if (i >= 1 && i <= n) s_pos[ty][i - 1] = a.pos[at];
    }
    __syncthreads();
    if (n == 0) return;
    const uint32_t* key = &s_key[ty][1];
    const Cols<kVec> c((int64_t)blockIdx.y * kSlab, a.cols, threadIdx.x, team);
    if (c.count == 0) return;
    const TY* dy = static_cast<const TY*>(a.dy);
    float* partial = a.partial + chunk * 2 * a.ld_partial;
    const uint32_t vocab = (uint32_t)a.vocab;
    f2 acc[4] = {};
    bool from_front = key[-1] == key[0];
    constexpr int kAhead = RawRow<TY, kVec>::kWords == 4 ? 8 : 4;
#pragma unroll 1
    for (int i = 0; i < n; i += kAhead) {
        RawRow<TY, kVec> x[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (i + u < n && key[i + u] < vocab) x[u].load(c, dy + (int64_t)s_pos[ty][i + u] * a.lddy);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i + u >= n || key[i + u] >= vocab) break;
            x[u].add_to(acc);
            const bool last = i + u + 1 == n, goes_on = key[i + u + 1] == key[i + u];
            if (!last && goes_on) continue;
            float sum[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                unpair(acc[j], sum[2 * j], sum[2 * j + 1]);
                acc[j] = pair(0.0f);
            }
            if (from_front) c.store(partial, sum);
            else if (goes_on) c.store(partial + a.ld_partial, sum);
            else put_row<TD, kVec>(a, c, key[i + u], sum);
            from_front = false;
        }
    }
}

// ---- gradient, third launch: ids that cross chunks --------------------------------------------------------------------
// The block of the chunk in which such an id begins adds that chunk's partial sum and those of the chunks it goes on in:
// its teams take consecutive shares of them, which are added in order.
constexpr int kJoinTeams = 4;
template <typename TD, int kVec>
__global__ void __launch_bounds__(128 * kJoinTeams) embed_join_kernel(const __grid_constant__ SumArgs a) {
    grid_dependency_wait();
    __shared__ float s[kJoinTeams - 1][8][128];
    const int64_t chunk = blockIdx.x, end = (chunk + 1) * a.chunk;
    if (end >= a.tokens) return;
    const uint32_t id = a.key[end - 1];
    if (id >= a.vocab || a.key[end] != id) return;                        // nothing leaves
    if (chunk > 0 && a.key[end - a.chunk] == id && a.key[end - a.chunk - 1] == id) return;   // began earlier
    // the last chunk whose first key is this id: every thread looks at one, as long as all of them are
    const int threads = blockDim.x * blockDim.y, tid = threadIdx.y * blockDim.x + threadIdx.x;
    int64_t lo = chunk;
    for (int found = threads; found == threads; lo += found) {
        const int64_t k = lo + 1 + tid;
        found = __syncthreads_count(k < a.chunks && a.key[k * a.chunk] == id);
    }
    const Cols<kVec> c((int64_t)blockIdx.y * kSlab, a.cols, threadIdx.x, blockDim.x);
    const int64_t each = (lo - chunk + 1 + kJoinTeams - 1) / kJoinTeams;       // the first partial sum is the chunk's own
    const int64_t first = chunk + each * threadIdx.y, last = min(lo + 1, first + each);
    float acc[8] = {};
    constexpr int kAhead = 4;
    if (c.count)
        for (int64_t k = first; k < last; k += kAhead) {
            float x[kAhead][8];
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (k + u < last) c.load(a.partial + ((k + u) * 2 + (k + u == chunk)) * a.ld_partial, x[u]);
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (k + u < last)
#pragma unroll
                    for (int j = 0; j < 8; ++j) acc[j] += x[u][j];
        }
    if (threadIdx.y > 0)
#pragma unroll
        for (int j = 0; j < 8; ++j) s[threadIdx.y - 1][j][threadIdx.x] = acc[j];
    __syncthreads();
    if (threadIdx.y > 0 || c.count == 0) return;
    for (int t = 0; t < kJoinTeams - 1; ++t)
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += s[t][j][threadIdx.x];
    put_row<TD, kVec>(a, c, id, acc);
}

// ---- host -------------------------------------------------------------------------------------------------------------
struct Layout {
    size_t key[2], pos[2], partial, bytes;
    int64_t chunks, ld_partial;
    int chunk;
};

// A team adds 32 tokens, fewer where that would leave SMs without teams (four for each of 148), but at least four: every
// chunk may leave two partial sums.  2153 tokens of 426 bf16: the sums take 28 us in chunks of 32 (34 blocks) and the whole call 37 us; in chunks of four the call takes 22 us.
int chunk_of(int64_t tokens) {
    int chunk = 4;
    while (chunk < kMaxChunk && tokens >= (int64_t)chunk * 2 * 4 * 148) chunk *= 2;
    return chunk;
}

Layout layout_of(int64_t tokens, int64_t cols) {
    Layout l;
    l.chunk = chunk_of(tokens);
    size_t at = 0;
    const auto take = [&](size_t n) { const size_t here = at; at += (n + 255) / 256 * 256; return here; };
    for (int i = 0; i < 2; ++i) {
        l.key[i] = take((size_t)tokens * 4);
        l.pos[i] = take((size_t)tokens * 4);
    }
    l.chunks = (tokens + l.chunk - 1) / l.chunk;
    l.ld_partial = (cols + 7) / 8 * 8;
    l.partial = take((size_t)l.chunks * 2 * (size_t)l.ld_partial * 4);
    l.bytes = at;
    return l;
}

template <typename TW, typename TO>
cudaError_t embed(Ids ids, int64_t tokens, const void* w, int64_t vocab, int64_t cols, int64_t ldw, float scale, void* out, int64_t ldo,
                  int vec, int* dev_status, cudaStream_t st) {
    // a thread moves two pieces of eight; the team is a power of two of up to 256 threads
    int team = 32;
    while (team < 256 && team * 16 < cols) team *= 2;
    const int rows = 256 / team;
    const int64_t pieces = (cols + team * 8 - 1) / (team * 8);
    const dim3 grid((unsigned)((tokens + rows - 1) / rows), (unsigned)std::min<int64_t>(pieces / 2 + pieces % 2, 65535));
    auto kernel = vec == 8 ? &embed_kernel<TW, TO, 8> : vec == 2 ? &embed_kernel<TW, TO, 2> : &embed_kernel<TW, TO, 1>;
    return launch_dependent(kernel, grid, dim3(team, rows), 0, st, ids, tokens, static_cast<const TW*>(w), vocab, cols, ldw, scale,
                            static_cast<TO*>(out), ldo, dev_status);
}

template <typename TY, typename TD>
cudaError_t sums(const SumArgs& a, int vec, cudaStream_t st) {
    const int64_t slab = std::min<int64_t>(kSlab, (a.cols + 7) / 8 * 8);
    const int team = (int)((slab / 8 + 31) / 32 * 32), teams = team <= 32 ? 4 : team <= 64 ? 2 : 1;
    const dim3 grid((unsigned)((a.chunks + teams - 1) / teams), (unsigned)((a.cols + kSlab - 1) / kSlab)), block(team, teams);
    cudaError_t e = launch_dependent(
        vec == 8 ? &embed_sum_kernel<TY, TD, 8> : vec == 2 ? &embed_sum_kernel<TY, TD, 2> : &embed_sum_kernel<TY, TD, 1>, grid, block, 0, st, a);
    if (e != cudaSuccess || a.chunks < 2) return e;
    return launch_dependent(vec == 8 ? &embed_join_kernel<TD, 8> : vec == 2 ? &embed_join_kernel<TD, 2> : &embed_join_kernel<TD, 1>, dim3((unsigned)a.chunks, grid.y),
                            dim3(team, kJoinTeams), 0, st, a);
}

cudaError_t launch_sort(const SortArgs& a, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(kSortCtas);
    cfg.blockDim = dim3(kSortThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = kSortCtas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, &embed_sort_kernel, a);
}

}  // namespace
}  // namespace mvue

using namespace mvue;

extern "C" {

int mvue_embedding(const void* ids, int id_bits, int64_t tokens, const void* W, int w_dtype, int64_t vocab, int64_t cols, int64_t ldW,
                   float scale, void* out, int out_dtype, int64_t ldout, int* dev_status, void* stream) {
    if (tokens < 0 || vocab <= 0 || cols <= 0 || ldW < cols || ldout < cols || tokens > 0x7FFFFFFF || vocab > 0x7FFFFFFF) return MVUE_ERR_SHAPE;
    if ((w_dtype != MVUE_F32 && w_dtype != MVUE_BF16) || (out_dtype != MVUE_F32 && out_dtype != MVUE_BF16) || (id_bits != 32 && id_bits != 64))
        return MVUE_ERR_DTYPE;
    if (tokens == 0) return MVUE_OK;
    if (!ids || !W || !out) return MVUE_ERR_NULL;
    if (off(ids, id_bits / 8) || off(W, size_of(w_dtype)) || off(out, size_of(out_dtype)) || off(dev_status, 4)) return MVUE_ERR_ALIGN;
    DeviceInfo dev;
    if (int s = current_device_info(&dev)) return s;
    const int vec = std::min(row_vector(W, ldW, cols, w_dtype), row_vector(out, ldout, cols, out_dtype));
    const Ids list{ids, id_bits == 64};
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (w_dtype == MVUE_BF16)
        e = out_dtype == MVUE_BF16 ? embed<__nv_bfloat16, __nv_bfloat16>(list, tokens, W, vocab, cols, ldW, scale, out, ldout, vec, dev_status, st)
                                   : embed<__nv_bfloat16, float>(list, tokens, W, vocab, cols, ldW, scale, out, ldout, vec, dev_status, st);
    else
        e = out_dtype == MVUE_BF16 ? embed<float, __nv_bfloat16>(list, tokens, W, vocab, cols, ldW, scale, out, ldout, vec, dev_status, st)
                                   : embed<float, float>(list, tokens, W, vocab, cols, ldW, scale, out, ldout, vec, dev_status, st);
    if (e != cudaSuccess) { set_cuda_error(e, "mvue_embedding launch"); return MVUE_ERR_CUDA; }
    return MVUE_OK;
}

int mvue_embedding_grad_workspace_bytes(int64_t tokens, int64_t cols, size_t* bytes) {
    if (!bytes) return MVUE_ERR_NULL;
    if (tokens < 0 || cols <= 0 || tokens > 0x7FFFFFFF) return MVUE_ERR_SHAPE;
    *bytes = layout_of(tokens, cols).bytes;
    return MVUE_OK;
}

int mvue_embedding_grad(const void* ids, int id_bits, int64_t tokens, const void* dy, int dy_dtype, int64_t cols, int64_t lddy, float scale,
                        int64_t padding_idx, void* dW, int dW_dtype, int64_t vocab, int64_t lddW, int accumulate, void* workspace,
                        size_t workspace_bytes, int* dev_status, void* stream) {
    if (tokens < 0 || vocab <= 0 || cols <= 0 || lddy < cols || lddW < cols || tokens > 0x7FFFFFFF || vocab > 0x7FFFFFFE) return MVUE_ERR_SHAPE;
    if ((cols + kSlab - 1) / kSlab > 65535) return MVUE_ERR_SHAPE;
    if ((dy_dtype != MVUE_F32 && dy_dtype != MVUE_BF16) || (dW_dtype != MVUE_F32 && dW_dtype != MVUE_BF16) || (id_bits != 32 && id_bits != 64) ||
        (accumulate && dW_dtype != MVUE_F32))
        return MVUE_ERR_DTYPE;
    if (!dW || (tokens > 0 && (!ids || !dy))) return MVUE_ERR_NULL;
    if (off(ids, id_bits / 8) || off(dy, size_of(dy_dtype)) || off(dW, size_of(dW_dtype)) || off(dev_status, 4)) return MVUE_ERR_ALIGN;
    if (tokens == 0 && accumulate) return MVUE_OK;
    const Layout l = layout_of(tokens, cols);
    if (l.bytes > 0 && (!workspace || workspace_bytes < l.bytes || off(workspace, 32))) return MVUE_ERR_WORKSPACE;
    DeviceInfo dev;
    if (int s = current_device_info(&dev)) return s;
    cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    char* ws = static_cast<char*>(workspace);
    SortArgs a = {};
    a.ids = Ids{ids, id_bits == 64};
    a.tokens = tokens;
    a.vocab = vocab;
    a.padding = padding_idx;
    for (int i = 0; i < 2; ++i) {
        a.key[i] = reinterpret_cast<uint32_t*>(ws + l.key[i]);
        a.pos[i] = reinterpret_cast<uint32_t*>(ws + l.pos[i]);
    }
    int bits = 1;                                       // of the largest key: `vocab`, that of tokens without a row
    while (bits < 32 && vocab >> bits) ++bits;
    a.passes = tokens == 0 ? 0 : (bits + kMaxDigitBits - 1) / kMaxDigitBits;
    a.digit_bits = a.passes ? (bits + a.passes - 1) / a.passes : 1;
    a.dw = dW;
    a.cols = cols;
    a.lddw = lddW;
    a.elem_bytes = (int)size_of(dW_dtype);
    a.wide = !off(dW, 32) && cols * a.elem_bytes % 32 == 0 && lddW * a.elem_bytes % 32 == 0;
    a.dev_status = dev_status;
    cudaError_t e;
    if (tokens <= kRankTokens) {
        a.passes = 1;                                   // sorted into the first pair of lists
        e = launch_dependent(&embed_rank_kernel, dim3((unsigned)dev.sm_count), dim3(kSortThreads), 0, st, a, (int)!accumulate);
    } else {
        e = launch_sort(a, st);
    }
    // one block on every SM that the sort leaves
    if (e == cudaSuccess && !accumulate && tokens > kRankTokens)
        e = launch_dependent(&embed_fill_kernel, dim3((unsigned)std::max(1, dev.sm_count - kSortCtas)), dim3(kSortThreads), 0, st, a);
    if (e == cudaSuccess && tokens > 0) {
        const int last = (a.passes - 1) & 1;
        SumArgs b = {a.key[last], a.pos[last], tokens, vocab, l.chunks, l.chunk, dy, cols, lddy, scale, dW, lddW, accumulate,
                     reinterpret_cast<float*>(ws + l.partial), l.ld_partial};
        const int vec = std::min(row_vector(dy, lddy, cols, dy_dtype), row_vector(dW, lddW, cols, dW_dtype));
        if (dy_dtype == MVUE_BF16)
            e = dW_dtype == MVUE_BF16 ? sums<__nv_bfloat16, __nv_bfloat16>(b, vec, st) : sums<__nv_bfloat16, float>(b, vec, st);
        else
            e = dW_dtype == MVUE_BF16 ? sums<float, __nv_bfloat16>(b, vec, st) : sums<float, float>(b, vec, st);
    }
    if (e != cudaSuccess) { set_cuda_error(e, "mvue_embedding_grad launch"); return MVUE_ERR_CUDA; }
    return MVUE_OK;
}

}  // extern "C"
