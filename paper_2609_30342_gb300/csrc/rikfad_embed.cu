// rikfad_embed.cu -- token embedding: out_t = scale W[id_t], and the table's
// gradient dW_v = scale sum_{t: id_t = v} dout_t.
//
// Forward is a copy of rows.  Backward sorts the tokens by id (stable, so a row's
// tokens stay in order) and sums runs of equal ids, `chunk` sorted tokens a warp,
// in float32 registers.  A run within its chunk is written at once; a run over
// several leaves a partial row in each, joined by a second kernel in the chunks'
// order.  Nothing depends on which block is first.
//
// Memory bounds both: dout is read once, every row of dW written once (rows without
// a token as zeros, while the tokens are sorted and beside the sums).  65536 tokens of
// 4096 in bfloat16, table of 131072: forward 121 us (0.74 GB, 6.1 TB/s), gradient 276
// (1.6 GB, 5.8 TB/s); 16384 of 768 in float32, table of 50257: 12 and 49 us, the latter
// 18 for the sort, beside which the others write zeros to 62 MB.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <string>

#include "rikfad.h"
#include "rikfad_host.hpp"
#include "rikfad_kernels.cuh"
#include "rikfad_types.cuh"

using namespace rikfad;

namespace {

constexpr int kSms = 152;
constexpr int kForwardThreads = 256, kForwardRows = 4;
constexpr int kNarrowThreads = 128, kNarrowColumns = 256;
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32, kSortCtas = 8, kSortItems = 8;
constexpr int kSortTile = kSortThreads * kSortItems;
constexpr int kSortBits = 9;            // of a pass: the warps' counts of 2^9 digits take 32 KB
constexpr int kSumThreads = 128, kSumWarps = kSumThreads / 32, kSumAhead = 8;
constexpr int kJoinThreads = 256, kJoinWarps = kJoinThreads / 32, kJoinAhead = 8, kJoinBlocks = 4 * kSms;
// Of all multiprocessors but the sorting ones: 62 MB beside the sort of 16384 tokens, which takes 18 us with them and 15
// alone, 136 MB beside that of 65536, 37 and 35.
constexpr double kZeroBytesPerUs = 4.2e6;
constexpr int kShortRun = 32;           // chunks that a run joined by one warp goes on in, at most
constexpr int kCountThreads = 256, kMostCounted = 6144;

struct EmbedParams {
    const void *ids;
    void *table, *rows;
    int64_t table_stride, row_stride;
    int64_t tokens, vocab;
    int32_t width, units;               // units: vectors of a row
    int32_t id_bytes, accumulate;
    float scale;
    // backward
    uint2 *order;                       // (id, token), sorted; ids outside the table last, as vocab
    float *head, *tail;                 // partial rows of chunks, `pitch` floats apart
    int32_t *counts, *starts;           // chunks where a run over several starts: how many, which
    int64_t pitch, chunks;
    int64_t zero_from;                  // rows from here on are zero already
    int32_t chunk, slabs;               // tokens of a chunk; warps side by side over a row
    int64_t sum_blocks;
    int32_t zero_rows;                  // of a warp that writes zeros
};

// An id outside the table as vocab.
__device__ __forceinline__ uint32_t id_at(const void *ids, int id_bytes, int64_t i, int64_t vocab)
{
    const int64_t id = id_bytes == 4 ? (int64_t)static_cast<const int32_t *>(ids)[i] : static_cast<const int64_t *>(ids)[i];
    return (uint32_t)(id >= 0 && id < vocab ? id : vocab);
}

template <typename T, int V> __device__ __forceinline__ void load(Vec<T, V> &r, const T *p)
{
    r.word = *reinterpret_cast<const decltype(r.word) *>(p);
}
template <typename T, int V> __device__ __forceinline__ void store(const Vec<T, V> &r, T *p)
{
    *reinterpret_cast<decltype(r.word) *>(p) = r.word;
}

// Zeros to n elements, 16 bytes at a time wherever they start.
template <typename W> __device__ __forceinline__ void zero(W *to, int64_t n, int64_t thread, int64_t threads)
{
    constexpr int E = 16 / sizeof(W);
    const int64_t lead = min((int64_t)((16 - (uint32_t)(uintptr_t)to % 16) % 16 / sizeof(W)), n), vectors = (n - lead) / E;
    for (int64_t i = thread; i < vectors; i += threads)
        reinterpret_cast<uint4 *>(to + lead)[i] = make_uint4(0, 0, 0, 0);
    if (thread < n - vectors * E)
        to[thread < lead ? thread : thread + vectors * E] = from_f32<W>(0.f);
}

// A block's threads are `lanes` across a row (blockDim.x) and blockDim.y rows; a
// thread has kForwardRows rows under way.
template <typename W, typename O, int V>
__global__ void __launch_bounds__(kForwardThreads) rikfad_embed_forward_kernel(const __grid_constant__ EmbedParams p)
{
    wait_for_predecessor();
    allow_successor_launch();
    const W *table = static_cast<const W *>(p.table);
    const int64_t first = ((int64_t)blockIdx.x * blockDim.y + threadIdx.y) * kForwardRows;
    const W *from[kForwardRows];
    O *to[kForwardRows];
    bool inside[kForwardRows];
#pragma unroll
    for (int r = 0; r < kForwardRows; ++r) {
        const int64_t t = first + r;
        const uint32_t id = t < p.tokens ? id_at(p.ids, p.id_bytes, t, p.vocab) : (uint32_t)p.vocab;
        inside[r] = id < p.vocab;
        from[r] = table + id * p.table_stride;
        to[r] = t < p.tokens ? static_cast<O *>(p.rows) + t * p.row_stride : nullptr;
    }
    for (int u = blockIdx.y * blockDim.x + threadIdx.x; u < p.units; u += blockDim.x * gridDim.y) {
        Vec<W, V> in[kForwardRows];
#pragma unroll
        for (int r = 0; r < kForwardRows; ++r)
            if (inside[r])
                load(in[r], from[r] + (int64_t)u * V);
#pragma unroll
        for (int r = 0; r < kForwardRows; ++r) {
            float f[V];
            widen(in[r], f);
#pragma unroll
            for (int e = 0; e < V; ++e)
                f[e] = inside[r] ? f[e] * p.scale : 0.f;
            Vec<O, V> out;
            narrow(f, out);
            if (to[r])
                store(out, to[r] + (int64_t)u * V);
        }
    }
}

// Rows that start anywhere: a warp has 256 columns of kForwardRows rows, read and written 16
// bytes at a time where elements have 2 bytes, by way of shared memory, and neighbours side by
// side where they have 4.
template <typename W, typename O>
__global__ void __launch_bounds__(kNarrowThreads) rikfad_embed_forward_narrow_kernel(const __grid_constant__ EmbedParams p)
{
    constexpr int kSlot = kNarrowColumns * 2 + 16, kEach = kNarrowColumns / 32;
    __shared__ uint4 buffers[kNarrowThreads / 32][kForwardRows][kSlot / 16];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, slabs = p.slabs;
    const int64_t item = (int64_t)blockIdx.x * (kNarrowThreads / 32) + warp;
    const int64_t first = item / slabs * kForwardRows;
    const int column = (int)(item % slabs) * kNarrowColumns, here = min(kNarrowColumns, p.width - column);
    wait_for_predecessor();
    allow_successor_launch();
    if (first >= p.tokens)
        return;
    const W *from[kForwardRows];
    bool inside[kForwardRows];
    uint4 in[kForwardRows][2];
    float f[kForwardRows][kEach];
#pragma unroll
    for (int r = 0; r < kForwardRows; ++r) {
        const uint32_t id = first + r < p.tokens ? id_at(p.ids, p.id_bytes, first + r, p.vocab) : (uint32_t)p.vocab;
        inside[r] = id < p.vocab;
        from[r] = static_cast<const W *>(p.table) + id * p.table_stride + column;
    }
#pragma unroll
    for (int r = 0; r < kForwardRows; ++r) {
        if constexpr (sizeof(W) == 2) {
            const int skip = (int)((uintptr_t)from[r] % 16), words = (skip + here * 2 + 15) / 16;
            const uint4 *words_from = reinterpret_cast<const uint4 *>(reinterpret_cast<const char *>(from[r]) - skip);
            if (inside[r] && lane < words)
                in[r][0] = words_from[lane];
            if (inside[r] && lane + 32 < words)
                in[r][1] = words_from[lane + 32];
        } else {
#pragma unroll
            for (int j = 0; j < kEach; ++j)
                f[r][j] = inside[r] && lane + 32 * j < here ? to_f32(from[r][lane + 32 * j]) : 0.f;
        }
    }
    if constexpr (sizeof(W) == 2) {
#pragma unroll
        for (int r = 0; r < kForwardRows; ++r) {
            buffers[warp][r][lane] = in[r][0];
            if (lane + 32 < kSlot / 16)
                buffers[warp][r][lane + 32] = in[r][1];
        }
        __syncwarp();
#pragma unroll
        for (int r = 0; r < kForwardRows; ++r) {
            const W *at = reinterpret_cast<const W *>(reinterpret_cast<const char *>(buffers[warp][r]) + (uintptr_t)from[r] % 16);
#pragma unroll
            for (int j = 0; j < kEach; ++j)
                f[r][j] = inside[r] && lane + 32 * j < here ? to_f32(at[lane + 32 * j]) : 0.f;
        }
        __syncwarp();
    }
#pragma unroll
    for (int r = 0; r < kForwardRows; ++r) {
        if (first + r >= p.tokens)
            break;
        O *to = static_cast<O *>(p.rows) + (first + r) * p.row_stride + column;
        if constexpr (sizeof(O) == 2) {
            constexpr int E = 8;
            const int skip = (int)((uintptr_t)to % 16), lead = min((16 - skip) % 16 / 2, here);
            const int words = (here - lead) / E, edges = here - words * E;
            O *const place = reinterpret_cast<O *>(reinterpret_cast<char *>(buffers[warp][r]) + skip);
#pragma unroll
            for (int j = 0; j < kEach; ++j)
                if (lane + 32 * j < here)
                    place[lane + 32 * j] = from_f32<O>(f[r][j] * p.scale);
            __syncwarp();
            if (lane < words)
                reinterpret_cast<uint4 *>(to + lead)[lane] = reinterpret_cast<const uint4 *>(place + lead)[lane];
            if (lane < edges)
                to[lane < lead ? lane : lane + words * E] = place[lane < lead ? lane : lane + words * E];
        } else {
#pragma unroll
            for (int j = 0; j < kEach; ++j)
                if (lane + 32 * j < here)
                    to[lane + 32 * j] = from_f32<O>(f[r][j] * p.scale);
        }
    }
}

// --------------------------------------------------------------- sorted tokens

struct SortParams {
    const void *ids;
    uint2 *from, *to;               // of the passes in turn; the last one writes to `to`
    int64_t vocab;
    int32_t tokens, id_bytes, passes, bits;
    int32_t count_blocks;
    int32_t *counts;                // zeroed for the sums
    // rows of the table from zero_from on get zeros from the blocks that do not sort
    void *table;
    int64_t table_stride, zero_from;
    int32_t width, table_bytes;     // bytes of an element
};

// Rows from zero_from on, by `blocks` blocks of which this is the one numbered `block`.
__device__ __forceinline__ void zero_rows(const SortParams &p, int64_t block, int64_t blocks)
{
    const int64_t rows = p.vocab - p.zero_from, size = (int64_t)p.width * p.table_bytes, stride = p.table_stride * p.table_bytes;
    char *first = static_cast<char *>(p.table) + p.zero_from * stride;
    if (rows <= 0)
        return;
    auto part = [&](char *at, int64_t n, int64_t thread, int64_t threads) {
        if (p.table_bytes == 4)
            zero(reinterpret_cast<float *>(at), n / 4, thread, threads);
        else
            zero(reinterpret_cast<__half *>(at), n / 2, thread, threads);
    };
    if (stride == size || rows == 1) {
        part(first, rows * size, block * blockDim.x + threadIdx.x, blocks * blockDim.x);
        return;
    }
    const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    for (int64_t row = block * warps + (threadIdx.x >> 5); row < rows; row += blocks * warps)
        part(first + row * stride, size, lane, 32);
}

__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

__device__ __forceinline__ uint32_t cluster_read(const uint32_t *mine, int rank)
{
    uint32_t at, v;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(mine)), "r"(rank));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}

// The lanes that have this lane's digit; `there`: whether it has one.
__device__ __forceinline__ uint32_t lanes_alike(uint32_t digit, bool there, int bits)
{
    uint32_t same = __ballot_sync(~0u, there);
#pragma unroll
    for (int b = 0; b < kSortBits; ++b)
        if (b < bits) {
            const uint32_t set = __ballot_sync(~0u, digit >> b & 1);
            same &= digit >> b & 1 ? set : ~set;
        }
    return same;
}

// Exclusive sum over the block's threads.
__device__ __forceinline__ uint32_t block_exclusive(uint32_t v, uint32_t *sums)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t s = v;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const uint32_t o = __shfl_up_sync(~0u, s, d);
        s += lane >= d ? o : 0;
    }
    if (lane == 31)
        sums[warp] = s;
    __syncthreads();
    uint32_t w = lane < kSortWarps ? sums[lane] : 0;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const uint32_t o = __shfl_up_sync(~0u, w, d);
        w += lane >= d ? o : 0;
    }
    const uint32_t before = __shfl_sync(~0u, w, max(warp - 1, 0));
    return s - v + (warp ? before : 0);
}

// One cluster of 8 blocks (the portable size; its barriers cost less than launches) sorts the
// tokens by id, `bits` bits a pass, the lowest
// first.  Every block has a run of the pass's input: it counts its digits, learns the
// other blocks' counts through their shared memory, and moves its entries, a tile
// at a time, each warp's 32 neighbours in turn, so that equal digits keep their order.
// Alone it takes 12 us for 8192 tokens, 15 for 16384, 33 for 65536 (one tile a block), 83 for
// 131072 (two): chains of loads and barriers, then scattered writes of 8 bytes.
__global__ void __launch_bounds__(kSortThreads) rikfad_embed_sort_kernel(const __grid_constant__ SortParams p)
{
    extern __shared__ uint32_t smem[];
    const int bins = 1 << p.bits;
    uint32_t *total = smem, *base = total + bins, *start = base + bins, *sums = start + bins;
    uint16_t *counts = reinterpret_cast<uint16_t *>(sums + 32);     // [warp][digit]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t rank;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const int64_t share = ((int64_t)p.tokens + kSortCtas - 1) / kSortCtas;
    const int begin = (int)min(share * rank, (int64_t)p.tokens), end = (int)min(share * (rank + 1), (int64_t)p.tokens);
    wait_for_predecessor();
    allow_successor_launch();
    if (blockIdx.x >= kSortCtas) {
        zero_rows(p, blockIdx.x - kSortCtas, gridDim.x - kSortCtas);
        return;
    }
    if (blockIdx.x == 0 && threadIdx.x < 2)
        p.counts[threadIdx.x] = 0;
    for (int pass = 0; pass < p.passes; ++pass) {
        const uint2 *from = (p.passes - pass) % 2 ? p.from : p.to;
        uint2 *to = (p.passes - pass) % 2 ? p.to : p.from;
        const int shift = pass * p.bits;
        auto entry = [&](int i) {
            return pass == 0 ? make_uint2(id_at(p.ids, p.id_bytes, i, p.vocab), (uint32_t)i) : __ldcg(from + i);
        };
        // a digit's first place for this block: after all lower digits and the blocks before it
        auto first_places = [&] {
            cluster_barrier();
            uint32_t before = 0, all = 0;
            if (threadIdx.x < bins) {
#pragma unroll
                for (int r = 0; r < kSortCtas; ++r) {
                    const uint32_t n = cluster_read(total + threadIdx.x, r);
                    before += r < rank ? n : 0;
                    all += n;
                }
            }
            const uint32_t first = block_exclusive(all, sums);
            if (threadIdx.x < bins)
                base[threadIdx.x] = first + before;
        };
        const bool one_tile = end - begin <= kSortTile;
        if (!one_tile) {
            for (int b = threadIdx.x; b < bins; b += kSortThreads)
                total[b] = 0;
            __syncthreads();
            for (int i = begin + warp * 32; i < end; i += kSortThreads) {
                const bool there = i + lane < end;
                const uint32_t digit = there ? entry(i + lane).x >> shift & (bins - 1) : 0;
                const uint32_t same = lanes_alike(digit, there, p.bits);
                if (there && lane == __ffs(same) - 1)
                    atomicAdd(total + digit, __popc(same));     // integers: any order
            }
            first_places();
        }
        for (int tile = begin; tile < end || (one_tile && tile == begin); tile += kSortTile) {
            uint2 e[kSortItems];
            uint32_t place[kSortItems];
            uint16_t *mine = counts + warp * bins;
            // every warp has `rounds` times 32 neighbours
            const int rounds = (min(end - tile, kSortTile) + kSortThreads - 1) / kSortThreads, first = tile + warp * rounds * 32 + lane;
            auto item = [&](int k) { return k < rounds ? first + k * 32 : end; };
#pragma unroll
            for (int k = 0; k < kSortItems; ++k)
                e[k] = item(k) < end ? entry(item(k)) : make_uint2(0, 0);
            for (int b = threadIdx.x; b < bins * kSortWarps / 2; b += kSortThreads)
                reinterpret_cast<uint32_t *>(counts)[b] = 0;
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kSortItems; ++k) {
                const int i = item(k);
                if (k >= rounds)
                    break;
                const uint32_t digit = e[k].x >> shift & (bins - 1);
                const uint32_t same = lanes_alike(digit, i < end, p.bits);
                const int leader = __ffs(same) - 1;
                uint32_t old = 0;
                if (lane == leader && i < end) {
                    old = mine[digit];
                    mine[digit] = (uint16_t)(old + __popc(same));
                }
                __syncwarp();
                place[k] = __shfl_sync(~0u, old, leader) + __popc(same & ((1u << lane) - 1));
            }
            __syncthreads();
            uint32_t n = 0;
            if (threadIdx.x < bins) {
                uint16_t here[kSortWarps];
#pragma unroll
                for (int w = 0; w < kSortWarps; ++w)
                    here[w] = counts[w * bins + threadIdx.x];
#pragma unroll
                for (int w = 0; w < kSortWarps; ++w) {
                    counts[w * bins + threadIdx.x] = (uint16_t)n;
                    n += here[w];
                }
            }
            if (one_tile) {
                if (threadIdx.x < bins)
                    total[threadIdx.x] = n;
                first_places();
            }
            if (threadIdx.x < bins) {
                start[threadIdx.x] = base[threadIdx.x];
                base[threadIdx.x] += n;
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kSortItems; ++k) {
                const uint32_t digit = e[k].x >> shift & (bins - 1);
                if (item(k) < end)
                    to[start[digit] + mine[digit] + place[k]] = e[k];
            }
            __syncthreads();
        }
        cluster_barrier();          // the next pass reads what every block wrote
    }
}

// Few tokens: each one's place is the number of ids below its own and of equal ids before
// it, counted by a warp.  The blocks from count_blocks on write zeros.  4099 tokens in 9 us,
// where the cluster's sort takes 12.
__global__ void __launch_bounds__(kCountThreads) rikfad_embed_count_kernel(const __grid_constant__ SortParams p)
{
    __shared__ uint4 all[kMostCounted / 4];
    uint32_t *const ids = reinterpret_cast<uint32_t *>(all);
    const int lane = threadIdx.x & 31, warps = kCountThreads / 32, n4 = (p.tokens + 3) / 4;
    wait_for_predecessor();
    allow_successor_launch();
    if (blockIdx.x >= p.count_blocks) {
        zero_rows(p, blockIdx.x - p.count_blocks, gridDim.x - p.count_blocks);
        return;
    }
    if (blockIdx.x == 0 && threadIdx.x < 2)
        p.counts[threadIdx.x] = 0;
    for (int i0 = threadIdx.x; i0 < 4 * n4; i0 += 8 * kCountThreads) {
        uint32_t id[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = i0 + j * kCountThreads;
            id[j] = i < p.tokens ? id_at(p.ids, p.id_bytes, i, p.vocab) : ~0u;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (i0 + j * kCountThreads < 4 * n4)
                ids[i0 + j * kCountThreads] = id[j];
    }
    __syncthreads();
    for (int t = blockIdx.x * warps + (threadIdx.x >> 5); t < p.tokens; t += p.count_blocks * warps) {
        const uint32_t id = ids[t];
        int before = 0;
        // ids up to its own before the four where it is, ids below its own from there on
#pragma unroll 4
        for (int i = lane; i < n4; i += 32) {
            const uint4 v = all[i];
            const uint32_t end = id + (i < t / 4);
            before += (v.x < end) + (v.y < end) + (v.z < end) + (v.w < end);
        }
        for (int i = t / 4 * 4; i < t; ++i)
            before += lane == 0 && ids[i] == id;
        before = __reduce_add_sync(~0u, before);
        if (lane == 0)
            p.to[before] = make_uint2(id, (uint32_t)t);
    }
}

// -------------------------------------------------------------------- the sums

// The first of the n sorted entries whose id is at least `id`.
__device__ __forceinline__ int64_t lower_bound(const uint2 *order, int64_t n, uint32_t id)
{
    int64_t lo = 0;
    while (n > 0) {
        const int64_t half = n / 2;
        const bool less = order[lo + half].x < id;
        lo = less ? lo + half + 1 : lo;
        n = less ? n - half - 1 : half;
    }
    return lo;
}

template <typename W, int V>
__device__ __forceinline__ void write_row(const EmbedParams &p, uint32_t id, int unit, float (&sum)[V])
{
    W *at = static_cast<W *>(p.table) + id * p.table_stride + (int64_t)unit * V;
    Vec<W, V> r;
#pragma unroll
    for (int e = 0; e < V; ++e)
        sum[e] *= p.scale;
    if (p.accumulate) {
        float old[V];
        load(r, at);
        widen(r, old);
#pragma unroll
        for (int e = 0; e < V; ++e)
            sum[e] += old[e];
    }
    narrow(sum, r);
    store(r, at);
}

template <int BYTES> __device__ __forceinline__ void copy_async(uint32_t to, const void *from)
{
    if constexpr (BYTES == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from), "n"(BYTES) : "memory");
}

// The first blocks write zeros to the rows without a token, zero_rows of them a warp; the last
// sum_blocks sum chunks of sorted tokens, a warp 32 vectors of the row.
//
// The ring holds kSumAhead rows' parts on their way for every warp without registers: 16384
// tokens of 768 and 65536 of 4096, forward and gradient, took 68 and 443 us with eight rows
// in registers, 67 and 414 with eight in the ring, 69 and 426 with sixteen (with all that follows
// 65 and 397).
template <typename W, typename O, int V, int M>
__global__ void __launch_bounds__(kSumThreads) rikfad_embed_sum_kernel(const __grid_constant__ EmbedParams p)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    wait_for_predecessor();
    allow_successor_launch();
    // zeros first: their blocks begin with a search, during which the others' loads are under way
    const int64_t zero_blocks = gridDim.x - p.sum_blocks;
    if (blockIdx.x < zero_blocks) {
        const int64_t row0 = ((int64_t)blockIdx.x * kSumWarps + warp) * p.zero_rows, row = row0 + lane;
        bool absent = false;
        if (lane < p.zero_rows && row < p.zero_from) {
            const int64_t at = lower_bound(p.order, p.tokens, (uint32_t)row);
            absent = at == p.tokens || p.order[at].x != row;
        }
        uint32_t todo = __ballot_sync(~0u, absent);
        for (; todo; todo &= todo - 1)
            zero(static_cast<W *>(p.table) + (row0 + __ffs(todo) - 1) * p.table_stride, p.width, lane, 32);
        return;
    }
    const int64_t item = (blockIdx.x - zero_blocks) * kSumWarps + warp, chunk = item / p.slabs;
    if (chunk >= p.chunks)
        return;
    const int unit = (int)(item % p.slabs) * 32 * M + lane;         // and every 32nd after it, M in all
    const int first_unit = unit - lane, here_units = min(32 * M, p.units - first_unit);
    auto active = [&](int m) { return unit + 32 * m < p.units; };
    const int64_t first = chunk * p.chunk, last = min(first + p.chunk, p.tokens);
    const O *rows = static_cast<const O *>(p.rows) + (int64_t)unit * V;
    uint32_t run = p.order[first].x;
    bool from_before = first > 0 && p.order[first - 1].x == run;
    const uint32_t after = last < p.tokens ? p.order[last].x : ~0u;
    float sum[M][V];
    auto clear = [&] {
#pragma unroll
        for (int m = 0; m < M; ++m) {
#pragma unroll
            for (int e = 0; e < V; ++e)
                sum[m][e] = 0.f;
        }
    };
    clear();
    auto finish = [&](bool goes_on) {
        if (run < p.vocab) {
#pragma unroll
            for (int m = 0; m < M; ++m) {
                if (!active(m))
                    continue;
                if (from_before || goes_on) {
                    float *part = (from_before ? p.head : p.tail) + chunk * p.pitch + (int64_t)(unit + 32 * m) * V;
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        part[e] = sum[m][e];
                } else
                    write_row<W, V>(p, run, unit + 32 * m, sum[m]);
            }
            if (unit == 0 && goes_on && !from_before) {     // a run over several chunks starts here
                const int64_t far = chunk + kShortRun + 1;
                const int longer = far < p.chunks && p.order[far * p.chunk].x == run;
                const int at = atomicAdd(p.counts + longer, 1);     // in any order: each writes its own row
                p.starts[longer ? p.chunks - 1 - at : at] = (int32_t)chunk;
            }
        }
        clear();
        from_before = false;
    };
    auto window = [&](int64_t base) { return base + lane < last ? p.order[base + lane] : make_uint2(~0u, 0); };
    auto step = [&](uint32_t id, const Vec<O, V> (&in)[M]) {
        if (id != run) {
            finish(false);
            run = id;
        }
        if (id < p.vocab) {             // elements beyond the row's end are added up, but not written
#pragma unroll
            for (int m = 0; m < M; ++m) {
                float f[V];
                widen(in[m], f);
#pragma unroll
                for (int e = 0; e < V; ++e)
                    sum[m][e] += f[e];
            }
        }
    };
    // a ring of kSumAhead rows' parts in shared memory
    extern __shared__ uint4 rings[];
    constexpr int kSlot = V > 1 ? 32 * V * (int)sizeof(O) : 32 * M * (int)sizeof(O) + 16;
    char *const ring = reinterpret_cast<char *>(rings) + warp * (kSumAhead * kSlot);
    uint2 mine = window(first), then = window(first + 32);
    auto ask = [&](int j, int slot, const uint2 &entries) {
        const uint32_t id = __shfl_sync(~0u, entries.x, j), token = __shfl_sync(~0u, entries.y, j);
        if (id < p.vocab) {
            const uint32_t to = (uint32_t)__cvta_generic_to_shared(ring + slot * kSlot);
            if constexpr (V > 1) {
                if (active(0))          // each lane's vector, for itself
                    copy_async<V * (int)sizeof(O)>(to + lane * (V * (int)sizeof(O)), rows + token * p.row_stride);
            } else {                    // all of the 16 bytes that the part begins and ends in, wherever that is
                const char *from = reinterpret_cast<const char *>(static_cast<const O *>(p.rows) + token * p.row_stride + first_unit);
                const int skip = (int)((uintptr_t)from % 16), words = (skip + here_units * (int)sizeof(O) + 15) / 16;
                for (int i = lane; i < words; i += 32)
                    copy_async<16>(to + 16 * i, from - skip + 16 * i);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    for (int j = 0; j < kSumAhead - 1; ++j)
        ask(j, j, mine);
    for (int64_t base = first; base < last; base += 32) {
        const int here = (int)min((int64_t)32, last - base);
#pragma unroll(V > 1 ? 4 : 2)
        for (int j = 0; j < here; ++j) {
            const int k = j + kSumAhead - 1;
            ask(k % 32, k % kSumAhead, k < 32 ? mine : then);
            asm volatile("cp.async.wait_group %0;" ::"n"(kSumAhead - 1) : "memory");
            const uint32_t id = __shfl_sync(~0u, mine.x, j);
            const char *at = ring + j % kSumAhead * kSlot;
            Vec<O, V> in[M];
            if constexpr (V > 1)
                in[0].word = *reinterpret_cast<const decltype(in[0].word) *>(at + lane * (V * (int)sizeof(O)));
            else {
                __syncwarp();           // other lanes' copies
                const uint32_t token = __shfl_sync(~0u, mine.y, j);
                at += (uintptr_t)(static_cast<const O *>(p.rows) + token * p.row_stride + first_unit) % 16;
#pragma unroll
                for (int m = 0; m < M; ++m)
                    in[m].v[0] = reinterpret_cast<const O *>(at)[lane + 32 * m];
                __syncwarp();           // before the place is written again
            }
            step(id, in);
        }
        mine = then;
        then = window(base + 64);
    }
    finish(run == after);
}

// Runs over several chunks: the partial row of the chunk where one starts, then those
// of the chunks that it goes on in.  128 columns of a run that goes on in up to kShortRun
// chunks are a warp's, of a longer one a block's.
template <typename W> __global__ void __launch_bounds__(kJoinThreads) rikfad_embed_join_kernel(const __grid_constant__ EmbedParams p)
{
    __shared__ float4 part[kJoinWarps][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, slabs = (int)((p.pitch + 127) / 128);
    wait_for_predecessor();
    allow_successor_launch();
    const int64_t short_runs = (int64_t)p.counts[0] * slabs, long_runs = (int64_t)p.counts[1] * slabs;
    auto add = [](float4 &s, const float4 &v) {
        s.x += v.x;
        s.y += v.y;
        s.z += v.z;
        s.w += v.w;
    };
    // columns from `column` on of the head rows [from, to), added to s
    auto heads = [&](float4 &s, int64_t column, int64_t from, int64_t to) {
        const float *row = p.head + from * p.pitch + column;
        for (int64_t n = to - from; n > 0 && column < p.pitch; n -= kJoinAhead, row += kJoinAhead * p.pitch) {
            float4 v[kJoinAhead];
#pragma unroll
            for (int j = 0; j < kJoinAhead; ++j)
                if (j < n)
                    v[j] = __ldcs(reinterpret_cast<const float4 *>(row + j * p.pitch));
#pragma unroll
            for (int j = 0; j < kJoinAhead; ++j)
                if (j < n)
                    add(s, v[j]);
        }
    };
    auto write = [&](uint32_t id, int64_t column, const float4 &s) {
        const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (column + e < p.width) {
                float one[1] = {v[e]};
                write_row<W, 1>(p, id, (int)(column + e), one);
            }
    };
    const float4 nothing = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int64_t i = blockIdx.x; i < long_runs; i += gridDim.x) {
        const int64_t chunk = p.starts[p.chunks - 1 - i / slabs], column = i % slabs * 128 + lane * 4;
        const uint32_t id = p.order[(chunk + 1) * p.chunk].x;
        int64_t last = chunk + 1 + kShortRun, end = p.chunks;           // the first chunk that does not start with id
        while (last < end) {            // 32 places at a time
            const int64_t step = (end - last + 31) / 32, c = last + lane * step;
            const int same = __popc(__ballot_sync(~0u, c < end && p.order[c * p.chunk].x == id));
            end = min(end, last + same * step);
            last = same ? last + (same - 1) * step + 1 : end;
        }
        const int64_t share = (last - chunk - 1 + kJoinWarps - 1) / kJoinWarps, from = chunk + 1 + share * warp;
        float4 s = warp == 0 && column < p.pitch ? *reinterpret_cast<const float4 *>(p.tail + chunk * p.pitch + column) : nothing;
        heads(s, column, from, min(from + share, last));
        part[warp][lane] = s;
        __syncthreads();
        if (warp == 0) {
            for (int w = 1; w < kJoinWarps; ++w)
                add(s, part[w][lane]);
            write(id, column, s);
        }
        __syncthreads();
    }
    for (int64_t i = (int64_t)blockIdx.x * kJoinWarps + warp; i < short_runs; i += (int64_t)gridDim.x * kJoinWarps) {
        const int64_t chunk = p.starts[i / slabs], column = i % slabs * 128 + lane * 4;
        const uint32_t id = p.order[(chunk + 1) * p.chunk].x;
        const int64_t c = chunk + 1 + lane;
        const uint32_t more = __ballot_sync(~0u, c < p.chunks && p.order[c * p.chunk].x == id);
        float4 s = column < p.pitch ? __ldcs(reinterpret_cast<const float4 *>(p.tail + chunk * p.pitch + column)) : nothing;
        heads(s, column, chunk + 1, chunk + 1 + (more == ~0u ? 32 : __ffs(~more) - 1));
        write(id, column, s);
    }
}

// ------------------------------------------------------------------------ host

int bad(const std::string &msg) { return report_error(RIKFAD_ERR_ARG, msg); }

int check_sizes(const rikfad_embedding *p)
{
    if (p == nullptr)
        return bad("p is NULL");
    if (p->tokens < 0 || p->tokens > (int64_t)1 << 30 || p->vocab < 0 || p->vocab > (int64_t)1 << 30)
        return bad("tokens and vocab must be in [0, 2^30]");
    if (p->width < 1 || p->width > 1 << 20)
        return bad("width must be in [1, 2^20]");
    if (!dtype_ok(p->table_dtype) || !dtype_ok(p->dtype))
        return bad("table_dtype and dtype must be a rikfad_dtype");
    if (p->id_bytes != 4 && p->id_bytes != 8)
        return bad("id_bytes must be 4 or 8");
    if (!std::isfinite(p->scale) || !std::isfinite((float)p->scale))
        return bad("scale must be finite");
    return RIKFAD_OK;
}

int check_rows(const rikfad_rows &r, const char *name, int dtype, int64_t rows, int64_t width, int device)
{
    if (rows == 0)
        return RIKFAD_OK;
    if (r.data == nullptr)
        return bad(std::string(name) + " is NULL");
    if (rows > 1 && (r.stride < width || r.stride > (int64_t)1 << 32))
        return bad(std::string("the row stride of ") + name + " must be at least width");
    if ((uintptr_t)r.data % (uintptr_t)dtype_bytes(dtype))
        return report_error(RIKFAD_ERR_ALIGN, std::string(name) + " is not aligned to its element type");
    return check_address(r.data, device, name);
}

int check(const rikfad_embedding *p, int &device)
{
    int rc = check_sizes(p);
    if (rc)
        return rc;
    const cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess)
        return report_cuda(e, "cudaGetDevice");
    if (p->tokens > 0) {
        if (p->ids == nullptr)
            return bad("ids is NULL");
        if ((uintptr_t)p->ids % (uintptr_t)p->id_bytes)
            return report_error(RIKFAD_ERR_ALIGN, "ids is not aligned");
        rc = check_address(p->ids, device, "ids");
    }
    if (!rc) rc = check_rows(p->table, "table", p->table_dtype, p->vocab, p->width, device);
    if (!rc) rc = check_rows(p->rows, "rows", p->dtype, p->tokens, p->width, device);
    return rc;
}

// Vectors of 16 bytes in the wider type where the width, the strides and the addresses
// allow them, else single elements.
int vector_of(const rikfad_embedding *p)
{
    const int tb = dtype_bytes(p->table_dtype), rb = dtype_bytes(p->dtype);
    uint64_t parts = (uint64_t)p->width | (uint64_t)(uintptr_t)p->table.data / tb | (uint64_t)(uintptr_t)p->rows.data / rb;
    if (p->vocab > 1)
        parts |= (uint64_t)p->table.stride;
    if (p->tokens > 1)
        parts |= (uint64_t)p->rows.stride;
    const int v = 16 / std::max(tb, rb);
    return parts % v ? 1 : v;
}

EmbedParams params(const rikfad_embedding *p)
{
    EmbedParams e{};
    e.ids = p->ids;
    e.table = p->table.data;
    e.rows = p->rows.data;
    e.table_stride = p->vocab > 1 ? p->table.stride : 0;
    e.row_stride = p->tokens > 1 ? p->rows.stride : 0;
    e.tokens = p->tokens;
    e.vocab = p->vocab;
    e.width = (int32_t)p->width;
    e.id_bytes = p->id_bytes;
    e.accumulate = p->accumulate;
    e.scale = (float)p->scale;
    return e;
}

template <typename W, typename O, int V> cudaError_t launch_forward(EmbedParams p, cudaStream_t s)
{
    if constexpr (V == 1) {
        p.slabs = (p.width + kNarrowColumns - 1) / kNarrowColumns;
        const int64_t items = (p.tokens + kForwardRows - 1) / kForwardRows * p.slabs, warps = kNarrowThreads / 32;
        const int64_t blocks = (items + warps - 1) / warps;
        if (blocks > INT32_MAX)
            return cudaErrorInvalidConfiguration;
        return launch_chained(rikfad_embed_forward_narrow_kernel<W, O>, dim3((unsigned)blocks), kNarrowThreads, 0, s, p);
    } else {
        p.units = p.width / V;
        int lanes = 32;
        while (lanes < kForwardThreads && lanes < p.units)
            lanes *= 2;
        const int rows = kForwardThreads / lanes;
        const int64_t blocks = (p.tokens + rows * kForwardRows - 1) / (rows * kForwardRows);
        // few rows: several blocks for each
        const int64_t most = (p.units + lanes - 1) / lanes;
        const int64_t across = std::max<int64_t>(1, std::min<int64_t>(most, 4 * kSms / blocks));
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)blocks, (unsigned)across);
        cfg.blockDim = dim3((unsigned)lanes, (unsigned)rows);
        cfg.stream = s;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        return cudaLaunchKernelEx(&cfg, rikfad_embed_forward_kernel<W, O, V>, p);
    }
}

cudaError_t launch_sort(const SortParams &p, cudaStream_t s)
{
    const int bins = 1 << p.bits;
    cudaLaunchConfig_t cfg = {};
    // the other multiprocessors write zeros
    const int others = p.zero_from < p.vocab ? kSms / kSortCtas - 1 : 0;
    cfg.gridDim = dim3(kSortCtas * (1 + others));
    cfg.blockDim = dim3(kSortThreads);
    cfg.dynamicSmemBytes = sizeof(uint32_t) * (3 * bins + 32) + sizeof(uint16_t) * kSortWarps * bins;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = kSortCtas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, rikfad_embed_sort_kernel, p);
}

struct Workspace {
    int64_t chunk, chunks, pitch;
    size_t entries, lists, bytes;       // bytes of one list of entries, of the chunks where runs start, of all
};

Workspace workspace_of(const rikfad_embedding *p)
{
    Workspace w;
    // Chunks of more tokens leave fewer partial rows, as long as there are warps enough, of
    // 512 bytes of a row each: some to have work at all (4099 tokens of 1001, forward and
    // gradient: 47 us with 32 a chunk, 37 with 8), many before partial rows are few.
    const int64_t slabs = (p->width * dtype_bytes(p->dtype) + 511) / 512;
    w.chunk = 8;
    while (w.chunk < 256 && p->tokens / w.chunk * slabs > kSms * (w.chunk < 32 ? 16 : 96))
        w.chunk *= 2;
    w.chunks = (p->tokens + w.chunk - 1) / w.chunk;
    w.pitch = (p->width + 3) / 4 * 4;
    w.entries = ((size_t)p->tokens * sizeof(uint2) + 15) / 16 * 16;
    w.lists = p->tokens ? ((size_t)w.chunks + 2 + 3) / 4 * 4 * sizeof(int32_t) : 0;
    w.bytes = 2 * w.entries + w.lists + 2 * (size_t)w.chunks * (size_t)w.pitch * sizeof(float);
    return w;
}

template <typename W, typename O, int V> cudaError_t launch_backward(EmbedParams p, cudaStream_t s)
{
    p.units = p.width / V;
    constexpr int M = V > 1 ? 1 : 16 / (int)sizeof(O);      // vectors of a lane
    p.slabs = (p.units + 32 * M - 1) / (32 * M);
    p.sum_blocks = (p.chunks * p.slabs + kSumWarps - 1) / kSumWarps;
    p.zero_rows = 32;                   // some 32 KB
    while (p.zero_rows > 1 && p.zero_rows * (int64_t)p.width * (int64_t)sizeof(W) > 32 << 10)
        p.zero_rows /= 2;
    const int64_t zeros = (p.zero_from + p.zero_rows * kSumWarps - 1) / (p.zero_rows * kSumWarps);
    if (p.sum_blocks + zeros == 0)
        return cudaSuccess;
    if (p.sum_blocks + zeros > INT32_MAX)
        return cudaErrorInvalidConfiguration;
    cudaError_t e = launch_chained(rikfad_embed_sum_kernel<W, O, V, M>, dim3((unsigned)(p.sum_blocks + zeros)), kSumThreads,
                                   (size_t)kSumAhead * kSumWarps * (V > 1 ? 32 * V * sizeof(O) : 528), s, p);
    if (e != cudaSuccess || p.chunks < 2)
        return e;
    const int64_t slabs = (p.pitch + 127) / 128, blocks = (p.chunks * slabs + kJoinWarps - 1) / kJoinWarps;
    return launch_chained(rikfad_embed_join_kernel<W>, dim3((unsigned)std::min<int64_t>(blocks, kJoinBlocks)), kJoinThreads, 0, s, p);
}

template <typename W, typename O, bool BACKWARD, int V> cudaError_t launch(const EmbedParams &p, int v, cudaStream_t s)
{
    if constexpr (V > 1)
        if (v < V)
            return launch<W, O, BACKWARD, 1>(p, v, s);
    if constexpr (BACKWARD)
        return launch_backward<W, O, V>(p, s);
    else
        return launch_forward<W, O, V>(p, s);
}

template <typename W, bool BACKWARD> cudaError_t launch(const EmbedParams &p, int dtype, int v, cudaStream_t s)
{
    constexpr int kNarrow = sizeof(W) == 2 ? 8 : 4;
    return dtype == RIKFAD_F32    ? launch<W, float, BACKWARD, 4>(p, v, s)
           : dtype == RIKFAD_BF16 ? launch<W, __nv_bfloat16, BACKWARD, kNarrow>(p, v, s)
                                  : launch<W, __half, BACKWARD, kNarrow>(p, v, s);
}

template <bool BACKWARD> cudaError_t launch(const rikfad_embedding *d, const EmbedParams &p, cudaStream_t s)
{
    const int v = vector_of(d);
    return d->table_dtype == RIKFAD_F32    ? launch<float, BACKWARD>(p, d->dtype, v, s)
           : d->table_dtype == RIKFAD_BF16 ? launch<__nv_bfloat16, BACKWARD>(p, d->dtype, v, s)
                                           : launch<__half, BACKWARD>(p, d->dtype, v, s);
}

}  // namespace

extern "C" {

RIKFAD_API size_t rikfad_embedding_workspace(const rikfad_embedding *p)
{
    RK_ENTRY_BEGIN
    if (check_sizes(p))
        return 0;
    report_error(RIKFAD_OK, "");
    return workspace_of(p).bytes;
    }
    catch (...)
    {
        return 0;
    }
}

RIKFAD_API int rikfad_embedding_forward(const rikfad_embedding *p, void *stream)
{
    RK_ENTRY_BEGIN
    int device = -1;
    const int rc = check(p, device);
    if (rc)
        return rc;
    cudaError_t e = cudaPeekAtLastError();
    if (e != cudaSuccess)
        return report_cuda(e, "earlier CUDA error");
    if (p->tokens == 0)
        return RIKFAD_OK;
    e = launch<false>(p, params(p), (cudaStream_t)stream);
    return e == cudaSuccess ? RIKFAD_OK : report_cuda(e, "launch rikfad_embed_forward_kernel");
    RK_ENTRY_END
}

RIKFAD_API int rikfad_embedding_backward(const rikfad_embedding *p, void *stream)
{
    RK_ENTRY_BEGIN
    int device = -1;
    int rc = check(p, device);
    if (rc)
        return rc;
    const Workspace w = workspace_of(p);
    if (w.bytes > 0) {
        if (p->workspace == nullptr || p->workspace_bytes < w.bytes)
            return bad("the workspace is smaller than rikfad_embedding_workspace");
        if ((uintptr_t)p->workspace % 16)
            return report_error(RIKFAD_ERR_ALIGN, "workspace is not aligned");
        rc = check_address(p->workspace, device, "workspace");
        if (rc)
            return rc;
    }
    cudaError_t e = cudaPeekAtLastError();
    if (e != cudaSuccess)
        return report_cuda(e, "earlier CUDA error");
    if (p->vocab == 0)
        return RIKFAD_OK;
    EmbedParams q = params(p);
    char *at = static_cast<char *>(p->workspace);
    q.order = reinterpret_cast<uint2 *>(at);
    q.counts = reinterpret_cast<int32_t *>(at + 2 * w.entries);
    q.starts = q.counts + 2;
    q.head = reinterpret_cast<float *>(at + 2 * w.entries + w.lists);
    q.tail = q.head + w.chunks * w.pitch;
    q.chunk = (int32_t)w.chunk;
    q.chunks = w.chunks;
    q.pitch = w.pitch;
    q.zero_from = p->accumulate ? 0 : p->vocab;
    const cudaStream_t s = (cudaStream_t)stream;
    if (p->tokens > 0) {
        SortParams r{};
        // While a few multiprocessors sort, the others write zeros to the last rows of the
        // table, about as many as that time allows; those with tokens are written again.
        // To all rows where tokens are few to them: what is written twice is an eighth at most.
        if (!p->accumulate && p->tokens <= p->vocab / 8)
            q.zero_from = 0;
        else if (!p->accumulate) {
            const double us = p->tokens <= kMostCounted ? 3 : 9 + (double)p->tokens / 2800;      // 12.3 at 8192, 32.7 at 65536
            const double rows = us * kZeroBytesPerUs / ((double)p->width * dtype_bytes(p->table_dtype));
            q.zero_from = p->vocab - (int64_t)std::min((double)p->vocab, rows);
        }
        r.zero_from = p->accumulate ? p->vocab : q.zero_from;
        r.counts = q.counts;
        r.table = q.table;
        r.table_stride = q.table_stride;
        r.width = q.width;
        r.table_bytes = dtype_bytes(p->table_dtype);
        r.ids = p->ids;
        r.to = q.order;
        r.from = reinterpret_cast<uint2 *>(at + w.entries);
        r.vocab = p->vocab;
        r.tokens = (int32_t)p->tokens;
        r.id_bytes = p->id_bytes;
        int bits = 1;                   // of ids up to vocab
        while (p->vocab >> bits)
            ++bits;
        r.passes = (bits + kSortBits - 1) / kSortBits;
        r.bits = (bits + r.passes - 1) / r.passes;
        r.count_blocks = (int32_t)std::min<int64_t>(2 * kSms, (p->tokens + 7) / 8);
        const int zero_blocks = r.zero_from < p->vocab ? 6 * kSms : 0;
        e = p->tokens <= kMostCounted
                ? launch_chained(rikfad_embed_count_kernel, dim3((unsigned)(r.count_blocks + zero_blocks)), kCountThreads, 0, s, r)
                : launch_sort(r, s);
        if (e != cudaSuccess)
            return report_cuda(e, "launch of the embedding's sort");
    }
    e = launch<true>(p, q, s);
    return e == cudaSuccess ? RIKFAD_OK : report_cuda(e, "launch of the embedding's backward kernels");
    RK_ENTRY_END
}

}  // extern "C"
