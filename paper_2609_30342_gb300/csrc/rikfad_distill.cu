// rikfad_distill.cu -- loss of rows of logits s against a teacher's top logits t at
// indices i and a label, and its gradient:
//   p = softmax(t / T), q_T = softmax(s / T), q_1 = softmax(s)
//   loss = a T^2 sum_k p_k (log p_k - log q_T[i_k]) - b log q_1[label]
//   ds = g (a T (q_T - p) + b (q_1 - e_label))
//
// Everything is in powers of two of x c - r, with c = log2(e) / T (or log2(e)) and a
// reference r = m c that is rounded once and used alike for sums, losses and gradients:
// its rounding cancels.  m is the largest of some of the row's elements, of every thread's
// first vector; where a thread's sum shows that this is too low for its others (by 40 powers
// of two), the largest of all of its elements.
//
// Memory bounds it: the logits are read once for the sums, once more, from the L2 cache,
// for the gradient, and the gradient is written once.  8192 rows of 50257 in bfloat16 at
// two temperatures take 305 us (1.65 GB, 5.4 TB/s; four powers an element, which alone
// take 180), of 131072 at one 726 (4.3 GB, 5.9 TB/s); cross entropy of 50257 276.  Rows go
// element by element, at several times that, where they have no term, where a thread's first
// vector is masked, and where rows of the gradient start elsewhere than the logits'.
#include <cuda_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <new>
#include <string>
#include <type_traits>

#include "rikfad.h"
#include "rikfad_host.hpp"
#include "rikfad_kernels.cuh"
#include "rikfad_pairs.cuh"
#include "rikfad_types.cuh"

using namespace rikfad;

namespace {

constexpr int kMaxThreads = 256;
constexpr int kSms = 152;
constexpr int kMaxEntries = 1024;           // of a teacher's row
constexpr int kMaxCluster = 8;
constexpr int64_t kUnderWay = 64 << 20;      // bytes of rows that blocks have at one time, of 129 MB of L2
constexpr int kBlocksPerSm = 4;
constexpr int kSmemPerSm = 228 << 10;
// A reference's rounding is a factor of up to 2^(r 2^-24) in every power: r stays below
// this, and lower logits count as the one there.
constexpr float kFarthest = 0x1p29f;
// A named element below it (a type's lowest value; its product with c may leave float32's range) adds x c to a log share
// that is less than 2^-60 of that beside it.
constexpr float kRemote = -0x1p100f;
constexpr float kLargestSum = 0x1p40f;      // of a thread, beyond which its reference is too low
constexpr int kEntriesAhead = 4;            // entries of a lane under way
constexpr int kAhead = 4;                      // vectors of a thread under way

struct Params {
    const void *logits, *teacher, *index, *labels;
    void *dlogits;
    const float *dloss;
    float *loss;
    float4 *stats;                  // r and sum at temperature T, r and sum at 1
    int64_t rows, logits_stride, teacher_stride, index_stride, dlogits_stride;
    int32_t vocab, k, teacher_dtype, index_bytes, label_bytes;
    int32_t cluster;                // blocks of a row
    int32_t names;                  // places of the table of indices
    bool distils, labelled;         // the terms that the call has
    bool wide;                      // every row of dlogits starts as far from 16 bytes as the logits'
    float a, b;                     // a T and b, of the gradient
    float loss_a, loss_b;           // a T^2 ln 2 and b ln 2
    float c_t, c_1, grad_scale;     // log2(e) / T, log2(e)
    float lowest;                   // finite logits below it count as it
    float lowest_t, lowest_1;       // references below which a row has nothing else
};

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ f2 exp2_fast(f2 p)
{
    float x, y;
    apart(p, x, y);
    return pair(exp2_fast(x), exp2_fast(y));
}

// The largest of a vector's elements; NaN is passed over.
template <typename T, int V> __device__ __forceinline__ float largest(const Vec<T, V> &r)
{
    if constexpr (sizeof(T) == 2) {
        using T2 = std::conditional_t<std::is_same_v<T, __half>, __half2, __nv_bfloat162>;
        T2 m = *reinterpret_cast<const T2 *>(&r.pairs[0]);
#pragma unroll
        for (int i = 1; i < V / 2; ++i)
            m = __hmax2(m, *reinterpret_cast<const T2 *>(&r.pairs[i]));
        return fmaxf(to_f32(m.x), to_f32(m.y));
    } else {
        float m = r.v[0];
#pragma unroll
        for (int i = 1; i < V; ++i)
            m = fmaxf(m, r.v[i]);
        return m;
    }
}

__device__ __forceinline__ int64_t integer_at(const void *p, int bytes, int64_t i)
{
    return bytes == 4 ? (int64_t)static_cast<const int32_t *>(p)[i] : static_cast<const int64_t *>(p)[i];
}

__device__ __forceinline__ float float_at(const void *p, int dtype, int64_t i)
{
    return dtype == RIKFAD_F32    ? static_cast<const float *>(p)[i]
           : dtype == RIKFAD_BF16 ? to_f32(static_cast<const __nv_bfloat16 *>(p)[i])
                                  : to_f32(static_cast<const __half *>(p)[i]);
}

__device__ __forceinline__ float at_least(float x, float lowest) { return x < lowest && x > -INFINITY ? lowest : x; }

__device__ __forceinline__ float reference(float top, float c)
{
    const float r = top * c;
    return top == -INFINITY ? 0.f : r > kFarthest ? INFINITY : r;
}

// A row's element as it counts in sums: not below the lowest value.
template <typename T> __device__ __forceinline__ float element(const T *row, int i, float lowest)
{
    return to_f32(from_f32<T>(at_least(to_f32(row[i]), lowest)));
}

// What a part's sum counts for a larger maximum.
__device__ __forceinline__ float moved(float sum, float from, float to, float c)
{
    return sum == 0.f ? 0.f : sum * exp2_fast(reference(from, c) - reference(to, c));
}

// A maximum and the sums of 2^(x c - r), r = max c, at two temperatures (BOTH) or one.
template <bool BOTH> struct Sums {
    float top = -INFINITY, t = 0.f, one = 0.f;

    __device__ __forceinline__ void add(float x, float sum_t, float sum_1, float c_t, float c_1)
    {
        const float m = fmaxf(top, x);
        t = moved(t, top, m, c_t) + moved(sum_t, x, m, c_t);
        if (BOTH)
            one = moved(one, top, m, c_1) + moved(sum_1, x, m, c_1);
        top = m;
    }
    __device__ __forceinline__ void add_one(float x, float c_t, float c_1)
    {
        add(x, exp2_fast(fmaf(x, c_t, -reference(x, c_t))), exp2_fast(fmaf(x, c_1, -reference(x, c_1))), c_t, c_1);
    }
    // Those of the warp's lanes together, in all of them.
    __device__ __forceinline__ void join(float c_t, float c_1)
    {
        float m = top;
#pragma unroll
        for (int d = 16; d > 0; d /= 2)
            m = fmaxf(m, __shfl_xor_sync(~0u, m, d));
        t = moved(t, top, m, c_t);
        if (BOTH)
            one = moved(one, top, m, c_1);
        top = m;
#pragma unroll
        for (int d = 16; d > 0; d /= 2) {
            t += __shfl_xor_sync(~0u, t, d);
            if (BOTH)
                one += __shfl_xor_sync(~0u, one, d);
        }
    }
};

__device__ __forceinline__ void cluster_arrive_relaxed()
{
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_arrive()
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait()
{
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_write(const float *mine, int rank, float v)
{
    uint32_t at;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(mine)), "r"(rank));
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(v) : "memory");
}

// The part of a row that a block has: vectors of 16 bytes [begin, end) between the
// row's first and last elements outside whole vectors, which block 0 has.
template <typename T> struct Slice {
    static constexpr int V = 16 / sizeof(T);
    int lead, vectors, begin, end, share, edges;

    __device__ __forceinline__ Slice(const T *row, int vocab, int cluster, int rank)
    {
        lead = min((int)((16 - (uint32_t)(uintptr_t)row % 16) % 16 / sizeof(T)), vocab);
        vectors = (vocab - lead) / V;
        share = (vectors + cluster - 1) / cluster;
        begin = min(rank * share, vectors);
        end = min(begin + share, vectors);
        edges = rank == 0 ? vocab - vectors * V : 0;
    }
    __device__ __forceinline__ int edge(int i) const { return i < lead ? i : i + vectors * V; }
    __device__ __forceinline__ bool has(int element, int rank) const
    {
        const int v = element - lead;
        return v < 0 || v >= vectors * V ? rank == 0 : v / V >= begin && v / V < end;
    }
};

// forward: losses and statistics; fused: the gradient as well; backward: the gradient
// from the statistics.
enum Mode { kForward, kFused, kBackward };

// A row's entries in shared memory: log2 of the teacher's shares, the row's logits at
// the indices and the indices; one that is absent, or whose logit is -inf, has index
// -1.  The label is the last.
struct Entries {
    float *log_p, *at_index;
    int *index, *names;
    int terms;                  // which the row has: 1 the teacher's, 2 the label's
    bool repeated;              // some of the teacher's in the block's slice name one element

    __device__ __forceinline__ Entries(float *at, int count)
        : log_p(at), at_index(at + count), index(reinterpret_cast<int *>(at + 2 * count)), names(index + count), terms(0), repeated(false)
    {
    }
};

// One warp loads row r's entries.  They are the longest chain of a block, two loads after
// one another: with one round of them for every 32 entries 8192 rows of 131072 with 128
// entries took 1456 us instead of 1085.  Entries that name one element are rare but for
// the label's; comparing all pairs for them cost 200 us of 1065.
template <typename T>
__device__ __forceinline__ void load_entries(const Params &p, Entries &to, int64_t r, const Slice<T> &slice, int rank, bool gradient)
{
    const int lane = threadIdx.x & 31;
    const T *row = static_cast<const T *>(p.logits) + r * p.logits_stride;
    Sums<false> shares;
    bool present = false;
    const int64_t wanted = lane == 0 && p.labelled ? integer_at(p.labels, p.label_bytes, r) : -1;
    const bool label = wanted >= 0 && wanted < p.vocab;
    const int k = p.distils ? p.k : 0;
    // all of a round's loads before the first one's use: a warp waits twice for kEntriesAhead x 32 entries
    for (int e0 = lane; e0 < k; e0 += 32 * kEntriesAhead) {
        int64_t i[kEntriesAhead];
        float t[kEntriesAhead], x[kEntriesAhead];
#pragma unroll
        for (int j = 0; j < kEntriesAhead; ++j) {
            const int e = e0 + 32 * j;
            i[j] = e < k ? integer_at(p.index, p.index_bytes, r * p.index_stride + e) : -1;
            t[j] = e < k ? float_at(p.teacher, p.teacher_dtype, r * p.teacher_stride + e) : 0.f;
        }
#pragma unroll
        for (int j = 0; j < kEntriesAhead; ++j) {
            i[j] = i[j] < p.vocab && t[j] != -INFINITY ? i[j] : -1;
            x[j] = i[j] >= 0 ? to_f32(row[i[j]]) : 0.f;
        }
        float top = shares.top;
#pragma unroll
        for (int j = 0; j < kEntriesAhead; ++j) {
            const int e = e0 + 32 * j;
            t[j] = at_least(t[j], p.lowest);
            present = present || i[j] >= 0;
            top = i[j] >= 0 ? fmaxf(top, t[j]) : top;
            if (e < k) {
                to.index[e] = i[j] >= 0 ? (int)i[j] : -1;
                to.log_p[e] = t[j];
                to.at_index[e] = x[j];
            }
        }
        const float from = reference(top, p.c_t);
        shares.t = moved(shares.t, shares.top, top, p.c_t);
        shares.top = top;
#pragma unroll
        for (int j = 0; j < kEntriesAhead; ++j)
            shares.t += i[j] >= 0 ? exp2_fast(fmaf(t[j], p.c_t, -from)) : 0.f;
    }
    if (lane == 0) {
        to.index[p.k] = label ? (int)wanted : -1;
        to.at_index[p.k] = label ? to_f32(row[wanted]) : 0.f;
    }
    to.terms = (__any_sync(~0u, present) ? 1 : 0) | (__any_sync(~0u, label) ? 2 : 0);
    if (to.terms & 1) {
        shares.join(p.c_t, p.c_1);
        const float from = reference(shares.top, p.c_t), log_sum = log2f(shares.t);
        for (int e = lane; e < k; e += 32)
            to.log_p[e] = fmaf(to.log_p[e], p.c_t, -from) - log_sum;
    }
    __syncwarp();
    if (gradient && (to.terms & 1)) {
        // whether entries of the slice name one element: a hash table of their indices
        const int size = 2 << (31 - __clz(k));          // more than k, at most 2 k
        for (int n = lane; n < size; n += 32)
            to.names[n] = -1;
        __syncwarp();
        bool met = false;
        for (int e = lane; e < k; e += 32) {
            const int i = to.index[e];
            if (i < 0 || !slice.has(i, rank))
                continue;
            // indices are often evenly spaced: a multiplicative hash.  Ends: fewer names than places
            for (int n = (uint32_t)i * 2654435769u >> __clz(k);; n = (n + 1) & (size - 1)) {
                const int there = atomicCAS(to.names + n, -1, i);
                met = met || there == i;
                if (there == -1 || there == i)
                    break;
            }
        }
        to.repeated = __any_sync(~0u, met);
    }
}

// A row's block, or cluster of blocks, reads it for the sums and, from the L2 cache, again for the
// gradient.  The last warp has the entries as well.  BOTH: the two temperatures differ.
//
// Blocks are small and many, so that one's sums, its barrier and its entries' two rounds of
// loads lie over another's gradient: 8192 x 50257 took 573 us with 512 threads a block and 404
// with 256 (before the entries' table), 8192 x 131072 939 with two blocks a row and 727 with
// four, whose rows stay in L2.  Rows held in shared memory between the two readings were slower
// (452 and 1085 us): clusters' barriers and too few warps cost more than the second reading.
// The prefetch of a block's whole part took 8192 x 50257 from 336 to 315 us (305 since).
template <typename T, Mode MODE, bool BOTH>
__global__ void __launch_bounds__(kMaxThreads) rikfad_distill_kernel(const __grid_constant__ Params p)
{
    constexpr int V = 16 / sizeof(T);
    extern __shared__ float shared[];
    __shared__ int terms;
    const int threads = blockDim.x, warps = threads >> 5, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int rank = p.cluster > 1 ? (int)(blockIdx.x % p.cluster) : 0;
    const int64_t r = p.cluster > 1 ? blockIdx.x / p.cluster : blockIdx.x;
    const bool last_warp = warp == warps - 1;
    Entries entries(shared, p.k + 1);
    float *const parts = shared + 3 * (p.k + 1) + p.names;  // three of every warp of the row
    wait_for_predecessor();
    allow_successor_launch();
    if (MODE != kBackward && p.cluster > 1)
        cluster_arrive_relaxed();                           // this block has begun
    const T *row = static_cast<const T *>(p.logits) + r * p.logits_stride;
    const Slice<T> slice(row, p.vocab, p.cluster, rank);
    const uint4 *vectors = reinterpret_cast<const uint4 *>(row + slice.lead) + slice.begin;
    const int mine = slice.end - slice.begin;
    if (threadIdx.x == 0 && mine > 0)           // the part under way, up to 256 KB: more than the loads below ask for at once
        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(vectors), "r"(min(mine, 16384) * 16));
    if (last_warp) {
        load_entries<T>(p, entries, r, slice, rank, MODE != kForward);
        if (lane == 0)
            terms = entries.terms;
    }
    float r_t, r_1, sum_t, sum_1;
    if (MODE != kBackward) {
        // This thread's reference and sums.  Any element not far below the others does for a
        // reference, and the largest of the first vector hardly ever is; if it was, or if
        // that vector is masked, the thread goes over its part again and looks for the largest.
        Sums<BOTH> sums;
        if (threadIdx.x < mine) {
            f2 of_t = pair(0.f, 0.f), of_1 = pair(0.f, 0.f);
            float minus_t = 0.f, minus_1 = 0.f;
            for (int v = threadIdx.x; v < mine; v += threads * kAhead) {
                Vec<T, V> in[kAhead];
#pragma unroll
                for (int j = 0; j < kAhead; ++j)
                    if (v + j * threads < mine)
                        in[j].word = vectors[v + j * threads];
                if (v == threadIdx.x) {
                    sums.top = largest(in[0]);
                    minus_t = -reference(sums.top, p.c_t);
                    minus_1 = -reference(sums.top, p.c_1);
                }
#pragma unroll
                for (int j = 0; j < kAhead; ++j)
                    if (v + j * threads < mine) {
                        float x[V];
                        widen(in[j], x);
#pragma unroll
                        for (int e = 0; e < V; e += 2) {
                            const f2 both = pair(x[e], x[e + 1]);
                            of_t = add(of_t, exp2_fast(fma(both, pair(p.c_t, p.c_t), pair(minus_t, minus_t))));
                            if (BOTH)
                                of_1 = add(of_1, exp2_fast(fma(both, pair(p.c_1, p.c_1), pair(minus_1, minus_1))));
                        }
                    }
            }
            float even, odd;
            apart(of_t, even, odd);
            sums.t = even + odd;
            apart(of_1, even, odd);
            sums.one = even + odd;
            if (!(sums.top > p.lowest && sums.t < kLargestSum && sums.one < kLargestSum)) {
                sums = Sums<BOTH>();
                for (int v = threadIdx.x; v < mine; v += threads) {
#pragma unroll 1
                    for (int e = 0; e < V; ++e)
                        sums.add_one(element<T>(row, slice.lead + (slice.begin + v) * V + e, p.lowest), p.c_t, p.c_1);
                }
            }
        }
        if (threadIdx.x < slice.edges)
            sums.add_one(element<T>(row, slice.edge(threadIdx.x), p.lowest), p.c_t, p.c_1);
        sums.join(p.c_t, p.c_1);
        // every warp's to all blocks of the row, where every warp adds them up
        if (p.cluster > 1) {
            cluster_wait();
            if (lane < p.cluster) {
                float *to = parts + 3 * (rank * warps + warp);
                cluster_write(to, lane, sums.top);
                cluster_write(to + 1, lane, sums.t);
                cluster_write(to + 2, lane, sums.one);
            }
            cluster_arrive();
            cluster_wait();
        } else {
            if (lane == 0) {
                parts[3 * warp] = sums.top;
                parts[3 * warp + 1] = sums.t;
                parts[3 * warp + 2] = sums.one;
            }
            __syncthreads();
        }
        sums = Sums<BOTH>();
        for (int i = lane; i < p.cluster * warps; i += 32)
            sums.add(parts[3 * i], parts[3 * i + 1], parts[3 * i + 2], p.c_t, p.c_1);
        sums.join(p.c_t, p.c_1);
        r_t = reference(sums.top, p.c_t);
        r_1 = reference(sums.top, p.c_1);
        sum_t = sums.t;
        sum_1 = BOTH ? sums.one : sums.t;
    } else {
        __syncthreads();
        const float4 s = p.stats[r];
        r_t = s.x;
        sum_t = s.y;
        r_1 = s.z;
        sum_1 = s.w;
    }
    const bool distils = terms & 1, labelled = terms & 2;
    // The row has nothing above the lowest value that counts.
    const bool low = p.c_t > p.c_1 ? r_t <= p.lowest_t : r_1 <= p.lowest_1;
    auto logit = [&](float x) { return low ? to_f32(from_f32<T>(at_least(x, p.lowest))) : x; };
    if (MODE != kBackward && rank == 0 && last_warp) {
        float loss = 0.f;
        // log2 of the share without a remote element's x c, and that element: it is in the loss by a T (or b) times x
        auto log_share = [&](float at, float c, float ref, float log_sum, float &remote) {
            const float x = logit(at);
            remote = x < kRemote && x > -INFINITY ? x : 0.f;
            return fmaf(remote != 0.f ? 0.f : x, c, -ref) - log_sum;
        };
        float remote;
        if (distils) {
            const float log_q = log2f(sum_t);
            float remotes = 0.f;
            for (int e = lane; e < p.k; e += 32)
                if (entries.index[e] >= 0) {
                    const float lp = entries.log_p[e], share = exp2_fast(lp);
                    if (share != 0.f) {
                        loss += share * (lp - log_share(entries.at_index[e], p.c_t, r_t, log_q, remote));
                        remotes += share * remote;
                    }
                }
#pragma unroll
            for (int d = 16; d > 0; d /= 2) {
                loss += __shfl_xor_sync(~0u, loss, d);
                remotes += __shfl_xor_sync(~0u, remotes, d);
            }
            loss = loss * p.loss_a - p.a * remotes;
        }
        if (labelled) {
            loss -= p.loss_b * log_share(entries.at_index[p.k], p.c_1, r_1, log2f(sum_1), remote);
            loss -= p.b * remote;
        }
        if (lane == 0) {
            p.loss[r] = loss;
            if (p.stats)
                p.stats[r] = make_float4(r_t, sum_t, r_1, sum_1);
        }
    }
    if (MODE == kForward)
        return;

    // The gradient: all of the slice without the entries, then the entries' elements.
    const float scale = p.grad_scale * (p.dloss ? p.dloss[r] : 1.f);
    const float a = distils ? p.a * scale : 0.f, b = labelled ? p.b * scale : 0.f;
    const float f_t = a / sum_t, f_1 = b / sum_1;
    // Without both terms at two temperatures one power does.
    const bool none = !distils && !labelled, single = !BOTH || !distils || !labelled;
    const float c = BOTH && !distils ? p.c_1 : p.c_t, minus_r = BOTH && !distils ? -r_1 : -r_t;
    const float f = !BOTH ? f_t + f_1 : distils ? f_t : f_1;
    auto dense = [&](float x, float y, auto one_power) {
        const f2 both = pair(x, y);
        if constexpr (decltype(one_power)::value)
            return mul(pair(f, f), exp2_fast(fma(both, pair(c, c), pair(minus_r, minus_r))));
        const f2 g = mul(pair(f_t, f_t), exp2_fast(fma(both, pair(p.c_t, p.c_t), pair(-r_t, -r_t))));
        return fma(pair(f_1, f_1), exp2_fast(fma(both, pair(p.c_1, p.c_1), pair(-r_1, -r_1))), g);
    };
    auto dense_one = [&](float x) {
        float g, other;
        apart(single ? dense(logit(x), 0.f, std::true_type()) : dense(logit(x), 0.f, std::false_type()), g, other);
        return none ? 0.f : g;
    };
    T *out = static_cast<T *>(p.dlogits) + r * p.dlogits_stride;
    T *const to0 = out + slice.lead + (int64_t)slice.begin * V;
    auto all = [&](auto one_power) {
        for (int v = threadIdx.x; v < mine; v += threads * kAhead) {
            Vec<T, V> in[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                if (v + j * threads < mine)
                    in[j].word = __ldcs(vectors + v + j * threads);
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                if (v + j * threads < mine) {
                    float x[V];
                    widen(in[j], x);
#pragma unroll
                    for (int e = 0; e < V; e += 2)
                        apart(dense(x[e], x[e + 1], one_power), x[e], x[e + 1]);
                    narrow(x, in[j]);
                    T *to = to0 + (int64_t)(v + j * threads) * V;
                    if (p.wide)
                        __stcs(reinterpret_cast<uint4 *>(to), in[j].word);
                    else {
#pragma unroll
                        for (int e = 0; e < V; ++e)
                            to[e] = in[j].v[e];
                    }
                }
        }
    };
    if (none || low) {                  // zeros whatever the row holds; a row masked all over
#pragma unroll 1
        for (int i = threadIdx.x; i < mine * V; i += threads)
            to0[i] = from_f32<T>(dense_one(to_f32(row[slice.lead + slice.begin * V + i])));
    } else if (single)
        all(std::true_type());
    else
        all(std::false_type());
    if (threadIdx.x < slice.edges) {
        const int e = slice.edge(threadIdx.x);
        out[e] = from_f32<T>(dense_one(to_f32(row[e])));
    }
    __syncthreads();
    if (!last_warp)
        return;
    const int label = entries.index[p.k];
    bool named = false;                 // the label by one of the teacher's entries
    if (distils)
        for (int e = lane; e < p.k; e += 32) {
            const int i = entries.index[e];
            if (i < 0 || !slice.has(i, rank))
                continue;
            float part = -a * exp2_fast(entries.log_p[e]);
            bool first = true;
            if (entries.repeated)       // the first one's lane adds up, in order, those that name the element
                for (int m = 0; m < p.k; ++m)
                    if (m != e && entries.index[m] == i) {
                        first = first && m > e;
                        part -= a * exp2_fast(entries.log_p[m]);
                    }
            if (i == label) {
                part -= b;
                named = true;
            }
            if (first)
                out[i] = from_f32<T>(dense_one(entries.at_index[e]) + part);
        }
    named = __any_sync(~0u, named);
    if (lane == 0 && labelled && !named && slice.has(label, rank))
        out[label] = from_f32<T>(dense_one(entries.at_index[p.k]) - b);
}

// ------------------------------------------------------------------------ host

int bad(const std::string &msg) { return report_error(RIKFAD_ERR_ARG, msg); }

int check_rows(const rikfad_rows &r, const char *name, int bytes, int64_t rows, int64_t cols, int device)
{
    if (r.data == nullptr)
        return bad(std::string(name) + " is NULL");
    if (rows > 1 && (r.stride < cols || r.stride > (int64_t)1 << 32))
        return bad(std::string("the row stride of ") + name + " must be at least its columns");
    if ((uintptr_t)r.data % (uintptr_t)bytes)
        return report_error(RIKFAD_ERR_ALIGN, std::string(name) + " is not aligned to its element type");
    return check_address(r.data, device, name);
}

int check_vector(const void *v, const char *name, size_t align, int device)
{
    if (v == nullptr)
        return bad(std::string(name) + " is NULL");
    if ((uintptr_t)v % align)
        return report_error(RIKFAD_ERR_ALIGN, std::string(name) + " is not aligned");
    return check_address(v, device, name);
}

int check(const rikfad_distillation *p, bool backward)
{
    if (p == nullptr)
        return bad("p is NULL");
    if (p->rows < 0 || p->rows > (int64_t)1 << 28)
        return bad("rows must be in [0, 2^28]");
    if (p->vocab < 1 || p->vocab > 1 << 24)
        return bad("vocab must be in [1, 2^24]");
    if (p->k < 0 || p->k > kMaxEntries)
        return bad("k must be in [0, 1024]");
    if (!dtype_ok(p->dtype) || (p->k > 0 && !dtype_ok(p->teacher_dtype)))
        return bad("dtype and teacher_dtype must be a rikfad_dtype");
    if (p->k > 0 && p->index_bytes != 4 && p->index_bytes != 8)
        return bad("index_bytes must be 4 or 8");
    if (p->labels && p->label_bytes != 4 && p->label_bytes != 8)
        return bad("label_bytes must be 4 or 8");
    if (!std::isfinite(p->temperature) || p->temperature < 1e-3 || p->temperature > 1e3)
        return bad("temperature must be in [0.001, 1000]");
    for (const double w : {p->teacher_weight, p->label_weight, p->grad_scale})
        if (!std::isfinite((float)w))
            return bad("weights and grad_scale must be finite in float32");
    if (!std::isfinite((float)(p->teacher_weight * p->temperature * p->temperature)))
        return bad("teacher_weight times the squared temperature must be finite in float32");
    int device = -1;
    const cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess)
        return report_cuda(e, "cudaGetDevice");
    if (p->rows == 0)
        return RIKFAD_OK;
    const int b = dtype_bytes(p->dtype);
    int rc = check_rows(p->logits, "logits", b, p->rows, p->vocab, device);
    if (!rc && p->k > 0) rc = check_rows(p->teacher, "teacher", dtype_bytes(p->teacher_dtype), p->rows, p->k, device);
    if (!rc && p->k > 0) rc = check_rows(p->index, "index", p->index_bytes, p->rows, p->k, device);
    if (!rc && p->labels) rc = check_vector(p->labels, "labels", (size_t)p->label_bytes, device);
    if (!rc && !backward) rc = check_vector(p->loss, "loss", 4, device);
    if (!rc && (backward || p->stats)) rc = check_vector(p->stats, "stats", 16, device);
    if (!rc && p->dloss) rc = check_vector(p->dloss, "dloss", 4, device);
    if (!rc && (backward || p->dlogits.data)) rc = check_rows(p->dlogits, "dlogits", b, p->rows, p->vocab, device);
    if (!rc && p->dlogits.data == p->logits.data && p->rows > 1 && p->dlogits.stride != p->logits.stride)
        return bad("dlogits = logits needs equal strides");
    return rc;
}

template <typename T, Mode MODE, bool BOTH> cudaError_t launch(Params p, cudaStream_t s)
{
    const int64_t bytes = (int64_t)p.vocab * sizeof(T);
    int threads = 32;
    while (threads < kMaxThreads && bytes / 16 > 4 * threads)
        threads *= 2;
    // Blocks of a row: until the rows under way stay in the L2 cache between their sums and
    // their gradient, and until there are a few rounds of blocks of 16 KB at least (1021 rows of
    // 32003 in float32: 100 us with one block a row, 65 with two, 61 with four).
    const int64_t rounds = (MODE == kFused ? 4 : 1) * kBlocksPerSm * kSms;
    p.cluster = 1;
    while (p.cluster < kMaxCluster && (bytes / p.cluster * kBlocksPerSm * kSms > kUnderWay ||
                                       (p.rows * p.cluster < rounds && bytes / p.cluster > 32 << 10) ||
                                       (p.rows * p.cluster < 2 * kSms && bytes / p.cluster > 16 << 10)))
        p.cluster *= 2;
    if (p.rows * p.cluster > INT32_MAX)
        return cudaErrorInvalidConfiguration;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.rows * p.cluster));
    cfg.blockDim = dim3((unsigned)threads);
    while (MODE != kForward && p.names <= p.k && p.k > 0)
        p.names = p.names ? 2 * p.names : 2;
    cfg.dynamicSmemBytes = sizeof(float) * (3 * ((size_t)p.k + 1) + p.names + 3 * p.cluster * (threads / 32));
    if (MODE == kFused && !BOTH && threads == kMaxThreads) {
        // No more blocks on an SM than that: with more than a 1 / (n + 1) of the shared memory for
        // each, n.  At one temperature registers allow five (elements of 16 bits) or six: cross
        // entropy of 8192 rows of 50257 takes 275 us in bfloat16 with four, 317 with five, 562 in
        // float32 with four, 682 with six.  At two they allow four; to ask for the memory all the
        // same left less of it to the L1 cache (325 us instead of 316 in bfloat16).
        const int64_t most = std::max<int64_t>(kBlocksPerSm, kUnderWay * p.cluster / (bytes * kSms));
        if (most < 6)
            cfg.dynamicSmemBytes = std::max<size_t>(cfg.dynamicSmemBytes, (size_t)(kSmemPerSm / (most + 1)));
    }
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)p.cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = MODE != kBackward && p.cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, rikfad_distill_kernel<T, MODE, BOTH>, p);
}

template <typename T, Mode MODE> cudaError_t launch(const Params &p, cudaStream_t s)
{
    return p.c_t == p.c_1 ? launch<T, MODE, false>(p, s) : launch<T, MODE, true>(p, s);
}

template <typename T> cudaError_t launch(const Params &p, bool backward, cudaStream_t s)
{
    return backward ? launch<T, kBackward>(p, s) : p.dlogits ? launch<T, kFused>(p, s) : launch<T, kForward>(p, s);
}

int run(const rikfad_distillation *p, bool backward, void *stream)
{
    const int rc = check(p, backward);
    if (rc)
        return rc;
    cudaError_t e = cudaPeekAtLastError();
    if (e != cudaSuccess)
        return report_cuda(e, "earlier CUDA error");
    if (p->rows == 0)
        return RIKFAD_OK;
    constexpr double kLog2E = 1.4426950408889634074;
    const double T = p->temperature;
    Params q{};
    q.logits = p->logits.data;
    q.teacher = p->teacher.data;
    q.index = p->index.data;
    q.labels = p->labels;
    q.dlogits = p->dlogits.data;
    q.dloss = p->dloss;
    q.loss = p->loss;
    q.stats = reinterpret_cast<float4 *>(p->stats);
    q.rows = p->rows;
    q.logits_stride = p->logits.stride;
    q.teacher_stride = p->teacher.stride;
    q.index_stride = p->index.stride;
    q.dlogits_stride = p->dlogits.stride;
    q.vocab = (int32_t)p->vocab;
    q.k = p->k;
    q.teacher_dtype = p->teacher_dtype;
    q.index_bytes = p->index_bytes;
    q.label_bytes = p->label_bytes;
    q.distils = p->k > 0 && p->teacher_weight != 0;
    q.labelled = p->labels && p->label_weight != 0;
    const int64_t b = dtype_bytes(p->dtype);
    q.wide = ((uintptr_t)q.logits - (uintptr_t)q.dlogits) % 16 == 0 &&
             (p->rows == 1 || (q.logits_stride - q.dlogits_stride) * b % 16 == 0);
    q.a = (float)(p->teacher_weight * T);
    q.b = (float)p->label_weight;
    q.loss_a = (float)(p->teacher_weight * T * T / kLog2E);
    q.loss_b = (float)(p->label_weight / kLog2E);
    // a term that the call lacks has the other's temperature
    q.c_t = (float)(q.distils ? kLog2E / T : kLog2E);
    q.c_1 = (float)(q.labelled ? kLog2E : q.c_t);
    q.lowest = -kFarthest / std::max(q.c_t, q.c_1);
    q.lowest_t = 0.99f * q.lowest * q.c_t;
    q.lowest_1 = 0.99f * q.lowest * q.c_1;
    q.grad_scale = (float)p->grad_scale;
    const cudaStream_t s = (cudaStream_t)stream;
    e = p->dtype == RIKFAD_F32    ? launch<float>(q, backward, s)
        : p->dtype == RIKFAD_BF16 ? launch<__nv_bfloat16>(q, backward, s)
                                  : launch<__half>(q, backward, s);
    return e == cudaSuccess ? RIKFAD_OK : report_cuda(e, "launch rikfad_distill_kernel");
}

}  // namespace

extern "C" {

RIKFAD_API int rikfad_distillation_forward(const rikfad_distillation *p, void *stream)
{
    RK_ENTRY_BEGIN
    return run(p, false, stream);
    RK_ENTRY_END
}

RIKFAD_API int rikfad_distillation_backward(const rikfad_distillation *p, void *stream)
{
    RK_ENTRY_BEGIN
    return run(p, true, stream);
    RK_ENTRY_END
}

}  // extern "C"
