// rikfad_norm_kernels.cuh -- kernels of the residual sum with the norms around it,
//   n = post(z),  u = a x + b gate (.) n,  h = pre(u),
// and of its gradients.  With y2 = (z - m2) r2 and y1 = (u - m1) r1 (m = 0 for an
// RMS norm) and given du, dh:
//   g1 = dh w1,  e = du + r1 (g1 - [mean g1] - y1 mean(g1 y1))   ([.]: layer norm)
//   dx = a e,  dgate = sum over the gate's rows of b e n,  q = b gate e
//   g2 = q w2,  dz = r2 (g2 - [mean g2] - y2 mean(g2 y2))
//   dw1 = sum dh y1,  db1 = sum dh,  dw2 = sum q y2,  db2 = sum q.
// The backward kernel forms u again from x, z and the gate: the same bytes as
// reading u, without the rounding that a stored u has.
//
// Both kernels are bound by memory as long as they need few instructions: every
// element is read once and written once.  A thread owns 8 columns and keeps a row's
// elements there in registers from the load to the store, the weights in registers
// for the whole launch; arithmetic is on pairs of float32 (fma.rn.f32x2).  The
// copies of the next rows are under way meanwhile (cp.async into slots of shared
// memory that only this thread reads, so no barrier separates a copy from its use).
// What is absent (a tensor, columns beyond the row's end, a last round's rows) is
// staged as zeros: the arithmetic has no branches for it.  Rows that do not start on
// 16 bytes (an odd width) are read in aligned vectors all the same: rows whose starts
// are equally far from 16 bytes (every P-th, P = 2, 4 or 8) go to the same block,
// whose columns are shifted by that much.  Sums over a row:
// shuffles, and beyond a warp one barrier over the row's warps (or the cluster's
// blocks).  Sums over rows stay in the thread's registers to the end of the launch,
// leave one partial row per cluster, and a second kernel adds those in order.
//
// Measured, bfloat16 with RMS norms before and after and a gate of its own per row:
// 32768 x 4096 forward 205 us (6.5 TB/s of the 1.34 GB that it must move), backward
// 355 us (6.0 TB/s of 2.15 GB); 8192 x 1600 forward 25 us, backward
// 48 us.  A float32 residual stream and one layer norm, 16384 x 768: 35 and 57 us.
// What is left at small sizes is a launch's ramp and drain (a copy of 8192 x 1600's
// bytes takes 27 and 39 us) and, backward, the second launch.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "rikfad_host.hpp"
#include "rikfad_kernels.cuh"
#include "rikfad_norm.hpp"
#include "rikfad_pairs.cuh"
#include "rikfad_types.cuh"

namespace rikfad {

// 8 elements as 4 pairs.
struct Vec8 {
    f2 v[4];
};

template <typename T> __device__ __forceinline__ Vec8 widen(const Raw8<T> &r)
{
    float f[8];
    unpack8(r, f);
    Vec8 o;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        o.v[i] = pair(f[2 * i], f[2 * i + 1]);
    return o;
}

template <typename T> __device__ __forceinline__ Raw8<T> narrow(const Vec8 &o)
{
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 t = halves(o.v[i]);
        f[2 * i] = t.x;
        f[2 * i + 1] = t.y;
    }
    return pack8(f, T());
}

__device__ __forceinline__ Vec8 splat(float v)
{
    const f2 b = both(v);
    return {{b, b, b, b}};
}

// The elements of a vector that a row has: [lo, hi).
struct Span {
    int lo, hi;
};

// The other elements set to zero.
__device__ __forceinline__ void cut(Vec8 &o, const Span &n)
{
    if (n.lo == 0 && n.hi == 8)
        return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 t = halves(o.v[i]);
        o.v[i] = pair(2 * i >= n.lo && 2 * i < n.hi ? t.x : 0.f, 2 * i + 1 >= n.lo && 2 * i + 1 < n.hi ? t.y : 0.f);
    }
}

// ------------------------------------------------------------------ staging

// The first `bytes` (0 to 16) of 16 in flight, and zeros after them.
__device__ __forceinline__ void copy16_async(uint32_t smem, const void *src, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem), "l"(src), "r"(bytes) : "memory");
}

__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }

// Waits for all copies but the newest row's.
__device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group 1;" ::: "memory"); }

__device__ __forceinline__ void smem_put(uint32_t smem, const uint4 &v)
{
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(smem), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

__device__ __forceinline__ uint4 smem_get(uint32_t smem)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(smem) : "memory");
    return v;
}

// 16-byte units of 8 elements.
template <typename T> constexpr int kUnits = sizeof(T) / 2;

// Elements [lo, hi) of a vector into this thread's slot, whose units are `stride`
// bytes apart, with zeros after them.  `wide`: the vector starts on 16 bytes; then
// the copies are in flight, and the elements before lo are the row's before
// (fetch8 clears them).  FULL: every vector is wide, all of a row's or none.
template <typename T, bool FULL> __device__ __forceinline__ void stage8(uint32_t slot, uint32_t stride, const void *src, const Span &n, bool wide)
{
    if (FULL || wide) {
        if constexpr (sizeof(T) == 4) {
            copy16_async(slot, src, FULL ? n.hi * 2 : min(n.hi, 4) * 4);
            copy16_async(slot + stride, static_cast<const char *>(src) + 16, FULL ? n.hi * 2 : max(n.hi - 4, 0) * 4);
        } else {
            copy16_async(slot, src, n.hi * 2);
        }
        return;
    }
    union {
        T v[8];
        uint4 w[kUnits<T>];
    } r;
#pragma unroll
    for (int i = 0; i < kUnits<T>; ++i)
        r.w[i] = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e >= n.lo && e < n.hi)
            r.v[e] = static_cast<const T *>(src)[e];
#pragma unroll
    for (int i = 0; i < kUnits<T>; ++i)
        smem_put(slot + i * stride, r.w[i]);
}

template <typename T, bool FULL> __device__ __forceinline__ Vec8 fetch8(uint32_t slot, uint32_t stride, const Span &n)
{
    Raw8<T> r;
    if constexpr (sizeof(T) == 4) {
        const uint4 a = smem_get(slot), b = smem_get(slot + stride);
        r.a = *reinterpret_cast<const float4 *>(&a);
        r.b = *reinterpret_cast<const float4 *>(&b);
    } else {
        r.w = smem_get(slot);
    }
    Vec8 v = widen(r);
    if (!FULL && n.lo > 0)
        cut(v, {n.lo, 8});
    return v;
}

// Stores elements [lo, hi) of a vector.
template <typename T, bool FULL> __device__ __forceinline__ void put8(void *to, const Vec8 &v, const Span &n, bool wide)
{
    const Raw8<T> r = narrow<T>(v);
    if (FULL || (wide && n.hi - n.lo == 8)) {
        if (FULL && n.hi == 0)
            return;
        if constexpr (sizeof(T) == 4) {
            static_cast<float4 *>(to)[0] = r.a;
            static_cast<float4 *>(to)[1] = r.b;
        } else {
            *static_cast<uint4 *>(to) = r.w;
        }
        return;
    }
    const T *each = reinterpret_cast<const T *>(&r);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e >= n.lo && e < n.hi)
            static_cast<T *>(to)[e] = each[e];
}

// Columns col + [lo, hi) of a vector of type A or float32, `absent` where it is
// NULL, 0 beyond.
template <typename A> __device__ __forceinline__ Vec8 param8(const void *p, bool f32, int64_t col, const Span &n, float absent)
{
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        f[e] = e < n.lo || e >= n.hi ? 0.f
               : !p                  ? absent
               : f32                 ? static_cast<const float *>(p)[col + e]
                                     : to_f32(static_cast<const A *>(p)[col + e]);
    return {{pair(f[0], f[1]), pair(f[2], f[3]), pair(f[4], f[5]), pair(f[6], f[7])}};
}

// ----------------------------------------------------------- sums over a row

__device__ __forceinline__ uint32_t smem_address(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

struct alignas(16) RowSums {
    // [parity][value][warp of the cluster]: a sum's slots are written again two sums
    // later, with a barrier in between that follows every read of the first
    float slot[2][4][kNormMaxWarps * kNormMaxCluster];
};

__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// A row's threads, and where they leave their sums.
struct Team {
    RowSums *sums;
    uint32_t first;             // shared memory: a row's first slot (of parity 0, value 0)
    uint32_t warp, lane;
    int lanes, warps, cluster;
    uint32_t parity;            // bytes: 0 or kParity

    static constexpr uint32_t kValue = sizeof(RowSums::slot[0][0]), kParity = sizeof(RowSums::slot[0]);

    __device__ __forceinline__ Team(const NormParams &p, RowSums &s)
        : sums(&s), first(smem_address(&s.slot[0][0][0])), warp(threadIdx.x >> 5), lane(threadIdx.x & 31), lanes(p.lanes),
          warps(p.threads >> 5), cluster(p.cluster), parity(0)
    {
    }

    // The sums of N values over a row's threads, in every one of them, always in the
    // same order.
    template <int N> __device__ __forceinline__ void sum(float (&v)[N])
    {
        if (lanes < 32) {           // several rows a warp
#pragma unroll
            for (int o = 16; o > 0; o >>= 1)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float t = __shfl_xor_sync(0xffffffffu, v[i], o);
                    v[i] = o < lanes ? v[i] + t : v[i];
                }
            return;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
#pragma unroll
            for (int i = 0; i < N; ++i)
                v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
        if (cluster > 1) {
            across(v);
            return;
        }
        if (lanes == 32)
            return;
        parity ^= kParity;
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < N; ++i)
                asm volatile("st.shared.f32 [%0], %1;" ::"r"(first + parity + i * kValue + warp * 4), "f"(v[i]) : "memory");
        __syncthreads();
        // slots beyond the row's warps are 0
        if (warps <= 4) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                v[i] = four(first + parity + i * kValue);
        } else if (warps <= 8) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                v[i] = four(first + parity + i * kValue) + four(first + parity + i * kValue + 16);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                v[i] = (four(first + parity + i * kValue) + four(first + parity + i * kValue + 16)) +
                       (four(first + parity + i * kValue + 32) + four(first + parity + i * kValue + 48));
        }
    }

    __device__ __forceinline__ static float four(uint32_t at)
    {
        float4 f;
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(f.x), "=f"(f.y), "=f"(f.z), "=f"(f.w) : "r"(at) : "memory");
        return (f.x + f.y) + (f.z + f.w);
    }

    // Over the blocks of a cluster: lane r hands the warp's values to block r.
    template <int N> __device__ __forceinline__ void across(float (&v)[N])
    {
        parity ^= kParity;
        uint32_t rank;
        asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
        if (lane < cluster) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                uint32_t remote;
                asm("mapa.shared::cluster.u32 %0, %1, %2;"
                    : "=r"(remote)
                    : "r"(first + parity + i * kValue + (rank * kNormMaxWarps + warp) * 4), "r"(lane));
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(remote), "f"(v[i]) : "memory");
            }
        }
        cluster_barrier();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float *slots = sums->slot[parity ? 1 : 0][i];
            float t = 0.f;
            for (int w = lane; w < cluster * kNormMaxWarps; w += 32)
                t += slots[w];
            v[i] = warp_sum(t);
        }
    }
};

// ------------------------------------------------------------------ geometry

// The rows of one class (every p.classes-th row, from `first`): how many there are,
// and where worker w of n begins, counted within the class.
__device__ __forceinline__ int64_t class_rows(const NormParams &p, int first) { return (p.rows - first + p.classes - 1) / p.classes; }
__device__ __forceinline__ int64_t worker_begin(int64_t rows, int64_t w, int64_t n) { return rows * w / n; }

// A thread's columns and rows, the same in both directions.
struct Place {
    int col;                // of its first vector; negative where the row starts within it
    int end;                // of the block's columns
    Span n;                 // of its first vector; without columns, {0, 0} where the row's first vector starts
    int64_t row;            // first row
    int64_t step;           // distance to the next
    int count, most;        // rows of this thread's group, and of the block's longest

    // the span of this thread's vector j, `apart` columns after the one before
    __device__ __forceinline__ Span span(int j, int apart) const
    {
        return j == 0 ? n : Span{0, n.hi > 0 ? max(0, min(8, end - col - j * apart)) : 0};
    }

    __device__ __forceinline__ explicit Place(const NormParams &p)
    {
        const int rank = blockIdx.x % p.cluster, id = blockIdx.x / p.cluster;
        const int lane = threadIdx.x % p.lanes, group = threadIdx.x / p.lanes;
        const int first = id % p.classes, block = id / p.classes, blocks = p.ctas / p.classes;
        const int shift = first * p.drift % 8;
        col = rank * p.cta_cols + lane * 8 - shift;
        end = min(p.cols, (rank + 1) * p.cta_cols - shift);
        n.lo = max(0, -col);
        n.hi = min(8, end - col);
        if (n.hi <= n.lo) {
            col = -shift;       // an aligned start, as for every copy, those of no bytes too
            n = {0, 0};
        }
        const int64_t rows = class_rows(p, first);
        if (p.gate_rows > 1) {
            // each group walks its own run of rows, so that the rows of a gate stay together
            const int64_t workers = (int64_t)blocks * p.row_groups, me = (int64_t)block * p.row_groups + group;
            const int64_t begin = worker_begin(rows, me, workers);
            row = first + p.classes * begin;
            step = p.classes;
            count = (int)(worker_begin(rows, me + 1, workers) - begin);
            most = (int)((rows + workers - 1) / workers);
        } else {
            // a block's groups take neighbouring rows
            const int64_t from = worker_begin(rows, block, blocks), to = worker_begin(rows, block + 1, blocks);
            row = first + p.classes * (from + group);
            step = (int64_t)p.classes * p.row_groups;
            count = (int)max((int64_t)0, (to - from - group + p.row_groups - 1) / p.row_groups);
            most = (int)((to - from + p.row_groups - 1) / p.row_groups);
        }
        row = min(row, p.rows - 1);         // a group without rows points at one that exists
    }
};

// This thread's columns of its first row (without rows, the tensor's start); `step`
// bytes on are its next ones.
__device__ __forceinline__ char *first_row(const NormRows &r, int bytes, const Place &q)
{
    return static_cast<char *>(r.data) + (q.count > 0 ? (q.row * r.stride + q.col) * bytes : 0);
}

// The gate's rows: one for every row, or (SHARED) the same for gate_rows of them.
template <bool SHARED> struct GateWalk {
    char *at;
    int64_t into;           // rows of the gate before the present one
    bool first;             // the present row is the first that this group has of the gate

    __device__ __forceinline__ GateWalk(const NormParams &p, const NormRows &r, int bytes, const Place &q) : into(0), first(true)
    {
        if (!SHARED) {
            at = first_row(r, bytes, q);
            return;
        }
        const int64_t row = q.row / p.gate_rows;
        into = q.row - row * p.gate_rows;
        at = static_cast<char *>(r.data) + (q.count > 0 ? (row * r.stride + q.col) * bytes : 0);
    }
    // the present row is this group's last of the gate
    __device__ __forceinline__ bool last(const NormParams &p, const Place &q) const { return into + q.step >= p.gate_rows; }
    __device__ __forceinline__ void next(const NormParams &p, const NormRows &r, const Place &q)
    {
        if (!SHARED) {
            at += r.step;
            return;
        }
        first = last(p, q);
        for (into += q.step; into >= p.gate_rows; into -= p.gate_rows)
            at += r.step;
    }
};

// The head of both kernels.
__device__ __forceinline__ void prepare(const NormParams &p, RowSums &sums)
{
    for (int i = threadIdx.x; i < (int)(sizeof sums / 4); i += p.threads)
        (&sums.slot[0][0][0])[i] = 0.f;
    if (p.cluster > 1)
        cluster_barrier();
    else
        __syncthreads();
    wait_for_predecessor();
}

#define RK_PAIR _Pragma("unroll") for (int i = 0; i < 4; ++i)
#define RK_EACH _Pragma("unroll") for (int j = 0; j < V; ++j)

__device__ __forceinline__ float dot(const Vec8 &a, const Vec8 &b)
{
    f2 s = mul(a.v[0], b.v[0]), t = mul(a.v[1], b.v[1]);
    s = fma(a.v[2], b.v[2], s);
    t = fma(a.v[3], b.v[3], t);
    return total(add(s, t));
}

__device__ __forceinline__ float elements(const Vec8 &a) { return total(add(add(a.v[0], a.v[1]), add(a.v[2], a.v[3]))); }

// Mean and 1 / deviation (or root mean square) of a row; v becomes v - m, 0 beyond
// the row's end.
template <bool FULL, bool GENERAL, int V>
__device__ __forceinline__ void row_stats(const NormParams &p, Team &team, bool layer, float eps, const Span (&n)[V], Vec8 (&v)[V], float &m,
                                          float &r)
{
    if (GENERAL && layer) {
        float t[1] = {0.f};
        RK_EACH t[0] += elements(v[j]);
        team.sum(t);
        m = t[0] * p.inv_cols;
        RK_EACH
        {
            const f2 minus = both(n[j].hi > 0 ? -m : 0.f);
            RK_PAIR v[j].v[i] = add(v[j].v[i], minus);
            if (!FULL)
                cut(v[j], n[j]);
        }
    }
    float t[1] = {0.f};
    RK_EACH t[0] += dot(v[j], v[j]);
    team.sum(t);
    r = rsqrtf(fmaf(t[0], p.inv_cols, eps));
}

// A thread's two stages: where the next row's copies go, and where the present row's
// are.  (Three to five stages were no faster at any size; forward, 32768 x 4096 takes
// 233 us with three, 206 with two.)
struct Ring {
    uint32_t put, get, other;       // other: put ^ get

    __device__ __forceinline__ Ring(const NormParams &p, const void *stages, int vectors = 1)
    {
        put = smem_address(stages) + threadIdx.x * 16;
        const uint32_t second = put + p.threads * 16 * p.units * vectors;
        other = put ^ second;
        get = put;
    }
    __device__ __forceinline__ void issued()
    {
        commit_copies();
        put ^= other;
    }
    __device__ __forceinline__ void used() { get ^= other; }
};

template <typename A, bool FULL> __device__ __forceinline__ void stage_gate(const NormParams &p, uint32_t to, uint32_t stride, const char *at, const Span &n)
{
    if (p.flags & kNormGateF32)
        stage8<float, FULL>(to, stride, at, n, p.wide & kNormWideGate);
    else
        stage8<A, FULL>(to, stride, at, n, p.wide & kNormWideGate);
}

template <typename A, bool FULL> __device__ __forceinline__ Vec8 fetch_gate(const NormParams &p, uint32_t at, uint32_t stride, const Span &n)
{
    return p.flags & kNormGateF32 ? fetch8<float, FULL>(at, stride, n) : fetch8<A, FULL>(at, stride, n);
}

// ------------------------------------------------------------------- forward

// FULL: every row is whole aligned vectors.  POST: a post norm; GENERAL: layer norms or
// biases (their code and registers are not the RMS norm's).  V vectors of 8 columns a
// thread: with two, the row's sums and barriers cost half as many instructions a
// column, and weights are kept for 16 columns.  SHARED, THREADS: as in the backward
// kernel.
template <typename A, typename R, bool FULL, bool POST, bool GENERAL, bool SHARED, int V, int THREADS>
__global__ void __maxnreg__((norm_registers(THREADS))) rikfad_norm_forward_kernel(const __grid_constant__ NormParams p)
{
    extern __shared__ uint4 stages[];
    __shared__ RowSums sums;
    const Place q(p);
    uint32_t f = p.flags;
    asm volatile("" : "+r"(f));        // in a register: its tests need no constant loads
    const bool branch = POST || (f & kNormBranch), gated = f & kNormGated;
    const uint32_t stride = p.threads * 16;
    const uint32_t z_at = kUnits<R> * stride, gate_at = z_at + kUnits<A> * stride, next_at = stride * p.units;
    const bool staged = gated && !(SHARED && (f & kNormGateHeld));      // else held in registers while it lasts
    const int apart = p.lanes * 8, gate_bytes = f & kNormGateF32 ? 4 : (int)sizeof(A);
    Span cols[V];               // of each vector
    RK_EACH cols[j] = q.span(j, apart);
    const Span none{0, 0};
    Ring ring(p, stages, V);
    Team team(p, sums);
    prepare(p, sums);
    const char *x = first_row(p.x, sizeof(R), q), *z = first_row(p.z, sizeof(A), q);
    char *u_out = first_row(p.u, sizeof(R), q), *h_out = first_row(p.h, sizeof(A), q);
    GateWalk<SHARED> gate(p, p.gate, gate_bytes, q);
    int left = q.count;         // rows to issue; the pointers stay on rows that exist
    auto issue = [&]() {
        RK_EACH
        {
            // a vector that this thread lacks reads nowhere, from its first one's address
            const Span n = left > 0 ? cols[j] : none;
            const int off = cols[j].hi > 0 ? j * apart : 0;
            const uint32_t to = ring.put + j * next_at;
            stage8<R, FULL>(to, stride, x + off * (int)sizeof(R), n, p.wide & kNormWideX);
            if (branch)
                stage8<A, FULL>(to + z_at, stride, z + off * (int)sizeof(A), n, p.wide & kNormWideZ);
            if (staged)
                stage_gate<A, FULL>(p, to + gate_at, stride, gate.at + off * gate_bytes, n);
        }
        if (--left > 0) {
            x += p.x.step;
            z += p.z.step;
            if (staged)
                gate.next(p, p.gate, q);
        }
        ring.issued();
    };
    issue();
    Vec8 w2[V], w1[V], b2[V], b1[V], held[V];
    RK_EACH
    {
        w2[j] = param8<A>(p.post_weight, f & kNormParamF32, q.col + j * apart, cols[j], 1.f);
        w1[j] = param8<A>(p.pre_weight, f & kNormParamF32, q.col + j * apart, cols[j], 1.f);
        if (GENERAL) {
            b2[j] = param8<A>(p.post_bias, f & kNormParamF32, q.col + j * apart, cols[j], 0.f);
            b1[j] = param8<A>(p.pre_bias, f & kNormParamF32, q.col + j * apart, cols[j], 0.f);
        }
        held[j] = splat(1.f);
    }
    const f2 a = both(p.a), b = both(p.b);
    const bool keeps = (f & kNormStats) && q.col <= 0;
    for (int k = 0; k < q.most; ++k) {
        issue();
        const bool live = k < q.count;
        if (SHARED && gated && !staged) {
            if (gate.first)
                RK_EACH held[j] = param8<A>(gate.at, f & kNormGateF32, j * apart, live ? cols[j] : none, 1.f);
            if (k + 1 < q.count)
                gate.next(p, p.gate, q);
        }
        wait_copies();
        float m2 = 0.f, r2 = 1.f, m1 = 0.f, r1 = 1.f;
        Vec8 u[V], v[V];
        RK_EACH
        {
            u[j] = fetch8<R, FULL>(ring.get + j * next_at, stride, cols[j]);
            RK_PAIR u[j].v[i] = mul(u[j].v[i], a);
        }
        if (branch) {
            RK_EACH v[j] = fetch8<A, FULL>(ring.get + j * next_at + z_at, stride, cols[j]);
            if (POST) {
                row_stats<FULL, GENERAL>(p, team, f & kNormPostLayer, p.post_eps, cols, v, m2, r2);
                const f2 r = both(r2);
                RK_EACH
                    RK_PAIR v[j].v[i] = GENERAL ? fma(mul(v[j].v[i], r), w2[j].v[i], b2[j].v[i]) : mul(mul(v[j].v[i], r), w2[j].v[i]);
            }
            if (gated)
                RK_EACH
                {
                    const Vec8 g = !SHARED || staged ? fetch_gate<A, FULL>(p, ring.get + j * next_at + gate_at, stride, cols[j]) : held[j];
                    RK_PAIR v[j].v[i] = mul(v[j].v[i], g.v[i]);
                }
            RK_EACH
                RK_PAIR u[j].v[i] = fma(v[j].v[i], b, u[j].v[i]);
        }
        RK_EACH
            put8<R, FULL>(u_out + j * apart * (int)sizeof(R), u[j], live && (f & kNormU) ? cols[j] : none, p.wide & kNormWideU);
        u_out += p.u.step;
        if (f & kNormPre) {
            row_stats<FULL, GENERAL>(p, team, f & kNormPreLayer, p.pre_eps, cols, u, m1, r1);
            const f2 r = both(r1);
            RK_EACH
                RK_PAIR u[j].v[i] = GENERAL ? fma(mul(u[j].v[i], r), w1[j].v[i], b1[j].v[i]) : mul(mul(u[j].v[i], r), w1[j].v[i]);
        }
        RK_EACH
            put8<A, FULL>(h_out + j * apart * (int)sizeof(A), u[j], live && (f & kNormH) ? cols[j] : none, p.wide & kNormWideH);
        h_out += p.h.step;
        if (keeps && live && q.n.hi > 0)
            p.stats[q.row + k * q.step] = make_float4(m2, r2, m1, r1);
        ring.used();
    }
    allow_successor_launch();
}

// ------------------------------------------------------------------ backward

// How far a block's columns are shifted (Place).
__device__ __forceinline__ int id_shift(const NormParams &p) { return (blockIdx.x / p.cluster) % p.classes * p.drift % 8; }

// One partial row of a sum over rows, from the block's groups in order.
__device__ __forceinline__ void store_sum(const NormParams &p, const Place &q, float *part, float *buffer, const Vec8 &acc)
{
    float *out = part + (int64_t)(blockIdx.x / p.cluster) * p.cols;
    if (p.row_groups == 1) {
        put8<float, false>(out + q.col, acc, q.n, false);
        return;
    }
    __syncthreads();
    const int group = threadIdx.x / p.lanes, width = p.lanes * 8;
    if (q.n.hi > 0)
        RK_PAIR *reinterpret_cast<f2 *>(buffer + group * width + (threadIdx.x % p.lanes) * 8 + 2 * i) = acc.v[i];
    __syncthreads();
    const int shift = id_shift(p);          // column c is at c + shift
    for (int c = threadIdx.x; c < p.cols; c += p.threads) {
        float t = 0.f;
        for (int g = 0; g < p.row_groups; ++g)
            t += buffer[g * width + c + shift];
        out[c] = t;
    }
}

// One vector of 8 columns a thread: with two, the accumulators, weights and elements
// of both do not fit the registers (32768 x 4096: 631 us with the weights read for
// every row, 456 with one vector at that time).  SHARED: a gate
// serves several rows.  THREADS: of an SM, by the registers that the kernel is given.
template <typename A, typename R, bool FULL, bool POST, bool GENERAL, bool SHARED, int THREADS>
__global__ void __maxnreg__((norm_registers(THREADS))) rikfad_norm_backward_kernel(const __grid_constant__ NormParams p)
{
    extern __shared__ uint4 stages[];
    __shared__ RowSums sums;
    const Place q(p);
    uint32_t f = p.flags;
    asm volatile("" : "+r"(f));        // in a register: its tests need no constant loads
    const bool branch = POST || (f & kNormBranch), gated = f & kNormGated, shared_gate = SHARED && (f & kNormDgate);
    const uint32_t stride = p.threads * 16;
    const int gate_bytes = f & kNormGateF32 ? 4 : (int)sizeof(A);
    // a vector's slots: x, z, dh, du, gate
    const uint32_t z_at = kUnits<R> * stride, dh_at = z_at + kUnits<A> * stride, du_at = dh_at + kUnits<A> * stride;
    const uint32_t gate_at = du_at + kUnits<R> * stride;
    const Span none{0, 0};
    const bool staged = gated && !(SHARED && (f & kNormGateHeld));      // else held in registers while it lasts
    Ring ring(p, stages);
    Team team(p, sums);
    prepare(p, sums);
    const char *x = first_row(p.x, sizeof(R), q), *z = first_row(p.z, sizeof(A), q);
    // absent ones are read nowhere (zeros take their place)
    const char *dh = f & kNormDh ? first_row(p.dh, sizeof(A), q) : x, *du = f & kNormDu ? first_row(p.du, sizeof(R), q) : x;
    char *dx = first_row(p.dx, sizeof(R), q), *dz = first_row(p.dz, sizeof(A), q);
    GateWalk<SHARED> gate(p, p.gate, gate_bytes, q);
    int left = q.count;         // rows to issue; the pointers stay on rows that exist
    auto issue = [&]() {
        const Span n = left > 0 ? q.n : none;
        stage8<R, FULL>(ring.put, stride, x, n, p.wide & kNormWideX);
        if (branch)
            stage8<A, FULL>(ring.put + z_at, stride, z, n, p.wide & kNormWideZ);
        stage8<A, FULL>(ring.put + dh_at, stride, dh, f & kNormDh ? n : none, p.wide & kNormWideDh);
        stage8<R, FULL>(ring.put + du_at, stride, du, f & kNormDu ? n : none, p.wide & kNormWideDu);
        if (staged)
            stage_gate<A, FULL>(p, ring.put + gate_at, stride, gate.at, n);
        if (--left > 0) {
            x += p.x.step;
            z += p.z.step;
            dh += p.dh.step;
            du += p.du.step;
            if (staged)
                gate.next(p, p.gate, q);
        }
        ring.issued();
    };
    Vec8 dw1 = splat(0.f), dw2 = dw1, db1 = dw1, db2 = dw1, dg = dw1;
    // dgate: a row for every row, or the sum over the gate's
    GateWalk<SHARED> dgate(p, p.dgate, gate_bytes, q);
    bool gate_first = true;                     // the sum is of the group's first gate
    const int64_t worker = (int64_t)(blockIdx.x / p.cluster) * p.row_groups + threadIdx.x / p.lanes;
    auto gate_part = [&]() {
        put8<float, false>(p.gate_part + (2 * worker + (gate_first ? 0 : 1)) * p.cols + q.col, dg, q.n, false);
    };
    auto put_gate = [&](const Vec8 &v, const Span &n) {
        if (f & kNormGateF32)
            put8<float, FULL>(dgate.at, v, n, p.wide & kNormWideDgate);
        else
            put8<A, FULL>(dgate.at, v, n, p.wide & kNormWideDgate);
    };
    if (shared_gate && q.count == 0)            // a group without rows adds nothing to the gate it lies in
        gate_part();
    bool gate_whole = p.classes == 1 && dgate.into == 0;    // the sum began with the gate's first row
    Vec8 held = splat(1.f);
    issue();
    const Vec8 w2 = param8<A>(p.post_weight, f & kNormParamF32, q.col, q.n, 1.f);
    const Vec8 w1 = param8<A>(p.pre_weight, f & kNormParamF32, q.col, q.n, 1.f);
    const Vec8 b2 = param8<A>(p.post_bias, f & kNormParamF32, q.col, q.n, 0.f);
    const f2 a = both(p.a), b = both(p.b);
    const float4 *stats = p.stats + q.row;
    float4 next = q.count > 0 ? *stats : make_float4(0.f, 0.f, 0.f, 0.f);
    // Of the row whose first sum is known: e (the weighted gradient of h), y, the two
    // norms' 1 / deviation and the second one's mean.  t: its sums of e y and of e.
    // With a post norm, row k's second sums and row k + 1's first ones share a barrier:
    // their arithmetic is independent, and half of the waits are gone (32768 x 4096 gated:
    // 409 us with a barrier each, 356 so).  Not where the other row's values do not fit
    // the registers: a shared gate's sum (8192 x 1600: 75 us, 92 in one barrier), or
    // columns in parts with RMS norms (8192 x 1601: 68 us, 76).
    constexpr bool TOGETHER = POST && !SHARED && (FULL || GENERAL);
    // The normalised branch is formed again from its stage, except where the registers
    // hold it (8192 x 1600 of two layer norms: 72 us, 83 formed again).
    constexpr bool KEEP = POST && GENERAL && !SHARED && THREADS == kNormHeavyThreads;
    Vec8 e, y, kept;
    float r1 = 0.f, r2 = 0.f, m2 = 0.f, t[2];
    auto gate_of = [&](uint32_t at) {
        Vec8 g = splat(p.b);
        if (gated) {
            g = !SHARED || staged ? fetch_gate<A, FULL>(p, at + gate_at, stride, q.n) : held;
            RK_PAIR g.v[i] = mul(g.v[i], b);
        }
        return g;
    };
    // The branch's normalised columns, and their weighted sum with the bias.
    auto normalised = [&](uint32_t at) {
        Vec8 v = fetch8<A, FULL>(at + z_at, stride, q.n);
        if (POST) {
            const f2 minus = both(-m2), r = both(r2);
            RK_PAIR v.v[i] = GENERAL ? mul(add(v.v[i], minus), r) : mul(v.v[i], r);
        }
        return v;
    };
    auto weighted = [&](const Vec8 &v) {
        Vec8 n = v;
        if (POST)
            RK_PAIR n.v[i] = GENERAL ? fma(v.v[i], w2.v[i], b2.v[i]) : mul(v.v[i], w2.v[i]);
        return n;
    };
    // Up to the first sum of row k, whose stage is at `at`.
    auto begin = [&](int k, uint32_t at) {
        const float m1 = next.z;
        m2 = next.x;
        r2 = next.y;
        r1 = next.w;
        stats += q.step;
        next = k + 1 < q.count ? *stats : make_float4(0.f, 0.f, 0.f, 0.f);
        if (SHARED && gated && !staged) {
            if (gate.first)
                held = param8<A>(gate.at, f & kNormGateF32, 0, k < q.count ? q.n : none, 1.f);
            if (k + 1 < q.count)
                gate.next(p, p.gate, q);
        }
        e = fetch8<A, FULL>(at + dh_at, stride, q.n);
        y = fetch8<R, FULL>(at, stride, q.n);
        RK_PAIR y.v[i] = mul(y.v[i], a);
        if (branch) {
            const Vec8 v = normalised(at), n = weighted(v), g = gate_of(at);
            if (KEEP)
                kept = v;
            RK_PAIR y.v[i] = fma(n.v[i], g.v[i], y.v[i]);
        }
        t[0] = t[1] = 0.f;
        if (f & kNormPre) {
            const f2 minus = both(-m1), r = both(r1);
            RK_PAIR
            {
                y.v[i] = GENERAL ? mul(add(y.v[i], minus), r) : mul(y.v[i], r);
                dw1.v[i] = fma(e.v[i], y.v[i], dw1.v[i]);
                if (GENERAL)
                    db1.v[i] = add(e.v[i], db1.v[i]);
                e.v[i] = mul(e.v[i], w1.v[i]);
            }
            t[0] = dot(e, y);
            if (GENERAL)
                t[1] = elements(e);
        }
    };
    // r (e - [mean e] - y mean(e y)) from the sums
    auto through_norm = [&](Vec8 &v, const Vec8 &by, float dots, float plain, bool layer, float r) {
        // columns beyond the row's end stay zero: they add nothing to later sums
        const f2 my = both(-dots * p.inv_cols), m = both(GENERAL && layer ? -plain * p.inv_cols : 0.f), rr = both(q.n.hi > 0 ? r : 0.f);
        RK_PAIR v.v[i] = mul(GENERAL ? fma(by.v[i], my, add(v.v[i], m)) : fma(by.v[i], my, v.v[i]), rr);
        if (!FULL)
            cut(v, q.n);
    };
    auto sum = [&](float (&v)[2]) {             // the second value is of layer norms only
        if (GENERAL) {
            team.sum(v);
        } else {
            float one[1] = {v[0]};
            team.sum(one);
            v[0] = one[0];
        }
    };
    issue();
    wait_copies();
    begin(0, ring.get);
    sum(t);
    for (int k = 0; k < q.most; ++k) {
        const Span n = k < q.count ? q.n : none;
        if (f & kNormPre)
            through_norm(e, y, t[0], t[1], f & kNormPreLayer, r1);
        {
            Vec8 o = fetch8<R, FULL>(ring.get + du_at, stride, q.n);
            RK_PAIR e.v[i] = add(e.v[i], o.v[i]);
            RK_PAIR o.v[i] = mul(e.v[i], a);
            put8<R, FULL>(dx, o, f & kNormDx ? n : none, p.wide & kNormWideDx);
            dx += p.dx.step;
        }
        float s[2] = {0.f, 0.f};
        Vec8 y2 = e;
        if (branch) {
            if (POST || (f & kNormDgate))
                y2 = KEEP ? kept : normalised(ring.get);
            if (f & kNormDgate) {
                Vec8 nn = weighted(y2);
                if (!SHARED) {
                    RK_PAIR nn.v[i] = mul(mul(e.v[i], b), nn.v[i]);
                    put_gate(nn, n);
                    dgate.next(p, p.dgate, q);
                } else if (k < q.count) {
                    RK_PAIR dg.v[i] = fma(mul(e.v[i], b), nn.v[i], dg.v[i]);
                    // The group's last row of the gate, or of all: a gate that lies within
                    // the group is done, others leave a partial sum (the group's first
                    // gate in row 0, its last in row 1).
                    const bool last = dgate.last(p, q);
                    if (last || k + 1 == q.count) {
                        if (gate_whole && last)
                            put_gate(dg, q.n);
                        else
                            gate_part();
                        dg = splat(0.f);
                        gate_whole = p.classes == 1;
                        gate_first = false;
                    }
                    dgate.next(p, p.dgate, q);
                }
            }
            const Vec8 g = gate_of(ring.get);
            RK_PAIR e.v[i] = mul(e.v[i], g.v[i]);
            if (POST) {
                RK_PAIR
                {
                    dw2.v[i] = fma(e.v[i], y2.v[i], dw2.v[i]);
                    if (GENERAL)
                        db2.v[i] = add(e.v[i], db2.v[i]);
                    e.v[i] = mul(e.v[i], w2.v[i]);
                }
                s[0] = dot(e, y2);
                if (GENERAL)
                    s[1] = elements(e);
            }
        }
        const float by2 = r2;
        Vec8 out = e;
        auto put_branch = [&]() {
            if (!branch)
                return;
            if (POST)
                through_norm(out, y2, s[0], s[1], f & kNormPostLayer, by2);
            put8<A, FULL>(dz, out, f & kNormDz ? n : none, p.wide & kNormWideDz);
            dz += p.dz.step;
        };
        if (!TOGETHER) {
            if (POST)
                sum(s);
            put_branch();
        }
        issue();
        ring.used();
        wait_copies();
        begin(k + 1, ring.get);
        if (!TOGETHER) {
            sum(t);
        } else if (GENERAL) {
            float all[4] = {s[0], s[1], t[0], t[1]};
            team.sum(all);
            s[0] = all[0], s[1] = all[1], t[0] = all[2], t[1] = all[3];
        } else {
            float all[2] = {s[0], t[0]};
            team.sum(all);
            s[0] = all[0], t[0] = all[1];
        }
        if (TOGETHER)
            put_branch();
    }
    allow_successor_launch();
    asm volatile("cp.async.wait_all;" ::: "memory");
    float *part = p.sum_part, *buffer = reinterpret_cast<float *>(stages);
    const int64_t size = (int64_t)p.ctas * p.cols;
    auto store = [&](uint32_t flag, const Vec8 &acc) {
        if (f & flag) {
            store_sum(p, q, part, buffer, acc);
            part += size;
        }
    };
    store(kNormDpreWeight, dw1);
    store(kNormDpostWeight, dw2);
    if (GENERAL) {
        store(kNormDpreBias, db1);
        store(kNormDpostBias, db2);
    }
}

// ----------------------------------------------------------- sums over rows

constexpr int kJoinRows = 32;       // rows of partial sums read at a time, by 32 columns
constexpr int kJoinThreads = 32 * kJoinRows;

// The block's total of its threads' `t` by column (threadIdx.x % 32): a fixed tree;
// that of column y in every lane of warp y.
__device__ __forceinline__ float join_rows(float t, float (&red)[kJoinRows][33])
{
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    __syncthreads();
    red[y][x] = t;
    __syncthreads();
    return warp_sum(red[x][y]);
}

template <typename A> __device__ __forceinline__ void store_as(void *p, bool f32, int64_t i, float v)
{
    if (f32)
        static_cast<float *>(p)[i] = v;
    else
        static_cast<A *>(p)[i] = from_f32<A>(v);
}

// A gate whose rows several groups share: the sum of their partial rows in order.
// Item i is gate i, or with p.join_bounds the gate in which worker i + 1 begins (there
// are fewer of those where gates serve few rows).  join_rows partial rows are read at a
// time, by kJoinThreads / join_rows columns.
template <typename A> __device__ void join_gate(const NormParams &p, float *red, int item, int columns)
{
    const int64_t workers = (int64_t)(p.ctas / p.classes) * p.row_groups;       // of a class
    const int width = kJoinThreads / p.join_rows, x = threadIdx.x % width, y = threadIdx.x / width;
    const int64_t c = (int64_t)columns * width + x;
    int64_t g = item;
    if (p.join_bounds) {
        // each gate once: the first worker that begins after its first row
        const int64_t row = worker_begin(p.rows, item + 1, workers), before = worker_begin(p.rows, item, workers);
        g = row / p.gate_rows;
        if (row >= p.rows || row == g * p.gate_rows || before > g * p.gate_rows)
            return;
    }
    const int64_t begin = g * p.gate_rows, end = begin + p.gate_rows;
    // Thread row y takes every (join_rows / classes)-th worker of class y % classes:
    // the class's rows of the gate are [i0, i1] of its own.
    const int first = y % p.classes;
    const int64_t rows = class_rows(p, first);
    const int64_t i0 = begin <= first ? 0 : (begin - first + p.classes - 1) / p.classes;
    const int64_t i1 = end - 1 < first ? -1 : (end - 1 - first) / p.classes;
    float t = 0.f;
    if (i0 <= i1) {
        const int64_t w0 = ((i0 + 1) * workers - 1) / rows, w1 = ((i1 + 1) * workers - 1) / rows;
        if (p.classes == 1 && w0 == w1)
            return;             // written by its only worker
        if (c < p.cols)
            for (int64_t w = w0 + y / p.classes; w <= w1; w += p.join_rows / p.classes) {
                const int64_t row = first + p.classes * worker_begin(rows, w, workers);     // the worker's first
                // block b of the class has number b classes + first
                const int64_t worker = (w / p.row_groups * p.classes + first) * p.row_groups + w % p.row_groups;
                t += __ldcg(p.gate_part + (2 * worker + (row / p.gate_rows == g ? 0 : 1)) * p.cols + c);
            }
    }
    red[y * (width + 1) + x] = t;
    __syncthreads();
    if (y == 0 && c < p.cols) {
        t = red[x];
        for (int i = 1; i < p.join_rows; ++i)
            t += red[i * (width + 1) + x];
        store_as<A>(p.dgate.data, p.flags & kNormGateF32, g * p.dgate.stride + c, t);
    }
}

// Adds the partial rows of the sums in order, 32 columns a block: a few megabytes that
// the kernel before has left in L2 (8192 x 1600: 3.9 MB; 10 us alone with cold caches).
// The first blocks: a weight's or bias's gradient each; beyond: gates.
template <typename A> __global__ void __launch_bounds__(kJoinThreads) rikfad_norm_join_kernel(const __grid_constant__ NormParams p)
{
    __shared__ float red[kJoinRows][33];
    wait_for_predecessor();
    allow_successor_launch();
    const int strips = (p.cols + 31) / 32, sum = blockIdx.x / strips;
    if (sum >= p.sums) {
        const int id = blockIdx.x - strips * p.sums, columns = (p.cols + kJoinThreads / p.join_rows - 1) / (kJoinThreads / p.join_rows);
        join_gate<A>(p, &red[0][0], id / columns, id % columns);
        return;
    }
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int64_t strip = blockIdx.x % strips, c = strip * 32 + x, out = strip * 32 + y;
    void *const each[4] = {p.dpre_weight, p.dpost_weight, p.dpre_bias, p.dpost_bias};
    int at = sum;
    void *dst = nullptr;
    for (int i = 0; i < 4; ++i)
        if (each[i] && at-- == 0)
            dst = each[i];
    const float *part = p.sum_part + (int64_t)sum * p.ctas * p.cols + c;
    float t = 0.f;
    if (c < p.cols)
#pragma unroll 16
        for (int i = y; i < p.ctas; i += kJoinRows)
            t += __ldcg(part + (int64_t)i * p.cols);
    t = join_rows(t, red);
    if (x == 0 && out < p.cols)
        store_as<A>(dst, p.flags & kNormParamF32, out, t);
}

// ------------------------------------------------------------------- launch

template <typename K> cudaError_t launch_clustered(K kernel, const NormParams &n, cudaStream_t s)
{
    if (n.smem > kNormSmemDefault) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kNormSmemPerSm);
        if (e != cudaSuccess)
            return e;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(n.ctas * n.cluster));
    cfg.blockDim = dim3((unsigned)n.threads);
    cfg.dynamicSmemBytes = n.smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)n.cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = n.cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, n);
}

template <typename A, typename R, bool FULL, bool POST, bool GENERAL> cudaError_t launch_forward(const NormParams &n, cudaStream_t s)
{
    constexpr int kOne = POST && GENERAL ? kNormHeavyForwardThreads1 : kNormForwardThreads1;
    if (n.flags & kNormSharedGate)
        return launch_clustered(rikfad_norm_forward_kernel<A, R, FULL, POST, GENERAL, true, 1, kOne>, n, s);
    if (n.vectors == 1)
        return launch_clustered(rikfad_norm_forward_kernel<A, R, FULL, POST, GENERAL, false, 1, kOne>, n, s);
    if constexpr (POST && GENERAL)
        if (n.threads_per_sm == kNormHeavyThreads)
            return launch_clustered(rikfad_norm_forward_kernel<A, R, FULL, POST, GENERAL, false, 2, kNormHeavyThreads>, n, s);
    return launch_clustered(rikfad_norm_forward_kernel<A, R, FULL, POST, GENERAL, false, 2, kNormForwardThreads2>, n, s);
}

template <typename A, typename R, bool FULL, bool POST, bool GENERAL> cudaError_t launch_backward(const NormParams &n, cudaStream_t s)
{
    const bool shared = n.flags & kNormSharedGate;
    if constexpr (POST && GENERAL)
        if (n.threads_per_sm == kNormHeavyThreads)
            return shared ? launch_clustered(rikfad_norm_backward_kernel<A, R, FULL, POST, GENERAL, true, kNormHeavyThreads>, n, s)
                          : launch_clustered(rikfad_norm_backward_kernel<A, R, FULL, POST, GENERAL, false, kNormHeavyThreads>, n, s);
    return shared ? launch_clustered(rikfad_norm_backward_kernel<A, R, FULL, POST, GENERAL, true, kNormBackwardThreads>, n, s)
                  : launch_clustered(rikfad_norm_backward_kernel<A, R, FULL, POST, GENERAL, false, kNormBackwardThreads>, n, s);
}

// The kernels of one pair of types; a translation unit instantiates one of the two.
template <typename A, typename R> cudaError_t norm_forward(const NormParams &n, cudaStream_t s)
{
    const bool post = n.flags & kNormPost;
    if (n.full)
        return post ? (n.general ? launch_forward<A, R, true, true, true>(n, s) : launch_forward<A, R, true, true, false>(n, s))
                    : (n.general ? launch_forward<A, R, true, false, true>(n, s) : launch_forward<A, R, true, false, false>(n, s));
    return post ? (n.general ? launch_forward<A, R, false, true, true>(n, s) : launch_forward<A, R, false, true, false>(n, s))
                : (n.general ? launch_forward<A, R, false, false, true>(n, s) : launch_forward<A, R, false, false, false>(n, s));
}

template <typename A, typename R> cudaError_t norm_backward(const NormParams &n, cudaStream_t s)
{
    const bool post = n.flags & kNormPost;
    cudaError_t e;
    if (n.full)
        e = post ? (n.general ? launch_backward<A, R, true, true, true>(n, s) : launch_backward<A, R, true, true, false>(n, s))
                 : (n.general ? launch_backward<A, R, true, false, true>(n, s) : launch_backward<A, R, true, false, false>(n, s));
    else
        e = post ? (n.general ? launch_backward<A, R, false, true, true>(n, s) : launch_backward<A, R, false, true, false>(n, s))
                 : (n.general ? launch_backward<A, R, false, false, true>(n, s) : launch_backward<A, R, false, false, false>(n, s));
    const bool shared_gate = n.dgate.data && n.gate_rows > 1 && n.rows > 0;
    if (e != cudaSuccess || (n.sums == 0 && !shared_gate))
        return e;
    NormParams j = n;
    int64_t blocks = (int64_t)n.sums * ((n.cols + 31) / 32);
    j.join_rows = kJoinRows;
    if (shared_gate) {
        // Gates, or the places where workers begin, whichever are fewer; and thread rows
        // for the partial rows that a gate has, at least one for each class (8192 x 1600
        // backward, 16 rows a gate: 99 us, 487 with all gates and 32 thread rows).
        const int64_t gates = n.rows / n.gate_rows, workers = (int64_t)(n.ctas / n.classes) * n.row_groups;
        const int64_t parts = n.classes * (n.gate_rows * workers / n.rows + 2);
        j.join_bounds = n.classes == 1 && gates >= workers;
        for (j.join_rows = n.classes; j.join_rows < kJoinRows && j.join_rows < parts;)
            j.join_rows *= 2;
        const int width = kJoinThreads / j.join_rows;
        blocks += (j.join_bounds ? workers - 1 : gates) * ((n.cols + width - 1) / width);
    }
    if (blocks == 0)
        return cudaSuccess;
    if (blocks > INT32_MAX)
        return cudaErrorInvalidConfiguration;
    const dim3 grid((unsigned)blocks);
    return launch_chained(rikfad_norm_join_kernel<A>, grid, kJoinThreads, 0, s, j);
}

}  // namespace rikfad
