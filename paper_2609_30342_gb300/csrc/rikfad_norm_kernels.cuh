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
// element is read once and written once.  A thread owns 8 columns of N rows at a
// time and keeps them in registers from the load to the store; the rows share its
// weights' loads, its branches and the barriers of its sums, and hide one another's
// latencies.  Arithmetic is on pairs of float32 (fma.rn.f32x2).  The copies of the
// next rows are under way meanwhile (cp.async into slots of shared memory that only
// this thread reads, so no barrier separates a copy from its use).  Sums over a
// row: shuffles, and beyond a warp one barrier over the row's warps (or the
// cluster's blocks).  Sums over rows stay in the thread's registers to the end of
// the launch, leave one partial row per cluster, and a second kernel adds those in
// order.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "rikfad_host.hpp"
#include "rikfad_kernels.cuh"
#include "rikfad_norm.hpp"
#include "rikfad_types.cuh"

namespace rikfad {

// ------------------------------------------------- pairs of float32

typedef uint64_t f2;        // two float32, the first in the low half

__device__ __forceinline__ f2 pair(float lo, float hi)
{
    f2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ f2 both(float v) { return pair(v, v); }
__device__ __forceinline__ float2 halves(f2 v)
{
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ f2 add(f2 a, f2 b)
{
    f2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 mul(f2 a, f2 b)
{
    f2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 fma(f2 a, f2 b, f2 c)
{
    f2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ float total(f2 v)
{
    const float2 t = halves(v);
    return t.x + t.y;
}

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

// Elements n and beyond set to zero.
__device__ __forceinline__ void cut(Vec8 &o, int n)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 t = halves(o.v[i]);
        o.v[i] = pair(2 * i < n ? t.x : 0.f, 2 * i + 1 < n ? t.y : 0.f);
    }
}

// ------------------------------------------------------------------ staging

__device__ __forceinline__ void copy16_async(uint32_t smem, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(src) : "memory");
}

__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }

// Waits for all but the newest stages - 1 groups.
__device__ __forceinline__ void wait_copies(int stages)
{
    if (stages == 2)
        asm volatile("cp.async.wait_group 1;" ::: "memory");
    else
        asm volatile("cp.async.wait_group 2;" ::: "memory");
}

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

// n elements (1 to 8) into this thread's slot, whose units are `stride` bytes
// apart: copies in flight where the row starts on 16 bytes, else element by element.
// FULL: every row starts on 16 bytes and n is 8.
template <typename T, bool FULL> __device__ __forceinline__ void stage8(uint32_t slot, uint32_t stride, const void *src, int n, bool wide)
{
    if (FULL || (wide && n == 8)) {
        copy16_async(slot, src);
        if constexpr (sizeof(T) == 4)
            copy16_async(slot + stride, static_cast<const char *>(src) + 16);
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
        if (e < n)
            r.v[e] = static_cast<const T *>(src)[e];
#pragma unroll
    for (int i = 0; i < kUnits<T>; ++i)
        smem_put(slot + i * stride, r.w[i]);
}

template <typename T> __device__ __forceinline__ Vec8 fetch8(uint32_t slot, uint32_t stride)
{
    Raw8<T> r;
    if constexpr (sizeof(T) == 4) {
        const uint4 a = smem_get(slot), b = smem_get(slot + stride);
        r.a = *reinterpret_cast<const float4 *>(&a);
        r.b = *reinterpret_cast<const float4 *>(&b);
    } else {
        r.w = smem_get(slot);
    }
    return widen(r);
}

template <typename T, bool FULL> __device__ __forceinline__ void put8(void *to, const Vec8 &v, int n, bool wide)
{
    const Raw8<T> r = narrow<T>(v);
    if (FULL || (wide && n == 8)) {
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
        if (e < n)
            static_cast<T *>(to)[e] = each[e];
}

// Columns [col, col + n) of a weight or bias of type A or float32; `absent` where
// the vector is NULL, 0 beyond n.
template <typename A, bool FULL> __device__ __forceinline__ Vec8 param8(const void *p, bool f32, int col, int n, bool wide, float absent)
{
    if (n == 0)
        return splat(0.f);
    if (p == nullptr) {
        Vec8 o = splat(absent);
        if (!FULL)
            cut(o, n);
        return o;
    }
    if (FULL || (wide && n == 8))
        return f32 ? widen(load_raw8(static_cast<const float *>(p) + col)) : widen(load_raw8(static_cast<const A *>(p) + col));
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        f[e] = e >= n ? 0.f : f32 ? static_cast<const float *>(p)[col + e] : to_f32(static_cast<const A *>(p)[col + e]);
    return widen(Raw8<float>{make_float4(f[0], f[1], f[2], f[3]), make_float4(f[4], f[5], f[6], f[7])});
}

// ----------------------------------------------------------- sums over a row

__device__ __forceinline__ uint32_t smem_address(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

struct alignas(16) RowSums {
    // [parity][value][warp of the cluster]: a sum's slots are written again two sums
    // later, with a barrier in between that follows every read of the first
    float slot[2][4][kNormMaxWarps * 8];
};

__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// The sums of N values over a row's threads, in every one of them, always in the
// same order.
template <int N> __device__ __forceinline__ void row_sum(const NormParams &p, RowSums &s, int &parity, float (&v)[N])
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        if (o < p.lanes)
#pragma unroll
            for (int i = 0; i < N; ++i)
                v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    if (p.lanes <= 32 && p.cluster == 1)
        return;
    parity ^= 1;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (p.cluster == 1) {
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < N; ++i)
                s.slot[parity][i][warp] = v[i];
        __syncthreads();
        // 0 beyond the row's warps
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float4 f = *reinterpret_cast<const float4 *>(&s.slot[parity][i][0]);
            v[i] = (f.x + f.y) + (f.z + f.w);
            for (int w = 4; w * 32 < p.threads; w += 4) {
                f = *reinterpret_cast<const float4 *>(&s.slot[parity][i][w]);
                v[i] += (f.x + f.y) + (f.z + f.w);
            }
        }
        return;
    }
    // lane r < cluster hands the warp's values to block r
    uint32_t rank;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    if (lane < p.cluster) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            uint32_t remote;
            asm("mapa.shared::cluster.u32 %0, %1, %2;"
                : "=r"(remote)
                : "r"(smem_address(&s.slot[parity][i][rank * kNormMaxWarps + warp])), "r"(lane));
            asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(remote), "f"(v[i]) : "memory");
        }
    }
    cluster_barrier();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float t = 0.f;
        for (int w = lane; w < p.cluster * kNormMaxWarps; w += 32)
            t += s.slot[parity][i][w];
        v[i] = warp_sum(t);
    }
}

// ------------------------------------------------------------------ geometry

// A thread's columns and rows, the same in both directions.
struct Place {
    int col, n;             // first column, how many (0 to 8)
    int64_t row;            // first row
    int step;               // distance to the next
    int count, most;        // rows of this thread's group, and of the block's longest

    __device__ __forceinline__ explicit Place(const NormParams &p)
    {
        const int rank = blockIdx.x % p.cluster, id = blockIdx.x / p.cluster;
        const int lane = threadIdx.x % p.lanes, group = threadIdx.x / p.lanes;
        const int begin = rank * p.cta_cols, end = min(p.cols, begin + p.cta_cols);
        col = begin + lane * 8;
        n = max(0, min(8, end - col));
        if (p.gate_rows > 1) {
            // each group walks its own run of rows, so that the rows of a gate stay together
            const int64_t workers = (int64_t)p.ctas * p.row_groups, me = (int64_t)id * p.row_groups + group;
            row = p.rows * me / workers;
            step = 1;
            count = (int)(p.rows * (me + 1) / workers - row);
            most = (int)((p.rows + workers - 1) / workers);
        } else {
            // a block's groups take neighbouring rows
            const int64_t from = p.rows * id / p.ctas, to = p.rows * (id + 1) / p.ctas;
            row = from + group;
            step = p.row_groups;
            count = (int)max((int64_t)0, (to - row + p.row_groups - 1) / p.row_groups);
            most = (int)((to - from + p.row_groups - 1) / p.row_groups);
        }
    }
};

// Where this thread's columns of its first row are; `step` bytes on is its next.
__device__ __forceinline__ char *first_row(const NormRows &r, int bytes, const Place &q)
{
    return static_cast<char *>(r.data) + (q.row * r.stride + q.col) * bytes;
}

// The gate's rows: one for every row, or the same for gate_rows of them.
struct GateWalk {
    char *at;
    int left;               // rows of the gate row to go

    __device__ __forceinline__ GateWalk(const NormParams &p, const NormRows &r, int bytes, const Place &q)
    {
        const int64_t row = p.gate_rows > 1 ? q.row / p.gate_rows : q.row;
        left = p.gate_rows > 1 ? (int)min((row + 1) * p.gate_rows - q.row, (int64_t)INT32_MAX) : 1;
        at = static_cast<char *>(r.data) + (row * r.stride + q.col) * bytes;
    }
    __device__ __forceinline__ void next(const NormParams &p, const NormRows &r)
    {
        if (--left == 0) {
            at += r.step;
            left = p.gate_period;
        }
    }
};

// The head of both kernels: the slots of the sums and of threads without columns
// are zero.
__device__ __forceinline__ void prepare(const NormParams &p, RowSums &sums, const Place &q, uint32_t slot, int units)
{
    for (int i = threadIdx.x; i < (int)(sizeof sums / 4); i += p.threads)
        (&sums.slot[0][0][0])[i] = 0.f;
    if (q.n == 0)
        for (int i = 0; i < units; ++i)
            smem_put(slot + i * p.threads * 16, make_uint4(0, 0, 0, 0));
    if (p.cluster > 1)
        cluster_barrier();
    else
        __syncthreads();
    wait_for_predecessor();
}

// v - m, 0 beyond the row's end.
template <bool FULL> __device__ __forceinline__ Vec8 centred(const Vec8 &v, float m, int n)
{
    const f2 minus = both(n > 0 ? -m : 0.f);
    Vec8 d;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        d.v[i] = add(v.v[i], minus);
    if (!FULL)
        cut(d, n);
    return d;
}

__device__ __forceinline__ float squares(const Vec8 &v)
{
    f2 s = mul(v.v[0], v.v[0]);
#pragma unroll
    for (int i = 1; i < 4; ++i)
        s = fma(v.v[i], v.v[i], s);
    return total(s);
}

__device__ __forceinline__ float elements(const Vec8 &v) { return total(add(add(v.v[0], v.v[1]), add(v.v[2], v.v[3]))); }

// Means and 1 / deviations (or root mean squares) of N rows; v becomes v - m.
template <int N, bool FULL> __device__ __forceinline__ void row_stats(const NormParams &p, RowSums &s, int &parity, int kind, float eps, int n,
                                                                      Vec8 (&v)[N], float (&m)[N], float (&r)[N])
{
    float t[N];
    if (kind == RIKFAD_NORM_LAYER) {
#pragma unroll
        for (int j = 0; j < N; ++j)
            t[j] = elements(v[j]);
        row_sum(p, s, parity, t);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            m[j] = t[j] * p.inv_cols;
            v[j] = centred<FULL>(v[j], m[j], n);
        }
    }
#pragma unroll
    for (int j = 0; j < N; ++j)
        t[j] = squares(v[j]);
    row_sum(p, s, parity, t);
#pragma unroll
    for (int j = 0; j < N; ++j)
        r[j] = rsqrtf(fmaf(t[j], p.inv_cols, eps));
}

// ------------------------------------------------------------------- forward

template <typename A, typename R, int N, bool FULL>
__global__ void __maxnreg__((65536 / kNormForwardThreads / 8 * 8))
    rikfad_norm_forward_kernel(const __grid_constant__ NormParams p)
{
    extern __shared__ uint4 stages[];
    __shared__ RowSums sums;
    const Place q(p);
    const uint32_t stride = p.threads * 16, slot = smem_address(stages + threadIdx.x);
    const uint32_t row_bytes = stride * p.units, stage_bytes = row_bytes * N, end = slot + p.stages * stage_bytes;
    const bool branch = p.z.data != nullptr, gated = p.gate.data != nullptr;
    const bool post = branch && p.post != RIKFAD_NORM_NONE, pre = p.pre != RIKFAD_NORM_NONE;
    const uint32_t z_at = kUnits<R> * stride, gate_at = z_at + kUnits<A> * stride;
    int parity = 0;
    prepare(p, sums, q, slot, p.units * N * p.stages);
    char *x = first_row(p.x, sizeof(R), q), *z = first_row(p.z, sizeof(A), q);
    char *u_out = first_row(p.u, sizeof(R), q), *h_out = first_row(p.h, sizeof(A), q);
    GateWalk gate(p, p.gate, p.gate_f32 ? 4 : (int)sizeof(A), q);
    int ahead = 0;              // rows issued
    uint32_t issue_at = slot;
    auto issue = [&]() {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (ahead + j < q.count && q.n > 0) {
                const uint32_t at = issue_at + j * row_bytes;
                stage8<R, FULL>(at, stride, x, q.n, p.wide_x);
                x += p.x.step;
                if (branch) {
                    stage8<A, FULL>(at + z_at, stride, z, q.n, p.wide_z);
                    z += p.z.step;
                }
                if (gated) {
                    if (p.gate_f32)
                        stage8<float, FULL>(at + gate_at, stride, gate.at, q.n, p.wide_gate);
                    else
                        stage8<A, FULL>(at + gate_at, stride, gate.at, q.n, p.wide_gate);
                    gate.next(p, p.gate);
                }
            }
        commit_copies();
        ahead += N;
        issue_at += stage_bytes;
        if (issue_at == end)
            issue_at = slot;
    };
    for (int k = 0; k < p.stages - 1; ++k)
        issue();
    uint32_t at0 = slot;
    for (int k = 0; k < q.most; k += N) {
        issue();
        wait_copies(p.stages);
        Vec8 u[N], v[N];
        float m2[N], r2[N], m1[N], r1[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            m2[j] = m1[j] = 0.f;
            r2[j] = r1[j] = 1.f;
            u[j] = fetch8<R>(at0 + j * row_bytes, stride);
        }
        const f2 a2 = both(p.a);
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                u[j].v[i] = mul(u[j].v[i], a2);
        if (branch) {
#pragma unroll
            for (int j = 0; j < N; ++j)
                v[j] = fetch8<A>(at0 + j * row_bytes + z_at, stride);
            if (post) {
                row_stats<N, FULL>(p, sums, parity, p.post, p.post_eps, q.n, v, m2, r2);
                const Vec8 w = param8<A, FULL>(p.post_weight, p.param_f32, q.col, q.n, p.wide_params, 1.f);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const f2 r = both(r2[j]);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        v[j].v[i] = mul(mul(v[j].v[i], r), w.v[i]);
                }
                if (p.post_bias) {
                    const Vec8 b = param8<A, FULL>(p.post_bias, p.param_f32, q.col, q.n, p.wide_params, 0.f);
#pragma unroll
                    for (int j = 0; j < N; ++j)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            v[j].v[i] = add(v[j].v[i], b.v[i]);
                }
            }
            if (gated) {
                if (p.gate_f32) {
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        const Vec8 g = fetch8<float>(at0 + j * row_bytes + gate_at, stride);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            v[j].v[i] = mul(v[j].v[i], g.v[i]);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        const Vec8 g = fetch8<A>(at0 + j * row_bytes + gate_at, stride);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            v[j].v[i] = mul(v[j].v[i], g.v[i]);
                    }
                }
            }
            const f2 b2 = both(p.b);
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    u[j].v[i] = fma(v[j].v[i], b2, u[j].v[i]);
        }
        if (p.u.data) {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (k + j < q.count && q.n > 0) {
                    put8<R, FULL>(u_out, u[j], q.n, p.wide_u);
                    u_out += p.u.step;
                }
        }
        if (pre) {
            row_stats<N, FULL>(p, sums, parity, p.pre, p.pre_eps, q.n, u, m1, r1);
            const Vec8 w = param8<A, FULL>(p.pre_weight, p.param_f32, q.col, q.n, p.wide_params, 1.f);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const f2 r = both(r1[j]);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    u[j].v[i] = mul(mul(u[j].v[i], r), w.v[i]);
            }
            if (p.pre_bias) {
                const Vec8 b = param8<A, FULL>(p.pre_bias, p.param_f32, q.col, q.n, p.wide_params, 0.f);
#pragma unroll
                for (int j = 0; j < N; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        u[j].v[i] = add(u[j].v[i], b.v[i]);
            }
        }
        if (p.h.data) {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (k + j < q.count && q.n > 0) {
                    put8<A, FULL>(h_out, u[j], q.n, p.wide_h);
                    h_out += p.h.step;
                }
        }
        if (p.stats && q.col == 0) {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (k + j < q.count)
                    p.stats[q.row + (int64_t)(k + j) * q.step] = make_float4(m2[j], r2[j], m1[j], r1[j]);
        }
        at0 += stage_bytes;
        if (at0 == end)
            at0 = slot;
    }
    allow_successor_launch();
}

// ------------------------------------------------------------------ backward

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
#pragma unroll
    for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f2 *>(buffer + group * width + q.col + 2 * i) = acc.v[i];
    __syncthreads();
    for (int c = threadIdx.x; c < p.cols; c += p.threads) {
        float t = 0.f;
        for (int g = 0; g < p.row_groups; ++g)
            t += buffer[g * width + c];
        out[c] = t;
    }
}

// The branch's y2 and n are formed twice from the stages, on both sides of the
// first sum over the row: the registers go to the sums over rows.
template <typename A, typename R, int N, bool FULL, bool BIAS>
__global__ void __maxnreg__((65536 / kNormBackwardThreads<BIAS && (N > 1)> / 8 * 8))
    rikfad_norm_backward_kernel(const __grid_constant__ NormParams p)
{
    extern __shared__ uint4 stages[];
    __shared__ RowSums sums;
    const Place q(p);
    const uint32_t stride = p.threads * 16, slot = smem_address(stages + threadIdx.x);
    const uint32_t row_bytes = stride * p.units, stage_bytes = row_bytes * N, end = slot + p.stages * stage_bytes;
    const bool branch = p.z.data != nullptr, gated = p.gate.data != nullptr;
    const bool post = branch && p.post != RIKFAD_NORM_NONE, pre = p.pre != RIKFAD_NORM_NONE;
    const bool shared_gate = p.dgate.data && p.gate_rows > 1;
    const int gate_bytes = p.gate_f32 ? 4 : (int)sizeof(A);
    int parity = 0;
    prepare(p, sums, q, slot, p.units * N * p.stages);
    // a row's slots: x, z, dh, du, gate
    const uint32_t z_at = kUnits<R> * stride, dh_at = z_at + kUnits<A> * stride, du_at = dh_at + kUnits<A> * stride;
    const uint32_t gate_at = du_at + kUnits<R> * stride;
    char *x = first_row(p.x, sizeof(R), q), *z = first_row(p.z, sizeof(A), q);
    char *dh = first_row(p.dh, sizeof(A), q), *du = first_row(p.du, sizeof(R), q);
    char *dx = first_row(p.dx, sizeof(R), q), *dz = first_row(p.dz, sizeof(A), q);
    GateWalk gate(p, p.gate, gate_bytes, q);
    int ahead = 0;
    uint32_t issue_at = slot;
    auto issue = [&]() {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (ahead + j < q.count && q.n > 0) {
                const uint32_t at = issue_at + j * row_bytes;
                stage8<R, FULL>(at, stride, x, q.n, p.wide_x);
                x += p.x.step;
                if (branch) {
                    stage8<A, FULL>(at + z_at, stride, z, q.n, p.wide_z);
                    z += p.z.step;
                }
                if (p.dh.data) {
                    stage8<A, FULL>(at + dh_at, stride, dh, q.n, p.wide_dh);
                    dh += p.dh.step;
                }
                if (p.du.data) {
                    stage8<R, FULL>(at + du_at, stride, du, q.n, p.wide_du);
                    du += p.du.step;
                }
                if (gated) {
                    if (p.gate_f32)
                        stage8<float, FULL>(at + gate_at, stride, gate.at, q.n, p.wide_gate);
                    else
                        stage8<A, FULL>(at + gate_at, stride, gate.at, q.n, p.wide_gate);
                    gate.next(p, p.gate);
                }
            }
        commit_copies();
        ahead += N;
        issue_at += stage_bytes;
        if (issue_at == end)
            issue_at = slot;
    };
    Vec8 dw1 = splat(0.f), dw2 = dw1, db1 = dw1, db2 = dw1, dg = dw1;
    // dgate: a row for every row, or the sum over the gate's
    const int64_t gate_row0 = p.gate_rows > 1 ? q.row / p.gate_rows : q.row;
    GateWalk dgate(p, p.dgate, gate_bytes, q);
    bool gate_whole = p.gate_rows * gate_row0 == q.row;     // the sum began with the gate's first row
    bool gate_first = true;                                 // it is the group's first
    auto gate_part = [&](const Vec8 &v) {
        const int64_t worker = (int64_t)(blockIdx.x / p.cluster) * p.row_groups + threadIdx.x / p.lanes;
        put8<float, false>(p.gate_part + (2 * worker + (gate_first ? 0 : 1)) * p.cols + q.col, v, q.n, false);
    };
    auto put_gate = [&](const Vec8 &v) {
        if (q.n == 0)
            return;
        if (p.gate_f32)
            put8<float, FULL>(dgate.at, v, q.n, p.wide_dgate);
        else
            put8<A, FULL>(dgate.at, v, q.n, p.wide_dgate);
    };
    if (shared_gate && q.count == 0)            // a group without rows adds nothing to the gate it lies in
        gate_part(dg);
    for (int k = 0; k < p.stages - 1; ++k)
        issue();
    const float4 *stats = p.stats + q.row;
    float4 next[N];
#pragma unroll
    for (int j = 0; j < N; ++j)
        next[j] = j < q.count ? stats[j * q.step] : make_float4(0.f, 0.f, 0.f, 0.f);
    uint32_t at0 = slot;
    for (int k = 0; k < q.most; k += N) {
        issue();
        float m2[N], r2[N], m1[N], r1[N];
        stats += N * q.step;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            m2[j] = next[j].x;
            r2[j] = next[j].y;
            m1[j] = next[j].z;
            r1[j] = next[j].w;
            if (k + N + j < q.count)
                next[j] = stats[j * q.step];
        }
        wait_copies(p.stages);

        // y2 and n of every row
        Vec8 e[N], y[N], n[N];
        auto branch_of = [&](Vec8(&y2)[N]) {
#pragma unroll
            for (int j = 0; j < N; ++j)
                n[j] = fetch8<A>(at0 + j * row_bytes + z_at, stride);
            if (!post)
                return;
            const Vec8 w = param8<A, FULL>(p.post_weight, p.param_f32, q.col, q.n, p.wide_params, 1.f);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const f2 minus = both(-m2[j]), r = both(r2[j]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    y2[j].v[i] = mul(add(n[j].v[i], minus), r);
                    n[j].v[i] = mul(y2[j].v[i], w.v[i]);
                }
            }
            if (p.post_bias) {
                const Vec8 b = param8<A, FULL>(p.post_bias, p.param_f32, q.col, q.n, p.wide_params, 0.f);
#pragma unroll
                for (int j = 0; j < N; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        n[j].v[i] = add(n[j].v[i], b.v[i]);
            }
        };
        auto times_gate = [&](Vec8(&v)[N]) {
            if (p.gate_f32) {
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const Vec8 g = fetch8<float>(at0 + j * row_bytes + gate_at, stride);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        v[j].v[i] = mul(v[j].v[i], g.v[i]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const Vec8 g = fetch8<A>(at0 + j * row_bytes + gate_at, stride);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        v[j].v[i] = mul(v[j].v[i], g.v[i]);
                }
            }
        };
        // -mean(e y) and -mean(e) (a layer norm's) of every row
        auto means = [&](int kind, float(&t0)[N], float(&t1)[N]) {
            if (kind == RIKFAD_NORM_LAYER) {
                float t[2 * N];
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    f2 s = mul(e[j].v[0], y[j].v[0]);
#pragma unroll
                    for (int i = 1; i < 4; ++i)
                        s = fma(e[j].v[i], y[j].v[i], s);
                    t[2 * j] = total(s);
                    t[2 * j + 1] = elements(e[j]);
                }
                row_sum(p, sums, parity, t);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    t0[j] = -t[2 * j] * p.inv_cols;
                    t1[j] = -t[2 * j + 1] * p.inv_cols;
                }
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    f2 s = mul(e[j].v[0], y[j].v[0]);
#pragma unroll
                    for (int i = 1; i < 4; ++i)
                        s = fma(e[j].v[i], y[j].v[i], s);
                    t0[j] = total(s);
                }
                row_sum(p, sums, parity, t0);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    t0[j] *= -p.inv_cols;
                    t1[j] = 0.f;
                }
            }
        };

        // e: the gradient of h, then of u
        if (p.dh.data) {
#pragma unroll
            for (int j = 0; j < N; ++j)
                e[j] = fetch8<A>(at0 + j * row_bytes + dh_at, stride);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j)
                e[j] = splat(0.f);
        }
        float t0[N], t1[N];
        if (pre) {
            if (branch) {
                branch_of(y);
                if (gated)
                    times_gate(n);
            }
            const f2 a2 = both(p.a), b2 = both(p.b);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                y[j] = fetch8<R>(at0 + j * row_bytes, stride);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    y[j].v[i] = mul(y[j].v[i], a2);
            }
            if (branch) {
#pragma unroll
                for (int j = 0; j < N; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        y[j].v[i] = fma(n[j].v[i], b2, y[j].v[i]);
            }
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const f2 minus = both(-m1[j]), r = both(r1[j]);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    y[j].v[i] = mul(add(y[j].v[i], minus), r);
                if (k + j < q.count) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        dw1.v[i] = fma(e[j].v[i], y[j].v[i], dw1.v[i]);
                        if (BIAS)
                            db1.v[i] = add(e[j].v[i], db1.v[i]);
                    }
                }
            }
            if (p.pre_weight) {
                const Vec8 w = param8<A, FULL>(p.pre_weight, p.param_f32, q.col, q.n, p.wide_params, 1.f);
#pragma unroll
                for (int j = 0; j < N; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        e[j].v[i] = mul(e[j].v[i], w.v[i]);
            }
            means(p.pre, t0, t1);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const f2 my = both(t0[j]), m = both(t1[j]), r = both(r1[j]);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    e[j].v[i] = mul(fma(y[j].v[i], my, add(e[j].v[i], m)), r);
            }
        }
        if (p.du.data) {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const Vec8 d = fetch8<R>(at0 + j * row_bytes + du_at, stride);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    e[j].v[i] = add(e[j].v[i], d.v[i]);
            }
        }
        if (p.dx.data) {
            const f2 a2 = both(p.a);
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (k + j < q.count && q.n > 0) {
                    Vec8 o;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        o.v[i] = mul(e[j].v[i], a2);
                    put8<R, FULL>(dx, o, q.n, p.wide_dx);
                    dx += p.dx.step;
                }
        }
        if (branch) {
            const f2 b2 = both(p.b);
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    e[j].v[i] = mul(e[j].v[i], b2);
            if (post || p.dgate.data)
                branch_of(y);
            if (shared_gate) {
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (k + j < q.count) {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            dg.v[i] = fma(e[j].v[i], n[j].v[i], dg.v[i]);
                        // The gate's last row, or the group's: a gate that lies within
                        // the group is done, others leave a partial sum (the group's
                        // first gate in row 0, its last in row 1).
                        if (dgate.left == 1 || k + j + 1 == q.count) {
                            if (gate_whole && dgate.left == 1)
                                put_gate(dg);
                            else
                                gate_part(dg);
                            dg = splat(0.f);
                            gate_whole = true;
                            gate_first = false;
                        }
                        dgate.next(p, p.dgate);
                    }
            } else if (p.dgate.data) {
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (k + j < q.count) {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            n[j].v[i] = mul(e[j].v[i], n[j].v[i]);
                        put_gate(n[j]);
                        dgate.next(p, p.dgate);
                    }
            }
            if (gated)
                times_gate(e);
            if (post) {
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (k + j < q.count) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            dw2.v[i] = fma(e[j].v[i], y[j].v[i], dw2.v[i]);
                            if (BIAS)
                                db2.v[i] = add(e[j].v[i], db2.v[i]);
                        }
                    }
                const Vec8 w = param8<A, FULL>(p.post_weight, p.param_f32, q.col, q.n, p.wide_params, 1.f);
#pragma unroll
                for (int j = 0; j < N; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        e[j].v[i] = mul(e[j].v[i], w.v[i]);
                means(p.post, t0, t1);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const f2 my = both(t0[j]), m = both(t1[j]), r = both(r2[j]);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        e[j].v[i] = mul(fma(y[j].v[i], my, add(e[j].v[i], m)), r);
                }
            }
            if (p.dz.data) {
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (k + j < q.count && q.n > 0) {
                        put8<A, FULL>(dz, e[j], q.n, p.wide_dz);
                        dz += p.dz.step;
                    }
            }
        }
        at0 += stage_bytes;
        if (at0 == end)
            at0 = slot;
    }
    allow_successor_launch();
    asm volatile("cp.async.wait_all;" ::: "memory");
    float *part = p.sum_part, *buffer = reinterpret_cast<float *>(stages);
    const int64_t size = (int64_t)p.ctas * p.cols;
    if (p.dpre_weight) {
        store_sum(p, q, part, buffer, dw1);
        part += size;
    }
    if (p.dpost_weight) {
        store_sum(p, q, part, buffer, dw2);
        part += size;
    }
    if (BIAS && p.dpre_bias) {
        store_sum(p, q, part, buffer, db1);
        part += size;
    }
    if (BIAS && p.dpost_bias)
        store_sum(p, q, part, buffer, db2);
}

// ----------------------------------------------------------- sums over rows

constexpr int kJoinRows = 32;       // rows of partial sums read at a time, by 32 columns

// Column blockIdx.x * 32 + x of `count` partial rows, `stride` apart, in thread row
// 0: a fixed tree.
__device__ __forceinline__ float join_column(const float *part, int64_t count, int64_t stride, bool live, float (&red)[kJoinRows][33])
{
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    float t = 0.f;
    if (live)
#pragma unroll 8
        for (int64_t i = y; i < count; i += kJoinRows)
            t += __ldcg(part + i * stride);
    __syncthreads();
    red[y][x] = t;
    __syncthreads();
    return warp_sum(red[x][y]);     // of column y, in every lane
}

template <typename A> __device__ __forceinline__ void store_as(void *p, bool f32, int64_t i, float v)
{
    if (f32)
        static_cast<float *>(p)[i] = v;
    else
        static_cast<A *>(p)[i] = from_f32<A>(v);
}

// blockIdx.y below p.sums: a weight's or bias's gradient; beyond: gates whose rows
// several groups share.
template <typename A> __global__ void __launch_bounds__(32 * kJoinRows) rikfad_norm_join_kernel(const __grid_constant__ NormParams p)
{
    __shared__ float red[kJoinRows][33];
    wait_for_predecessor();
    allow_successor_launch();
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + x, out = (int64_t)blockIdx.x * 32 + y;
    if ((int)blockIdx.y < p.sums) {
        void *const each[4] = {p.dpre_weight, p.dpost_weight, p.dpre_bias, p.dpost_bias};
        int at = blockIdx.y;
        void *dst = nullptr;
        for (int i = 0; i < 4; ++i)
            if (each[i] && at-- == 0)
                dst = each[i];
        const float t = join_column(p.sum_part + (int64_t)blockIdx.y * p.ctas * p.cols + c, p.ctas, p.cols, c < p.cols, red);
        if (x == 0 && out < p.cols)
            store_as<A>(dst, p.param_f32, out, t);
        return;
    }
    const int64_t gates = p.rows / p.gate_rows, workers = (int64_t)p.ctas * p.row_groups;
    for (int64_t g = blockIdx.y - p.sums; g < gates; g += gridDim.y - p.sums) {
        // worker w has rows [rows w / workers, rows (w + 1) / workers)
        const int64_t begin = g * p.gate_rows, end = begin + p.gate_rows;
        const int64_t w0 = ((begin + 1) * workers - 1) / p.rows, w1 = (end * workers - 1) / p.rows;
        if (w0 == w1)
            continue;       // written by its only worker
        // the first worker's sum is of its last gate, unless that is its first as well
        const bool head = p.rows * w0 / workers / p.gate_rows == g;
        const float *first = p.gate_part + (2 * w0 + (head ? 0 : 1)) * p.cols;
        float t = join_column(p.gate_part + 2 * (w0 + 1) * p.cols + c, w1 - w0, (int64_t)2 * p.cols, c < p.cols, red);
        if (x == 0 && out < p.cols)
            store_as<A>(p.dgate.data, p.gate_f32, g * p.dgate.stride + out, __ldcg(first + out) + t);
    }
}

// ------------------------------------------------------------------- launch

template <typename K> cudaError_t launch_clustered(K kernel, const NormParams &n, cudaStream_t s)
{
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kNormSmemPerSm);
    if (e != cudaSuccess)
        return e;
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

template <typename A, typename R, bool FULL> cudaError_t launch_rows(const NormParams &n, bool backward, cudaStream_t s)
{
    if (!backward)
        return n.at_once == 1 ? launch_clustered(rikfad_norm_forward_kernel<A, R, 1, FULL>, n, s)
                              : launch_clustered(rikfad_norm_forward_kernel<A, R, kNormRows, FULL>, n, s);
    if (n.at_once == 1)
        return launch_clustered(rikfad_norm_backward_kernel<A, R, 1, FULL, true>, n, s);
    return n.bias ? launch_clustered(rikfad_norm_backward_kernel<A, R, kNormRows, FULL, true>, n, s)
                  : launch_clustered(rikfad_norm_backward_kernel<A, R, kNormRows, FULL, false>, n, s);
}

template <typename A, typename R> cudaError_t launch_norm(const NormParams &n, bool backward, cudaStream_t s)
{
    const cudaError_t e = n.full ? launch_rows<A, R, true>(n, backward, s) : launch_rows<A, R, false>(n, backward, s);
    if (!backward)
        return e;
    const bool shared_gate = n.dgate.data && n.gate_rows > 1;
    if (e != cudaSuccess || (n.sums == 0 && !shared_gate))
        return e;
    const int64_t gates = shared_gate ? n.rows / n.gate_rows : 0;
    const dim3 grid((unsigned)((n.cols + 31) / 32), (unsigned)(n.sums + (gates < 1024 ? gates : 1024)));
    return launch_chained(rikfad_norm_join_kernel<A>, grid, 32 * kJoinRows, 0, s, n);
}

}  // namespace rikfad
