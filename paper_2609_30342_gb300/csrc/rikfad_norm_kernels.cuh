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
// Both kernels are bound by memory: every element is read once and written once.
// A thread owns 8 columns of a row and keeps them in registers from the load to
// the store; the loads of the next rows are under way meanwhile (cp.async into
// slots of shared memory that only this thread reads, so no barrier separates a
// copy from its use).  Sums over a row: shuffles, then one barrier over the row's
// warps (or the cluster's blocks).  Sums over rows stay in the thread's registers
// to the end of the launch, leave one partial row per cluster, and a second kernel
// adds those in order.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "rikfad_host.hpp"
#include "rikfad_kernels.cuh"
#include "rikfad_norm.hpp"
#include "rikfad_types.cuh"

namespace rikfad {

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

// Up to n <= 8 elements into this thread's slot, whose units are `stride` bytes
// apart: copies in flight where the row starts on 16 bytes, else element by element.
template <typename T> __device__ __forceinline__ void stage8(uint32_t slot, uint32_t stride, const T *src, int n, bool wide)
{
    if (wide && n == 8) {
        copy16_async(slot, src);
        if constexpr (sizeof(T) == 4)
            copy16_async(slot + stride, src + 4);
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
            r.v[e] = src[e];
#pragma unroll
    for (int i = 0; i < kUnits<T>; ++i)
        smem_put(slot + i * stride, r.w[i]);
}

template <typename T> __device__ __forceinline__ void fetch8(uint32_t slot, uint32_t stride, float (&v)[8])
{
    Raw8<T> r;
    if constexpr (sizeof(T) == 4) {
        const uint4 a = smem_get(slot), b = smem_get(slot + stride);
        r.a = *reinterpret_cast<const float4 *>(&a);
        r.b = *reinterpret_cast<const float4 *>(&b);
    } else {
        r.w = smem_get(slot);
    }
    unpack8(r, v);
}

template <typename T> __device__ __forceinline__ void put8(T *dst, const float (&v)[8], int n, bool wide)
{
    if (wide && n == 8) {
        const Raw8<T> r = pack8(v, T());
        if constexpr (sizeof(T) == 4) {
            reinterpret_cast<float4 *>(dst)[0] = r.a;
            reinterpret_cast<float4 *>(dst)[1] = r.b;
        } else {
            *reinterpret_cast<uint4 *>(dst) = r.w;
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < n)
            dst[e] = from_f32<T>(v[e]);
}

// 8 weights or biases of type A or float32; `absent` where the vector is NULL, 0
// beyond the row's end.
template <typename A> __device__ __forceinline__ void param8(const void *p, bool f32, int col, int n, bool wide, float absent,
                                                             float (&v)[8])
{
    if (p == nullptr) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = e < n ? absent : 0.f;
    } else if (wide && n == 8) {
        if (f32)
            unpack8(load_raw8(static_cast<const float *>(p) + col), v);
        else
            unpack8(load_raw8(static_cast<const A *>(p) + col), v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = e >= n ? 0.f : f32 ? static_cast<const float *>(p)[col + e] : to_f32(static_cast<const A *>(p)[col + e]);
    }
}

// ----------------------------------------------------------- sums over a row

__device__ __forceinline__ uint32_t smem_address(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

struct alignas(16) RowSums {
    // [parity][value][warp of the cluster]: a sum's slots are written again two sums
    // later, with a barrier in between that follows every read of the first
    float slot[2][2][kNormMaxWarps * 8];
};

// The sums of N values over a row's threads, in every one of them, always in the
// same order.
template <int N> __device__ __forceinline__ void row_sum(const NormParams &p, RowSums &s, int &parity, float (&v)[N])
{
    const int width = min(p.lanes, 32);
    for (int o = width / 2; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    if (p.lanes <= 32 && p.cluster == 1)
        return;
    parity ^= 1;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = p.threads >> 5;
    if (p.cluster == 1) {
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < N; ++i)
                s.slot[parity][i][warp] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = 0.f;
            for (int w = 0; w < warps; w += 4) {
                const float4 f = *reinterpret_cast<const float4 *>(&s.slot[parity][i][w]);     // beyond the warps: 0
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
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float t = 0.f;
        for (int w = lane; w < p.cluster * kNormMaxWarps; w += 32)
            t += s.slot[parity][i][w];
        v[i] = warp_sum(t);
    }
}

// Mean and 1 / deviation (or root mean square) of 8 values a thread.
__device__ __forceinline__ void row_stats(const NormParams &p, RowSums &s, int &parity, int kind, float eps, int n,
                                          const float (&v)[8], float &m, float &r)
{
    m = 0.f;
    r = 1.f;
    if (kind == RIKFAD_NORM_NONE)
        return;
    float t[1];
    if (kind == RIKFAD_NORM_LAYER) {
        t[0] = ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
        row_sum(p, s, parity, t);
        m = t[0] * p.inv_cols;
    }
    t[0] = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float d = kind == RIKFAD_NORM_LAYER ? (e < n ? v[e] - m : 0.f) : v[e];
        t[0] = fmaf(d, d, t[0]);
    }
    row_sum(p, s, parity, t);
    r = rsqrtf(fmaf(t[0], p.inv_cols, eps));
}

// ------------------------------------------------------------------ geometry

// A thread's columns and a block's share of the rows.
struct Place {
    int col, n;             // first column, how many (0 to 8)
    int64_t row, step;      // first row and distance to the next
    int count, rounds;      // rows of this thread's group; rounds of the block
};

// `contiguous`: each group of lanes walks its own run of rows (sums over the rows
// of a gate stay with one group); otherwise a block's groups take neighbouring rows.
__device__ __forceinline__ Place place(const NormParams &p, bool contiguous)
{
    Place q;
    const int rank = blockIdx.x % p.cluster, id = blockIdx.x / p.cluster;
    const int lane = threadIdx.x % p.lanes, group = threadIdx.x / p.lanes;
    const int first = rank * p.cta_cols + lane * 8;
    q.n = lane * 8 < p.cta_cols ? max(0, min(8, p.cols - first)) : 0;
    q.col = q.n > 0 ? first : 0;
    if (contiguous) {
        const int64_t workers = (int64_t)p.ctas * p.row_groups, me = (int64_t)id * p.row_groups + group;
        q.row = p.rows * me / workers;
        q.step = 1;
        q.count = (int)(p.rows * (me + 1) / workers - q.row);
        q.rounds = (int)((p.rows + workers - 1) / workers);
    } else {
        const int64_t begin = p.rows * id / p.ctas, end = p.rows * (id + 1) / p.ctas;
        q.row = begin + group;
        q.step = p.row_groups;
        q.count = (int)max((int64_t)0, (end - q.row + p.row_groups - 1) / p.row_groups);
        q.rounds = (int)((end - begin + p.row_groups - 1) / p.row_groups);
    }
    return q;
}

template <typename A> __device__ __forceinline__ void stage_gate(const NormParams &p, uint32_t slot, uint32_t stride, int64_t row,
                                                                 const Place &q)
{
    const int64_t at = row / p.gate_rows * p.gate.stride + q.col;
    if (p.gate_f32)
        stage8(slot, stride, static_cast<const float *>(p.gate.data) + at, q.n, p.wide_gate);
    else
        stage8(slot, stride, static_cast<const A *>(p.gate.data) + at, q.n, p.wide_gate);
}

template <typename A> __device__ __forceinline__ void fetch_gate(const NormParams &p, uint32_t slot, uint32_t stride, float (&v)[8])
{
    if (p.gate_f32)
        fetch8<float>(slot, stride, v);
    else
        fetch8<A>(slot, stride, v);
}

__device__ __forceinline__ void clear_slots(const NormParams &p, uint32_t slot, uint32_t stride)
{
    for (int i = 0; i < p.units * p.stages; ++i)
        smem_put(slot + i * stride, make_uint4(0, 0, 0, 0));
}

// ------------------------------------------------------------------- forward

template <typename A, typename R>
__global__ void __launch_bounds__(kNormMaxThreads, kNormForwardThreads / kNormMaxThreads)
    rikfad_norm_forward_kernel(const __grid_constant__ NormParams p)
{
    extern __shared__ uint4 stages[];
    __shared__ RowSums sums;
    const Place q = place(p, false);
    const uint32_t stride = p.threads * 16, slot = smem_address(stages + threadIdx.x);
    const uint32_t stage_bytes = stride * p.units;
    const bool branch = p.z.data != nullptr, gated = p.gate.data != nullptr;
    int parity = 0;
    for (int i = threadIdx.x; i < (int)(sizeof sums / 4); i += p.threads)
        (&sums.slot[0][0][0])[i] = 0.f;
    if (q.n == 0)
        clear_slots(p, slot, stride);
    if (p.cluster > 1)
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    else
        __syncthreads();
    wait_for_predecessor();
    auto issue = [&](int k) {
        if (k < q.count && q.n > 0) {
            const int64_t row = q.row + k * q.step;
            uint32_t at = slot + (uint32_t)(k % p.stages) * stage_bytes;
            stage8(at, stride, static_cast<const R *>(p.x.data) + row * p.x.stride + q.col, q.n, p.wide_x);
            at += kUnits<R> * stride;
            if (branch) {
                stage8(at, stride, static_cast<const A *>(p.z.data) + row * p.z.stride + q.col, q.n, p.wide_z);
                at += kUnits<A> * stride;
            }
            if (gated)
                stage_gate<A>(p, at, stride, row, q);
        }
        commit_copies();
    };
    for (int k = 0; k < p.stages - 1; ++k)
        issue(k);
    for (int k = 0; k < q.rounds; ++k) {
        issue(k + p.stages - 1);
        wait_copies(p.stages);
        const int64_t row = q.row + k * q.step;
        const bool live = k < q.count;
        uint32_t at = slot + (uint32_t)(k % p.stages) * stage_bytes;
        float u[8], m2 = 0.f, r2 = 1.f, m1, r1;
        fetch8<R>(at, stride, u);
        at += kUnits<R> * stride;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            u[e] *= p.a;
        if (branch) {
            float v[8], w[8];
            fetch8<A>(at, stride, v);
            at += kUnits<A> * stride;
            row_stats(p, sums, parity, p.post, p.post_eps, q.n, v, m2, r2);
            if (p.post != RIKFAD_NORM_NONE) {
                param8<A>(p.post_weight, p.param_f32, q.col, q.n, p.wide_params, 1.f, w);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    v[e] = (v[e] - m2) * r2 * w[e];
                if (p.post_bias) {
                    param8<A>(p.post_bias, p.param_f32, q.col, q.n, p.wide_params, 0.f, w);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        v[e] += w[e];
                }
            }
            if (gated) {
                fetch_gate<A>(p, at, stride, w);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    v[e] *= w[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e)
                u[e] = fmaf(p.b, v[e], u[e]);
        }
        row_stats(p, sums, parity, p.pre, p.pre_eps, q.n, u, m1, r1);
        if (live && q.n > 0) {
            if (p.u.data)
                put8(static_cast<R *>(p.u.data) + row * p.u.stride + q.col, u, q.n, p.wide_u);
            if (p.h.data) {
                if (p.pre != RIKFAD_NORM_NONE) {
                    float w[8];
                    param8<A>(p.pre_weight, p.param_f32, q.col, q.n, p.wide_params, 1.f, w);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        u[e] = (u[e] - m1) * r1 * w[e];
                    if (p.pre_bias) {
                        param8<A>(p.pre_bias, p.param_f32, q.col, q.n, p.wide_params, 0.f, w);
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            u[e] += w[e];
                    }
                }
                put8(static_cast<A *>(p.h.data) + row * p.h.stride + q.col, u, q.n, p.wide_h);
            }
            if (p.stats && q.col == 0)
                p.stats[row] = make_float4(m2, r2, m1, r1);
        }
    }
    allow_successor_launch();
}

// ------------------------------------------------------------------ backward

// One partial row of a sum over rows, from the block's groups in order.
__device__ __forceinline__ void store_sum(const NormParams &p, const Place &q, float *part, int id, float *buffer, const float (&acc)[8])
{
    float *out = part + (int64_t)id * p.cols;
    if (p.row_groups == 1) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < q.n)
                out[q.col + e] = acc[e];
        return;
    }
    __syncthreads();
    const int group = threadIdx.x / p.lanes, width = p.lanes * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        buffer[group * width + (threadIdx.x % p.lanes) * 8 + e] = acc[e];
    __syncthreads();
    for (int c = threadIdx.x; c < p.cols; c += p.threads) {
        float t = 0.f;
        for (int g = 0; g < p.row_groups; ++g)
            t += buffer[g * width + c];
        out[c] = t;
    }
}

template <typename A, typename R, bool BIAS>
__global__ void __launch_bounds__(kNormMaxThreads, kNormBackwardThreads / kNormMaxThreads)
    rikfad_norm_backward_kernel(const __grid_constant__ NormParams p)
{
    extern __shared__ uint4 stages[];
    __shared__ RowSums sums;
    const Place q = place(p, p.shared_gate);
    const uint32_t stride = p.threads * 16, slot = smem_address(stages + threadIdx.x);
    const uint32_t stage_bytes = stride * p.units;
    const bool branch = p.z.data != nullptr, gated = p.gate.data != nullptr;
    const bool post = branch && p.post != RIKFAD_NORM_NONE, pre = p.pre != RIKFAD_NORM_NONE;
    int parity = 0;
    for (int i = threadIdx.x; i < (int)(sizeof sums / 4); i += p.threads)
        (&sums.slot[0][0][0])[i] = 0.f;
    if (q.n == 0)
        clear_slots(p, slot, stride);
    if (p.cluster > 1)
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    else
        __syncthreads();
    wait_for_predecessor();
    // a thread's slots of a row: x, z, dh, du, gate
    const uint32_t z_at = kUnits<R> * stride, dh_at = z_at + kUnits<A> * stride, du_at = dh_at + kUnits<A> * stride;
    const uint32_t gate_at = du_at + kUnits<R> * stride;
    auto issue = [&](int k) {
        if (k < q.count && q.n > 0) {
            const int64_t row = q.row + k * q.step;
            const uint32_t at = slot + (uint32_t)(k % p.stages) * stage_bytes;
            stage8(at, stride, static_cast<const R *>(p.x.data) + row * p.x.stride + q.col, q.n, p.wide_x);
            if (branch)
                stage8(at + z_at, stride, static_cast<const A *>(p.z.data) + row * p.z.stride + q.col, q.n, p.wide_z);
            if (p.dh.data)
                stage8(at + dh_at, stride, static_cast<const A *>(p.dh.data) + row * p.dh.stride + q.col, q.n, p.wide_dh);
            if (p.du.data)
                stage8(at + du_at, stride, static_cast<const R *>(p.du.data) + row * p.du.stride + q.col, q.n, p.wide_du);
            if (gated)
                stage_gate<A>(p, at + gate_at, stride, row, q);
        }
        commit_copies();
    };
    float dw1[8] = {}, dw2[8] = {}, db1[8] = {}, db2[8] = {}, dg[8] = {};
    int64_t gate_row = q.row / p.gate_rows;     // of the sum in dg
    int64_t gate_left = p.shared_gate ? (gate_row + 1) * p.gate_rows - q.row : 0;
    bool gate_whole = q.row % p.gate_rows == 0; // the sum began with the gate's first row
    int gate_slot = 0;                          // 0: the group's first gate, 1: its last
    const int64_t worker = (int64_t)(blockIdx.x / p.cluster) * p.row_groups + threadIdx.x / p.lanes;
    if (p.shared_gate && q.count == 0)          // a group without rows adds nothing to the gate it lies in
        for (int e = 0; e < q.n; ++e)
            p.gate_part[2 * worker * p.cols + q.col + e] = 0.f;
    for (int k = 0; k < p.stages - 1; ++k)
        issue(k);
    float4 next = q.count > 0 ? p.stats[q.row] : make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k = 0; k < q.rounds; ++k) {
        issue(k + p.stages - 1);
        const int64_t row = q.row + k * q.step;
        const bool live = k < q.count;
        const float m2 = next.x, r2 = next.y, m1 = next.z, r1 = next.w;
        if (k + 1 < q.count)
            next = p.stats[row + q.step];
        wait_copies(p.stages);
        const uint32_t at = slot + (uint32_t)(k % p.stages) * stage_bytes;
        float y1[8], y2[8], n[8], gate[8], g1[8], w[8];
        fetch8<R>(at, stride, y1);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            y1[e] *= p.a;
            y2[e] = n[e] = 0.f;
            gate[e] = 1.f;
        }
        if (branch) {
            fetch8<A>(at + z_at, stride, n);
            if (post) {
                param8<A>(p.post_weight, p.param_f32, q.col, q.n, p.wide_params, 1.f, w);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    y2[e] = (n[e] - m2) * r2;
                    n[e] = y2[e] * w[e];
                }
                if (p.post_bias) {
                    param8<A>(p.post_bias, p.param_f32, q.col, q.n, p.wide_params, 0.f, w);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        n[e] += w[e];
                }
            }
            if (gated)
                fetch_gate<A>(p, at + gate_at, stride, gate);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                y1[e] = fmaf(p.b, gate[e] * n[e], y1[e]);
        }
        float e1[8];            // du, then the gradient of u
        if (p.du.data)
            fetch8<R>(at + du_at, stride, e1);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e)
                e1[e] = 0.f;
        if (p.dh.data)
            fetch8<A>(at + dh_at, stride, g1);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e)
                g1[e] = 0.f;
        if (pre) {
            param8<A>(p.pre_weight, p.param_f32, q.col, q.n, p.wide_params, 1.f, w);
            float t[2] = {0.f, 0.f};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                y1[e] = (y1[e] - m1) * r1;
                if (live) {
                    dw1[e] = fmaf(g1[e], y1[e], dw1[e]);
                    if (BIAS)
                        db1[e] += g1[e];
                }
                g1[e] *= w[e];
                t[0] = fmaf(g1[e], y1[e], t[0]);
                t[1] += g1[e];
            }
            row_sum(p, sums, parity, t);
            t[0] *= p.inv_cols;
            t[1] = p.pre == RIKFAD_NORM_LAYER ? t[1] * p.inv_cols : 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                e1[e] = fmaf(r1, (g1[e] - t[1]) - y1[e] * t[0], e1[e]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                e1[e] += g1[e];
        }
        if (live && q.n > 0 && p.dx.data) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                w[e] = p.a * e1[e];
            put8(static_cast<R *>(p.dx.data) + row * p.dx.stride + q.col, w, q.n, p.wide_dx);
        }
        if (branch) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                e1[e] *= p.b;
            if (p.shared_gate) {
                if (live)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        dg[e] = fmaf(e1[e], n[e], dg[e]);
                // The gate's last row, or the group's: a gate that lies within the
                // group is done, others leave a partial sum.
                if (live && (--gate_left == 0 || k + 1 == q.count)) {
                    const bool whole = gate_whole && gate_left == 0;
                    if (whole) {
                        const int64_t to = gate_row * p.dgate.stride + q.col;
                        if (q.n > 0) {
                            if (p.gate_f32)
                                put8(static_cast<float *>(p.dgate.data) + to, dg, q.n, p.wide_dgate);
                            else
                                put8(static_cast<A *>(p.dgate.data) + to, dg, q.n, p.wide_dgate);
                        }
                    } else {
                        float *part = p.gate_part + (2 * worker + gate_slot) * p.cols + q.col;
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (e < q.n)
                                part[e] = dg[e];
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        dg[e] = 0.f;
                    ++gate_row;
                    gate_left = p.gate_rows;
                    gate_whole = true;
                    gate_slot = 1;
                }
            } else if (p.dgate.data && live && q.n > 0) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    w[e] = e1[e] * n[e];
                const int64_t to = row * p.dgate.stride + q.col;
                if (p.gate_f32)
                    put8(static_cast<float *>(p.dgate.data) + to, w, q.n, p.wide_dgate);
                else
                    put8(static_cast<A *>(p.dgate.data) + to, w, q.n, p.wide_dgate);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e)
                e1[e] *= gate[e];
            if (post) {
                param8<A>(p.post_weight, p.param_f32, q.col, q.n, p.wide_params, 1.f, w);
                float t[2] = {0.f, 0.f};
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (live) {
                        dw2[e] = fmaf(e1[e], y2[e], dw2[e]);
                        if (BIAS)
                            db2[e] += e1[e];
                    }
                    e1[e] *= w[e];
                    t[0] = fmaf(e1[e], y2[e], t[0]);
                    t[1] += e1[e];
                }
                row_sum(p, sums, parity, t);
                t[0] *= p.inv_cols;
                t[1] = p.post == RIKFAD_NORM_LAYER ? t[1] * p.inv_cols : 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    e1[e] = r2 * ((e1[e] - t[1]) - y2[e] * t[0]);
            }
            if (live && q.n > 0 && p.dz.data)
                put8(static_cast<A *>(p.dz.data) + row * p.dz.stride + q.col, e1, q.n, p.wide_dz);
        }
    }
    allow_successor_launch();
    asm volatile("cp.async.wait_all;" ::: "memory");
    float *part = p.sum_part;
    float *buffer = reinterpret_cast<float *>(stages);
    const int id = blockIdx.x / p.cluster;
    const int64_t size = (int64_t)p.ctas * p.cols;
    if (p.dpre_weight) {
        store_sum(p, q, part, id, buffer, dw1);
        part += size;
    }
    if (p.dpost_weight) {
        store_sum(p, q, part, id, buffer, dw2);
        part += size;
    }
    if (BIAS && p.dpre_bias) {
        store_sum(p, q, part, id, buffer, db1);
        part += size;
    }
    if (BIAS && p.dpost_bias)
        store_sum(p, q, part, id, buffer, db2);
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

template <typename A, typename R> cudaError_t launch_norm(const NormParams &n, bool backward, cudaStream_t s)
{
    if (!backward)
        return launch_clustered(rikfad_norm_forward_kernel<A, R>, n, s);
    const bool bias = n.dpre_bias || n.dpost_bias;
    const cudaError_t e = bias ? launch_clustered(rikfad_norm_backward_kernel<A, R, true>, n, s)
                               : launch_clustered(rikfad_norm_backward_kernel<A, R, false>, n, s);
    if (e != cudaSuccess || (n.sums == 0 && !n.shared_gate))
        return e;
    const int64_t gates = n.shared_gate ? n.rows / n.gate_rows : 0;
    const dim3 grid((unsigned)((n.cols + 31) / 32), (unsigned)(n.sums + (gates < 1024 ? gates : 1024)));
    return launch_chained(rikfad_norm_join_kernel<A>, grid, 32 * kJoinRows, 0, s, n);
}

}  // namespace rikfad
