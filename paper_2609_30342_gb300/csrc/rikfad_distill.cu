// rikfad_distill.cu -- loss of rows of logits s against a teacher's top logits t at
// indices i and a label, and its gradient:
//   p = softmax(t / T), q_T = softmax(s / T), q_1 = softmax(s)
//   loss = a T^2 sum_k p_k (log p_k - log q_T[i_k]) - b log q_1[label]
//   ds = g (a T (q_T - p) + b (q_1 - e_label))
//
// Everything is in powers of two of x c - r, with c = log2(e) / T (or log2(e)) and a
// reference r = max(x) c that is rounded once and used alike for sums, losses and
// gradients: its rounding cancels.
//
// Memory bounds it: the logits are read once for the sums (and once more for the
// gradient), the gradient is written once.
#include <cuda_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <new>
#include <string>

#include "rikfad.h"
#include "rikfad_host.hpp"
#include "rikfad_kernels.cuh"
#include "rikfad_types.cuh"

using namespace rikfad;

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kSms = 152;
constexpr int kMaxEntries = 1024;           // of a teacher's row
constexpr int kMaxCluster = 8;
// A reference's rounding is a factor of up to 2^(r 2^-24) in every power: r stays below
// this, and lower logits count as the one there.
constexpr float kFarthest = 0x1p29f;
constexpr int kAhead = 4;                   // vectors of a thread under way

struct Params {
    const void *logits, *teacher, *index, *labels;
    void *dlogits;
    const float *dloss;
    float *loss;
    float4 *stats;                  // r and sum at temperature T, r and sum at 1
    int64_t rows, logits_stride, teacher_stride, index_stride, dlogits_stride;
    int32_t vocab, k, teacher_dtype, index_bytes, label_bytes;
    int32_t cluster;                // blocks of a row
    bool distils, labelled;         // the terms that the call has
    bool wide;                      // every row of dlogits starts as far from 16 bytes as the logits'
    float a, b;                     // a T and b, of the gradient
    float loss_a, loss_b;           // a T^2 ln 2 and b ln 2
    float c_t, c_1, grad_scale;     // log2(e) / T, log2(e)
    float lowest;                   // finite logits below it count as it
};

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
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

// A maximum and the sums of 2^(x c - r), r = max c, at two temperatures.
struct Sums {
    float top, t, one;

    __device__ __forceinline__ static float reference(float top, float c)
    {
        const float r = top * c;
        return top == -INFINITY ? 0.f : r > kFarthest ? INFINITY : r;
    }
    // What a part's sum counts for a larger maximum.
    __device__ __forceinline__ static float moved(float sum, float from, float to, float c)
    {
        return sum == 0.f ? 0.f : sum * exp2_fast(reference(from, c) - reference(to, c));
    }
    __device__ __forceinline__ void add(const Sums &o, float c_t, float c_1)
    {
        const float m = fmaxf(top, o.top);
        t = moved(t, top, m, c_t) + moved(o.t, o.top, m, c_t);
        one = moved(one, top, m, c_1) + moved(o.one, o.top, m, c_1);
        top = m;
    }
};

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

template <typename T, Mode MODE>
__global__ void __launch_bounds__(kThreads) rikfad_distill_kernel(const __grid_constant__ Params p)
{
    constexpr int V = 16 / sizeof(T);
    extern __shared__ float entries[];
    const int count = p.k + 1;                          // the label is the last entry
    float *teacher = entries, *at_index = teacher + count;      // logits of the teacher, of the row at the indices
    int *index = reinterpret_cast<int *>(at_index + count);
    int *own = index + count;                           // entries of the block's slice, in order
    __shared__ Sums warp_sums[kWarps];
    __shared__ float2 warp_teacher[kWarps];
    __shared__ float warp_loss[kWarps];
    __shared__ float parts[kMaxCluster][3];
    __shared__ int own_count;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int rank = p.cluster > 1 ? (int)(blockIdx.x % p.cluster) : 0;
    const int64_t r = p.cluster > 1 ? blockIdx.x / p.cluster : blockIdx.x;
    wait_for_predecessor();
    allow_successor_launch();
    if (MODE != kBackward && p.cluster > 1)
        cluster_arrive();                               // the others have begun
    const T *row = static_cast<const T *>(p.logits) + r * p.logits_stride;
    const Slice<T> slice(row, p.vocab, p.cluster, rank);
    const uint4 *vectors = reinterpret_cast<const uint4 *>(row + slice.lead);

    // The entries: indices, the teacher's logits and the row's.  One that is absent, or
    // whose logit is -inf, has index -1.
    bool present = false;
    float teacher_top = -INFINITY, teacher_sum = 0.f;
    for (int e = threadIdx.x; e < count; e += kThreads) {
        int64_t i = -1;
        float t = 0.f;
        if (e < p.k) {
            if (p.distils) {
                i = integer_at(p.index, p.index_bytes, r * p.index_stride + e);
                t = float_at(p.teacher, p.teacher_dtype, r * p.teacher_stride + e);
                i = t == -INFINITY ? -1 : i;
                t = at_least(t, p.lowest);
            }
        } else if (p.labelled)
            i = integer_at(p.labels, p.label_bytes, r);
        const bool here = i >= 0 && i < p.vocab;
        index[e] = here ? (int)i : -1;
        teacher[e] = t;
        at_index[e] = here ? to_f32(row[i]) : 0.f;
        if (here && e < p.k) {
            present = true;
            const float m = fmaxf(teacher_top, t);
            teacher_sum = Sums::moved(teacher_sum, teacher_top, m, p.c_t) + exp2_fast(fmaf(t, p.c_t, -Sums::reference(m, p.c_t)));
            teacher_top = m;
        }
    }
    const bool distils = __syncthreads_or(present);
    const bool labelled = index[p.k] >= 0;

    Sums sums = {-INFINITY, 0.f, 0.f};
    if (MODE != kBackward) {
        // this thread's maximum and sums, kAhead vectors at a time
        auto take = [&](float (&x)[V], float top) {
            if (top < p.lowest) {       // masked with the type's lowest value: such elements count if the row has no others
#pragma unroll
                for (int e = 0; e < V; ++e)
                    x[e] = at_least(x[e], p.lowest);
                top = at_least(top, p.lowest);
            }
            if (top > sums.top) {
                sums.t = Sums::moved(sums.t, sums.top, top, p.c_t);
                sums.one = Sums::moved(sums.one, sums.top, top, p.c_1);
                sums.top = top;
            }
            const float r_t = Sums::reference(sums.top, p.c_t), r_1 = Sums::reference(sums.top, p.c_1);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                sums.t += exp2_fast(fmaf(x[e], p.c_t, -r_t));
                sums.one += exp2_fast(fmaf(x[e], p.c_1, -r_1));
            }
        };
        for (int v = slice.begin + threadIdx.x; v < slice.end; v += kThreads * kAhead) {
            Vec<T, V> in[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                if (v + j * kThreads < slice.end)
                    in[j].word = vectors[v + j * kThreads];
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                if (v + j * kThreads < slice.end) {
                    float x[V], top = -INFINITY;
                    widen(in[j], x);
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        top = fmaxf(top, x[e]);
                    take(x, top);
                }
        }
        if (threadIdx.x < slice.edges) {
            const float x = at_least(to_f32(row[slice.edge(threadIdx.x)]), p.lowest);
            sums.add({x, exp2_fast(fmaf(x, p.c_t, -Sums::reference(x, p.c_t))),
                      exp2_fast(fmaf(x, p.c_1, -Sums::reference(x, p.c_1)))}, p.c_t, p.c_1);
        }
        for (int d = 16; d > 0; d /= 2) {
            const Sums o = {__shfl_xor_sync(~0u, sums.top, d), __shfl_xor_sync(~0u, sums.t, d), __shfl_xor_sync(~0u, sums.one, d)};
            sums.add(o, p.c_t, p.c_1);
        }
        if (lane == 0)
            warp_sums[warp] = sums;
    }
    if (distils) {
        for (int d = 16; d > 0; d /= 2) {
            const float top = __shfl_xor_sync(~0u, teacher_top, d), sum = __shfl_xor_sync(~0u, teacher_sum, d);
            const float m = fmaxf(teacher_top, top);
            teacher_sum = Sums::moved(teacher_sum, teacher_top, m, p.c_t) + Sums::moved(sum, top, m, p.c_t);
            teacher_top = m;
        }
        if (lane == 0)
            warp_teacher[warp] = make_float2(teacher_top, teacher_sum);
    }
    if (MODE != kForward && warp == kWarps - 1) {
        // the entries of this block's slice, in order
        int n = 0;
        for (int e0 = 0; e0 < count; e0 += 32) {
            const int e = e0 + lane;
            const bool mine = e < count && index[e] >= 0 && slice.has(index[e], rank);
            const uint32_t all = __ballot_sync(~0u, mine);
            if (mine)
                own[n + __popc(all & ((1u << lane) - 1))] = e;
            n += __popc(all);
        }
        if (lane == 0)
            own_count = n;
    }
    __syncthreads();
    if (distils) {
        teacher_top = -INFINITY;
        teacher_sum = 0.f;
        for (int w = 0; w < kWarps; ++w) {
            const float2 o = warp_teacher[w];
            const float m = fmaxf(teacher_top, o.x);
            teacher_sum = Sums::moved(teacher_sum, teacher_top, m, p.c_t) + Sums::moved(o.y, o.x, m, p.c_t);
            teacher_top = m;
        }
    }
    float r_t, r_1, sum_t, sum_1;
    if (MODE != kBackward) {
        sums = warp_sums[0];
        for (int w = 1; w < kWarps; ++w)
            sums.add(warp_sums[w], p.c_t, p.c_1);
        if (p.cluster > 1) {
            cluster_wait();
            if (threadIdx.x < p.cluster) {
                cluster_write(&parts[rank][0], threadIdx.x, sums.top);
                cluster_write(&parts[rank][1], threadIdx.x, sums.t);
                cluster_write(&parts[rank][2], threadIdx.x, sums.one);
            }
            cluster_arrive();
            cluster_wait();
            sums = {parts[0][0], parts[0][1], parts[0][2]};
            for (int c = 1; c < p.cluster; ++c)
                sums.add({parts[c][0], parts[c][1], parts[c][2]}, p.c_t, p.c_1);
        }
        r_t = Sums::reference(sums.top, p.c_t);
        r_1 = Sums::reference(sums.top, p.c_1);
        sum_t = sums.t;
        sum_1 = sums.one;
    } else {
        const float4 s = p.stats[r];
        r_t = s.x;
        sum_t = s.y;
        r_1 = s.z;
        sum_1 = s.w;
    }
    const float teacher_r = Sums::reference(teacher_top, p.c_t);
    // The row has nothing above the lowest value that counts.
    const bool low = p.c_t > p.c_1 ? r_t == p.lowest * p.c_t : r_1 == p.lowest * p.c_1;
    auto logit = [&](float x) { return low ? at_least(x, p.lowest) : x; };
    if (MODE != kBackward && rank == 0) {
        float loss = 0.f;
        if (distils) {
            const float log_q = log2f(sum_t), log_p = log2f(teacher_sum);
            for (int e = threadIdx.x; e < p.k; e += kThreads)
                if (index[e] >= 0) {
                    const float lp = fmaf(teacher[e], p.c_t, -teacher_r) - log_p;
                    const float share = exp2_fast(lp);
                    if (share != 0.f)
                        loss += share * (lp - (fmaf(logit(at_index[e]), p.c_t, -r_t) - log_q));
                }
            for (int d = 16; d > 0; d /= 2)
                loss += __shfl_xor_sync(~0u, loss, d);
            if (lane == 0)
                warp_loss[warp] = loss;
            __syncthreads();
        }
        if (threadIdx.x == 0) {
            loss = 0.f;
            if (distils) {
                for (int w = 0; w < kWarps; ++w)
                    loss += warp_loss[w];
                loss *= p.loss_a;
            }
            if (labelled)
                loss -= p.loss_b * (fmaf(logit(at_index[p.k]), p.c_1, -r_1) - log2f(sum_1));
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
    auto dense = [&](float x) {         // a term that is absent adds nothing, whatever the row holds
        float g = 0.f;
        if (distils)
            g = f_t * exp2_fast(fmaf(x, p.c_t, -r_t));
        if (labelled)
            g = fmaf(f_1, exp2_fast(fmaf(x, p.c_1, -r_1)), g);
        return g;
    };
    T *out = static_cast<T *>(p.dlogits) + r * p.dlogits_stride;
    for (int v = slice.begin + threadIdx.x; v < slice.end; v += kThreads * kAhead) {
        Vec<T, V> in[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (v + j * kThreads < slice.end)
                in[j].word = vectors[v + j * kThreads];
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (v + j * kThreads < slice.end) {
                float x[V];
                widen(in[j], x);
                if (low) {
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        x[e] = at_least(x[e], p.lowest);
                }
#pragma unroll
                for (int e = 0; e < V; ++e)
                    x[e] = dense(x[e]);
                narrow(x, in[j]);
                T *to = out + slice.lead + (int64_t)(v + j * kThreads) * V;
                if (p.wide)
                    *reinterpret_cast<uint4 *>(to) = in[j].word;
                else
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        to[e] = in[j].v[e];
            }
    }
    if (threadIdx.x < slice.edges) {
        const int e = slice.edge(threadIdx.x);
        out[e] = from_f32<T>(dense(logit(to_f32(row[e]))));
    }
    __syncthreads();
    // An element that several entries name: the first one's thread adds them up in order.
    for (int n = threadIdx.x; n < own_count; n += kThreads) {
        const int i = index[own[n]];
        float part = 0.f;
        bool first = true;
        for (int m = 0; m < own_count; ++m) {
            const int e = own[m];
            if (index[e] != i)
                continue;
            first = first && m >= n;
            part -= e < p.k ? a * exp2_fast(fmaf(teacher[e], p.c_t, -teacher_r)) / teacher_sum : b;
        }
        if (first)
            out[i] = from_f32<T>(dense(logit(at_index[own[n]])) + part);
    }
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

template <typename T, Mode MODE> cudaError_t launch(Params p, cudaStream_t s)
{
    // Few rows: several blocks for each, of 16 KB at least.
    const int64_t bytes = (int64_t)p.vocab * sizeof(T);
    p.cluster = 1;
    while (p.cluster < kMaxCluster && p.rows * p.cluster < 2 * kSms && bytes / p.cluster > 16 << 10)
        p.cluster *= 2;
    if (p.rows * p.cluster > INT32_MAX)
        return cudaErrorInvalidConfiguration;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.rows * p.cluster));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = 4 * sizeof(float) * ((size_t)p.k + 1);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)p.cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = MODE != kBackward && p.cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, rikfad_distill_kernel<T, MODE>, p);
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
    q.c_t = (float)(kLog2E / T);
    q.c_1 = (float)kLog2E;
    q.lowest = -kFarthest / std::max(q.c_t, q.c_1);
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
