// rikfad_norm.cu -- residual sum of a transformer block with the norms around it,
//   n = post(z),  u = a x + b gate (.) n,  h = pre(u),
// and its gradients.  With y2 = (z - m2) r2 and y1 = (u - m1) r1 (m = 0 for an
// RMS norm) and given du, dh:
//   g1 = dh w1,  e = du + r1 (g1 - [mean g1] - y1 mean(g1 y1))   ([.]: layer norm)
//   dx = a e,  dgate = sum over the gate's rows of b e n,  q = b gate e
//   g2 = q w2,  dz = r2 (g2 - [mean g2] - y2 mean(g2 y2))
//   dw1 = sum dh y1,  db1 = sum dh,  dw2 = sum q y2,  db2 = sum q.
// The backward kernels form u again from x, z and the gate: the same bytes as
// reading u, without the rounding that a stored u has.
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

constexpr int kNormThreads = 256;

// Element i of an array of a type known at run time.
__device__ __forceinline__ float get(const void *p, int dtype, int64_t i)
{
    return dtype == RIKFAD_F32    ? static_cast<const float *>(p)[i]
           : dtype == RIKFAD_BF16 ? to_f32(static_cast<const __nv_bfloat16 *>(p)[i])
                                  : to_f32(static_cast<const __half *>(p)[i]);
}

__device__ __forceinline__ void put(void *p, int dtype, int64_t i, float v)
{
    if (dtype == RIKFAD_F32)
        static_cast<float *>(p)[i] = v;
    else if (dtype == RIKFAD_BF16)
        static_cast<__nv_bfloat16 *>(p)[i] = from_f32<__nv_bfloat16>(v);
    else
        static_cast<__half *>(p)[i] = from_f32<__half>(v);
}

struct NormParams {
    rikfad_residual_norm d;
    float a, b, post_eps, pre_eps;
    float *means;       // backward: 4 floats a row (mean g1, mean g1 y1, mean g2, mean g2 y2)
};

__device__ float block_sum(float v, float *red)
{
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0)
        red[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.f;
    for (int w = 0; w < kNormThreads / 32; ++w)
        v += red[w];
    return v;
}

struct Row {
    float m2, r2, m1, r1;
};

// Column c of a row: the branch before the gate, the sum, and the gate.
__device__ __forceinline__ float branch(const NormParams &p, const Row &s, int64_t row, int64_t c, float &y2)
{
    if (p.d.z.data == nullptr)
        return y2 = 0.f;
    const float z = get(p.d.z.data, p.d.dtype, row * p.d.z.stride + c);
    y2 = (z - s.m2) * s.r2;
    float n = p.d.post_weight ? y2 * get(p.d.post_weight, p.d.param_dtype, c) : y2;
    return p.d.post_bias ? n + get(p.d.post_bias, p.d.param_dtype, c) : n;
}

__device__ __forceinline__ float gate_at(const NormParams &p, int64_t row, int64_t c)
{
    return p.d.gate.data ? get(p.d.gate.data, p.d.gate_dtype, row / p.d.gate_rows * p.d.gate.stride + c) : 1.f;
}

__device__ __forceinline__ float sum_at(const NormParams &p, const Row &s, int64_t row, int64_t c)
{
    float y2;
    const float n = branch(p, s, row, c, y2);
    return fmaf(p.b, gate_at(p, row, c) * n, p.a * get(p.d.x.data, p.d.residual_dtype, row * p.d.x.stride + c));
}

template <typename F> __device__ void norm_stats(int kind, float eps, int64_t cols, float *red, F at, float &m, float &r)
{
    m = 0.f;
    r = 1.f;
    if (kind == RIKFAD_NORM_NONE)
        return;
    if (kind == RIKFAD_NORM_LAYER) {
        float s = 0.f;
        for (int64_t c = threadIdx.x; c < cols; c += kNormThreads)
            s += at(c);
        m = block_sum(s, red) / (float)cols;
    }
    float s = 0.f;
    for (int64_t c = threadIdx.x; c < cols; c += kNormThreads) {
        const float v = at(c) - m;
        s = fmaf(v, v, s);
    }
    r = rsqrtf(block_sum(s, red) / (float)cols + eps);
}

__global__ void __launch_bounds__(kNormThreads) rikfad_norm_forward_kernel(const __grid_constant__ NormParams p)
{
    __shared__ float red[kNormThreads / 32];
    for (int64_t row = blockIdx.x; row < p.d.rows; row += gridDim.x) {
        Row s{0.f, 1.f, 0.f, 1.f};
        if (p.d.z.data)
            norm_stats(p.d.post, p.post_eps, p.d.cols, red,
                       [&](int64_t c) { return get(p.d.z.data, p.d.dtype, row * p.d.z.stride + c); }, s.m2, s.r2);
        norm_stats(p.d.pre, p.pre_eps, p.d.cols, red, [&](int64_t c) { return sum_at(p, s, row, c); }, s.m1, s.r1);
        __syncthreads();        // every read of the row's inputs before the writes, which may go to them
        for (int64_t c = threadIdx.x; c < p.d.cols; c += kNormThreads) {
            const float u = sum_at(p, s, row, c);
            if (p.d.u.data)
                put(p.d.u.data, p.d.residual_dtype, row * p.d.u.stride + c, u);
            if (p.d.h.data) {
                float h = (u - s.m1) * s.r1;
                if (p.d.pre_weight)
                    h *= get(p.d.pre_weight, p.d.param_dtype, c);
                if (p.d.pre_bias)
                    h += get(p.d.pre_bias, p.d.param_dtype, c);
                put(p.d.h.data, p.d.dtype, row * p.d.h.stride + c, h);
            }
        }
        if (p.d.stats && threadIdx.x == 0)
            reinterpret_cast<float4 *>(p.d.stats)[row] = make_float4(s.m2, s.r2, s.m1, s.r1);
    }
}

// One element of the backward pass.
struct Element {
    float y1, y2, n, gate, g1, dh, e, q, g2;
};

__device__ __forceinline__ Element element(const NormParams &p, const Row &s, int64_t row, int64_t c, float mg1, float mg1y)
{
    Element v;
    v.n = branch(p, s, row, c, v.y2);
    v.gate = gate_at(p, row, c);
    const float u = fmaf(p.b, v.gate * v.n, p.a * get(p.d.x.data, p.d.residual_dtype, row * p.d.x.stride + c));
    v.y1 = (u - s.m1) * s.r1;
    v.dh = p.d.dh.data ? get(p.d.dh.data, p.d.dtype, row * p.d.dh.stride + c) : 0.f;
    v.g1 = p.d.pre_weight ? v.dh * get(p.d.pre_weight, p.d.param_dtype, c) : v.dh;
    v.e = s.r1 * (v.g1 - mg1 - v.y1 * mg1y);
    if (p.d.du.data)
        v.e += get(p.d.du.data, p.d.residual_dtype, row * p.d.du.stride + c);
    v.q = p.b * v.gate * v.e;
    v.g2 = p.d.post_weight ? v.q * get(p.d.post_weight, p.d.param_dtype, c) : v.q;
    return v;
}

__global__ void __launch_bounds__(kNormThreads) rikfad_norm_rows_kernel(const __grid_constant__ NormParams p)
{
    __shared__ float red[kNormThreads / 32];
    const float inv = 1.f / (float)p.d.cols;
    for (int64_t row = blockIdx.x; row < p.d.rows; row += gridDim.x) {
        const float4 st = reinterpret_cast<const float4 *>(p.d.stats)[row];
        const Row s{st.x, st.y, st.z, st.w};
        float s1 = 0.f, s2 = 0.f, mg1 = 0.f, mg1y = 0.f, mg2 = 0.f, mg2y = 0.f;
        if (p.d.pre != RIKFAD_NORM_NONE) {
            for (int64_t c = threadIdx.x; c < p.d.cols; c += kNormThreads) {
                const Element v = element(p, s, row, c, 0.f, 0.f);
                s1 += v.g1;
                s2 = fmaf(v.g1, v.y1, s2);
            }
            mg1 = p.d.pre == RIKFAD_NORM_LAYER ? block_sum(s1, red) * inv : 0.f;
            mg1y = block_sum(s2, red) * inv;
        }
        if (p.d.z.data && p.d.post != RIKFAD_NORM_NONE) {
            s1 = s2 = 0.f;
            for (int64_t c = threadIdx.x; c < p.d.cols; c += kNormThreads) {
                const Element v = element(p, s, row, c, mg1, mg1y);
                s1 += v.g2;
                s2 = fmaf(v.g2, v.y2, s2);
            }
            mg2 = p.d.post == RIKFAD_NORM_LAYER ? block_sum(s1, red) * inv : 0.f;
            mg2y = block_sum(s2, red) * inv;
        }
        if (threadIdx.x == 0)
            reinterpret_cast<float4 *>(p.means)[row] = make_float4(mg1, mg1y, mg2, mg2y);
    }
}

// dx, dz and the gate's gradient where every row has its own gate.
__global__ void __launch_bounds__(kNormThreads) rikfad_norm_elements_kernel(const __grid_constant__ NormParams p)
{
    for (int64_t row = blockIdx.x; row < p.d.rows; row += gridDim.x) {
        const float4 st = reinterpret_cast<const float4 *>(p.d.stats)[row];
        const float4 mean = reinterpret_cast<const float4 *>(p.means)[row];
        const Row s{st.x, st.y, st.z, st.w};
        for (int64_t c = threadIdx.x; c < p.d.cols; c += kNormThreads) {
            const Element v = element(p, s, row, c, mean.x, mean.y);
            if (p.d.dgate.data && p.d.gate_rows == 1)
                put(p.d.dgate.data, p.d.gate_dtype, row * p.d.dgate.stride + c, p.b * v.e * v.n);
            if (p.d.dx.data)
                put(p.d.dx.data, p.d.residual_dtype, row * p.d.dx.stride + c, p.a * v.e);
            if (p.d.dz.data)
                put(p.d.dz.data, p.d.dtype, row * p.d.dz.stride + c, s.r2 * (v.g2 - mean.z - v.y2 * mean.w));
        }
    }
}

// Sums over rows: blockIdx.y = 0 over all of them for the weights and biases,
// 1 + i over gate row i's.  A thread owns a column.  Runs before the kernel
// that may overwrite the inputs.
__global__ void __launch_bounds__(kNormThreads) rikfad_norm_columns_kernel(const __grid_constant__ NormParams p)
{
    const int64_t c = (int64_t)blockIdx.x * kNormThreads + threadIdx.x;
    if (c >= p.d.cols)
        return;
    const int64_t groups = p.d.dgate.data && p.d.gate_rows != 1 ? p.d.rows / p.d.gate_rows : 0;
    for (int64_t g = blockIdx.y; g <= groups; g += gridDim.y) {
        const int64_t begin = g == 0 ? 0 : (g - 1) * p.d.gate_rows;
        const int64_t end = g == 0 ? p.d.rows : g * p.d.gate_rows;
        float dw1 = 0.f, db1 = 0.f, dw2 = 0.f, db2 = 0.f, dg = 0.f;
        for (int64_t row = begin; row < end; ++row) {
            const float4 st = reinterpret_cast<const float4 *>(p.d.stats)[row];
            const float4 mean = reinterpret_cast<const float4 *>(p.means)[row];
            const Element v = element(p, Row{st.x, st.y, st.z, st.w}, row, c, mean.x, mean.y);
            dw1 = fmaf(v.dh, v.y1, dw1);
            db1 += v.dh;
            dw2 = fmaf(v.q, v.y2, dw2);
            db2 += v.q;
            dg = fmaf(p.b * v.e, v.n, dg);
        }
        if (g > 0) {
            put(p.d.dgate.data, p.d.gate_dtype, (g - 1) * p.d.dgate.stride + c, dg);
            continue;
        }
        if (p.d.dpre_weight)
            put(p.d.dpre_weight, p.d.param_dtype, c, dw1);
        if (p.d.dpre_bias)
            put(p.d.dpre_bias, p.d.param_dtype, c, db1);
        if (p.d.dpost_weight)
            put(p.d.dpost_weight, p.d.param_dtype, c, dw2);
        if (p.d.dpost_bias)
            put(p.d.dpost_bias, p.d.param_dtype, c, db2);
    }
}

int bad(const std::string &msg) { return report_error(RIKFAD_ERR_ARG, msg); }

int check_sizes(const rikfad_residual_norm *p)
{
    if (p == nullptr)
        return bad("p is NULL");
    if (p->rows < 0 || p->rows > (int64_t)1 << 40)
        return bad("rows is out of range");
    if (p->cols < 1 || p->cols > 32768)
        return bad("cols must be in [1, 32768]");
    if (!dtype_ok(p->dtype))
        return bad("dtype is not a rikfad_dtype");
    for (const int t : {p->residual_dtype, p->param_dtype, p->gate_dtype})
        if (t != RIKFAD_F32 && t != p->dtype)
            return bad("residual_dtype, param_dtype and gate_dtype must be RIKFAD_F32 or dtype");
    for (const int k : {p->post, p->pre})
        if (k != RIKFAD_NORM_NONE && k != RIKFAD_NORM_RMS && k != RIKFAD_NORM_LAYER)
            return bad("post and pre must be a rikfad_norm");
    for (const double v : {p->post_eps, p->pre_eps})
        if (!(std::isfinite(v) && v >= 0))
            return bad("post_eps and pre_eps must be finite and >= 0");
    for (const double v : {p->residual_scale, p->branch_scale})
        if (!std::isfinite(v))
            return bad("residual_scale and branch_scale must be finite");
    if (p->gate.data && (p->gate_rows < 1 || p->rows % p->gate_rows))
        return bad("gate_rows must be >= 1 and divide rows");
    if (p->rows > 0 && p->z.data == nullptr && (p->gate.data || p->post != RIKFAD_NORM_NONE || p->post_weight || p->post_bias))
        return bad("a post norm, its weights or a gate need z");
    if ((p->post == RIKFAD_NORM_NONE && (p->post_weight || p->post_bias)) ||
        (p->pre == RIKFAD_NORM_NONE && (p->pre_weight || p->pre_bias)))
        return bad("weights and biases need their norm");
    return RIKFAD_OK;
}

int check_rows(const rikfad_rows &r, const char *name, int dtype, int64_t rows, int64_t cols, int device)
{
    if (r.data == nullptr)
        return RIKFAD_OK;
    if (rows > 1 && (r.stride < cols || r.stride > (int64_t)1 << 40))
        return bad(std::string("the row stride of ") + name + " must be at least cols");
    if ((uintptr_t)r.data % (uintptr_t)dtype_bytes(dtype))
        return report_error(RIKFAD_ERR_ALIGN, std::string(name) + " is not aligned to its element type");
    return check_address(r.data, device, name);
}

int check_vector(const void *v, const char *name, size_t align, int device)
{
    if (v == nullptr)
        return RIKFAD_OK;
    if ((uintptr_t)v % align)
        return report_error(RIKFAD_ERR_ALIGN, std::string(name) + " is not aligned");
    return check_address(v, device, name);
}

int check_inputs(const rikfad_residual_norm *p, int &device)
{
    int rc = check_sizes(p);
    if (rc)
        return rc;
    const cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess)
        return report_cuda(e, "cudaGetDevice");
    if (p->rows > 0 && p->x.data == nullptr)
        return bad("x is NULL");
    const int64_t groups = p->gate.data ? p->rows / p->gate_rows : 0;
    const size_t pb = (size_t)dtype_bytes(p->param_dtype);
    if (!rc) rc = check_rows(p->x, "x", p->residual_dtype, p->rows, p->cols, device);
    if (!rc) rc = check_rows(p->z, "z", p->dtype, p->rows, p->cols, device);
    if (!rc) rc = check_rows(p->gate, "gate", p->gate_dtype, groups, p->cols, device);
    if (!rc) rc = check_vector(p->post_weight, "post_weight", pb, device);
    if (!rc) rc = check_vector(p->post_bias, "post_bias", pb, device);
    if (!rc) rc = check_vector(p->pre_weight, "pre_weight", pb, device);
    if (!rc) rc = check_vector(p->pre_bias, "pre_bias", pb, device);
    if (!rc) rc = check_vector(p->stats, "stats", 16, device);
    return rc;
}

NormParams params(const rikfad_residual_norm *p)
{
    NormParams n{};
    n.d = *p;
    n.a = (float)p->residual_scale;
    n.b = (float)p->branch_scale;
    n.post_eps = (float)p->post_eps;
    n.pre_eps = (float)p->pre_eps;
    n.means = static_cast<float *>(p->workspace);
    return n;
}

unsigned row_blocks(int64_t rows) { return (unsigned)std::min<int64_t>(rows, 152 * 8); }

}  // namespace

extern "C" {

RIKFAD_API size_t rikfad_residual_norm_workspace(const rikfad_residual_norm *p)
{
    if (check_sizes(p))
        return 0;
    report_error(RIKFAD_OK, "");
    return (size_t)p->rows * 4 * sizeof(float);
}

RIKFAD_API int rikfad_residual_norm_forward(const rikfad_residual_norm *p, void *stream)
{
    RK_ENTRY_BEGIN
    int device = -1;
    int rc = check_inputs(p, device);
    if (!rc) rc = check_rows(p->u, "u", p->residual_dtype, p->rows, p->cols, device);
    if (!rc) rc = check_rows(p->h, "h", p->dtype, p->rows, p->cols, device);
    if (rc)
        return rc;
    cudaError_t e = cudaPeekAtLastError();
    if (e != cudaSuccess)
        return report_cuda(e, "earlier CUDA error");
    if (p->rows == 0)
        return RIKFAD_OK;
    rikfad_norm_forward_kernel<<<row_blocks(p->rows), kNormThreads, 0, (cudaStream_t)stream>>>(params(p));
    e = cudaGetLastError();
    return e == cudaSuccess ? RIKFAD_OK : report_cuda(e, "launch rikfad_norm_forward_kernel");
    RK_ENTRY_END
}

RIKFAD_API int rikfad_residual_norm_backward(const rikfad_residual_norm *p, void *stream)
{
    RK_ENTRY_BEGIN
    int device = -1;
    int rc = check_inputs(p, device);
    if (rc)
        return rc;
    const int64_t groups = p->gate.data ? p->rows / p->gate_rows : 0;
    const size_t pb = (size_t)dtype_bytes(p->param_dtype);
    if (!rc) rc = check_rows(p->du, "du", p->residual_dtype, p->rows, p->cols, device);
    if (!rc) rc = check_rows(p->dh, "dh", p->dtype, p->rows, p->cols, device);
    if (!rc) rc = check_rows(p->dx, "dx", p->residual_dtype, p->rows, p->cols, device);
    if (!rc) rc = check_rows(p->dz, "dz", p->dtype, p->rows, p->cols, device);
    if (!rc) rc = check_rows(p->dgate, "dgate", p->gate_dtype, groups, p->cols, device);
    if (!rc) rc = check_vector(p->dpost_weight, "dpost_weight", pb, device);
    if (!rc) rc = check_vector(p->dpost_bias, "dpost_bias", pb, device);
    if (!rc) rc = check_vector(p->dpre_weight, "dpre_weight", pb, device);
    if (!rc) rc = check_vector(p->dpre_bias, "dpre_bias", pb, device);
    if (!rc) rc = check_vector(p->workspace, "workspace", 16, device);
    if (rc)
        return rc;
    if (p->rows > 0 && ((p->dz.data && p->z.data == nullptr) || (p->dgate.data && p->gate.data == nullptr)))
        return bad("dz needs z and dgate needs gate");
    if ((p->post == RIKFAD_NORM_NONE && (p->dpost_weight || p->dpost_bias)) ||
        (p->pre == RIKFAD_NORM_NONE && (p->dpre_weight || p->dpre_bias)))
        return bad("gradients of weights and biases need their norm");
    if (p->rows > 0 && p->stats == nullptr)
        return bad("stats is NULL");
    if (p->workspace_bytes < rikfad_residual_norm_workspace(p) || (p->rows > 0 && p->workspace == nullptr))
        return bad("the workspace is smaller than rikfad_residual_norm_workspace");
    cudaError_t e = cudaPeekAtLastError();
    if (e != cudaSuccess)
        return report_cuda(e, "earlier CUDA error");
    const cudaStream_t s = (cudaStream_t)stream;
    const NormParams n = params(p);
    if (p->rows > 0)
        rikfad_norm_rows_kernel<<<row_blocks(p->rows), kNormThreads, 0, s>>>(n);
    const int64_t sums = 1 + (p->dgate.data && p->gate_rows != 1 ? groups : 0);
    const dim3 grid((unsigned)((p->cols + kNormThreads - 1) / kNormThreads), (unsigned)std::min<int64_t>(sums, 1024));
    rikfad_norm_columns_kernel<<<grid, kNormThreads, 0, s>>>(n);
    if (p->rows > 0)
        rikfad_norm_elements_kernel<<<row_blocks(p->rows), kNormThreads, 0, s>>>(n);
    e = cudaGetLastError();
    return e == cudaSuccess ? RIKFAD_OK : report_cuda(e, "launch of a residual norm's backward kernels");
    RK_ENTRY_END
}

}  // extern "C"
