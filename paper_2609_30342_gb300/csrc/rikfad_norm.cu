// rikfad_norm.cu -- residual sum of a transformer block with the norms around it:
// argument checks, workspace and launch shapes.  The mathematics and the kernels
// are in rikfad_norm_kernels.cuh, instantiated per direction and element types in
// rikfad_norm_forward_*.cu and rikfad_norm_backward_*.cu.
#include <cuda_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <new>
#include <string>

#include "rikfad.h"
#include "rikfad_host.hpp"
#include "rikfad_norm.hpp"

using namespace rikfad;

namespace {

int bad(const std::string &msg) { return report_error(RIKFAD_ERR_ARG, msg); }

int check_sizes(const rikfad_residual_norm *p)
{
    if (p == nullptr)
        return bad("p is NULL");
    if (p->rows < 0 || p->rows > (int64_t)1 << 34)
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

bool wide(const rikfad_rows &r, int dtype, int64_t rows)
{
    return (uintptr_t)r.data % 16 == 0 && (rows <= 1 || r.stride * dtype_bytes(dtype) % 16 == 0);
}

NormParams params(const rikfad_residual_norm *p, bool backward)
{
    NormParams n{};
    n.rows = p->rows;
    n.cols = (int32_t)p->cols;
    n.inv_cols = 1.f / (float)p->cols;
    n.a = (float)p->residual_scale;
    n.b = (float)p->branch_scale;
    n.post_eps = (float)p->post_eps;
    n.pre_eps = (float)p->pre_eps;
    n.gate_rows = p->gate.data ? p->gate_rows : 1;
    n.post_weight = p->post_weight;
    n.post_bias = p->post_bias;
    n.pre_weight = p->pre_weight;
    n.pre_bias = p->pre_bias;
    n.stats = reinterpret_cast<float4 *>(p->stats);
    const int64_t gates = p->rows / std::max<int64_t>(n.gate_rows, 1);
    auto flag = [&](bool on, uint32_t bit) { n.flags |= on ? bit : 0; };
    auto tensor = [&](NormRows &to, const rikfad_rows &r, int dtype, int64_t rows, uint32_t on, uint32_t wide_bit) {
        to = {r.data, r.data ? r.stride : 0, 0};
        flag(r.data != nullptr, on);
        // absent tensors do not matter
        n.wide |= r.data == nullptr || wide(r, dtype, rows) ? wide_bit : 0;
    };
    tensor(n.x, p->x, p->residual_dtype, p->rows, 0, kNormWideX);
    tensor(n.z, p->z, p->dtype, p->rows, kNormBranch, kNormWideZ);
    tensor(n.gate, p->gate, p->gate_dtype, gates, kNormGated, kNormWideGate);
    flag(p->gate_dtype == RIKFAD_F32, kNormGateF32);
    flag(p->gate.data && p->gate_rows > 1, kNormSharedGate);
    flag(p->param_dtype == RIKFAD_F32, kNormParamF32);
    flag(p->z.data && p->post != RIKFAD_NORM_NONE, kNormPost);
    flag(p->post == RIKFAD_NORM_LAYER, kNormPostLayer);
    flag(p->pre != RIKFAD_NORM_NONE, kNormPre);
    flag(p->pre == RIKFAD_NORM_LAYER, kNormPreLayer);
    const void *const vectors[4] = {p->post_weight, p->post_bias, p->pre_weight, p->pre_bias};
    const uint32_t bits[4] = {kNormPostWeight, kNormPostBias, kNormPreWeight, kNormPreBias};
    for (int i = 0; i < 4; ++i)
        flag(vectors[i] != nullptr, bits[i]);
    n.general = p->post_bias || p->pre_bias || p->post == RIKFAD_NORM_LAYER || p->pre == RIKFAD_NORM_LAYER;
    if (!backward) {
        tensor(n.u, p->u, p->residual_dtype, p->rows, kNormU, kNormWideU);
        tensor(n.h, p->h, p->dtype, p->rows, kNormH, kNormWideH);
        flag(p->stats != nullptr, kNormStats);
        n.wide |= kNormWideDu | kNormWideDh | kNormWideDx | kNormWideDz | kNormWideDgate;
        return n;
    }
    n.wide |= kNormWideU | kNormWideH;
    tensor(n.du, p->du, p->residual_dtype, p->rows, kNormDu, kNormWideDu);
    tensor(n.dh, p->dh, p->dtype, p->rows, kNormDh, kNormWideDh);
    // An absent gradient's copies of no bytes start where x's do, and on 16 bytes they
    // have to start as well.
    if (!(n.wide & kNormWideX))
        n.wide &= ~((p->du.data ? 0 : kNormWideDu) | (p->dh.data ? 0 : kNormWideDh));
    tensor(n.dx, p->dx, p->residual_dtype, p->rows, kNormDx, kNormWideDx);
    tensor(n.dz, p->dz, p->dtype, p->rows, kNormDz, kNormWideDz);
    tensor(n.dgate, p->dgate, p->gate_dtype, gates, kNormDgate, kNormWideDgate);
    n.dpost_weight = p->dpost_weight;
    n.dpost_bias = p->dpost_bias;
    n.dpre_weight = p->dpre_weight;
    n.dpre_bias = p->dpre_bias;
    flag(p->dpre_weight, kNormDpreWeight);
    flag(p->dpost_weight, kNormDpostWeight);
    flag(p->dpre_bias, kNormDpreBias);
    flag(p->dpost_bias, kNormDpostBias);
    n.general = n.general || p->dpre_bias || p->dpost_bias;
    return n;
}

// Threads of a row that has `vectors` vectors, `v` of them a thread's.
int row_threads(int vectors, int v)
{
    const int threads = (vectors + v - 1) / v;
    int lanes = 1;
    while (lanes < 32 && lanes < threads)
        lanes *= 2;
    return threads <= 32 ? lanes : (threads + 31) / 32 * 32;
}

// Rows of odd widths: if every tensor's rows drift by the same number of elements
// from 16 bytes, from an aligned start, rows that drift equally far make a class
// with aligned vectors.  0: there is no such drift, each tensor's own rows decide.
int drift_of(const NormParams &n)
{
    if (n.wide == kNormWideAll || n.rows <= 1)
        return 0;
    const NormRows *const all[] = {&n.x, &n.z, &n.u, &n.h, &n.du, &n.dh, &n.dx, &n.dz,
                                   n.gate_rows > 1 ? nullptr : &n.gate, n.gate_rows > 1 ? nullptr : &n.dgate};
    int drift = -1;
    for (const NormRows *t : all) {
        if (t == nullptr || t->data == nullptr)
            continue;
        if ((uintptr_t)t->data % 16 || (drift >= 0 && t->stride % 8 != drift))
            return 0;
        drift = (int)(t->stride % 8);
    }
    return std::max(drift, 0);
}

void set_drift(NormParams &n, int drift)
{
    n.drift = drift;
    n.classes = drift == 0 ? 1 : drift % 4 == 0 ? 2 : drift % 2 == 0 ? 4 : 8;
    if (drift == 0)
        return;
    n.wide = kNormWideAll;
    if (n.gate_rows > 1)            // their rows are others than the rest's
        n.wide &= ~(kNormWideGate | kNormWideDgate);
}

// Vectors of a thread, threads of a row, columns of a block and blocks of a
// cluster, from the width; how far a thread's rows are apart.  A block has at most
// `most_threads` threads of `most_vectors` vectors each.
void shape(NormParams &n, const rikfad_residual_norm *p, int most_vectors, int most_threads, int drift)
{
    // A shifted row may need a vector more.  Where a cluster has no room for it (rows of
    // more than 32761 columns), every tensor's own rows decide.
    if ((n.cols + 7 + 7) / 8 > kNormMaxCluster * most_threads * most_vectors)
        drift = 0;
    set_drift(n, drift);
    const int vectors = (n.cols + (n.classes > 1 ? 7 : 0) + 7) / 8;     // a shifted row may begin within one
    n.cluster = 1;
    while ((vectors + n.cluster - 1) / n.cluster > most_threads * most_vectors)
        n.cluster *= 2;
    const int here = (vectors + n.cluster - 1) / n.cluster;
    n.cta_cols = here * 8;
    // A row's fixed work costs a thread about as much as one vector does (forward, with
    // two vectors instead of one: 32768 x 4096 205 us, 257; 8192 x 1600 25, 28).
    int best = 0;
    for (int v = 1; v <= most_vectors; ++v) {
        const int threads = n.cluster > 1 ? (row_threads(here, v) + 31) / 32 * 32 : row_threads(here, v);
        if (threads <= most_threads && (best == 0 || threads * (v + 1) < best)) {
            best = threads * (v + 1);
            n.vectors = v;
            n.lanes = threads;
        }
    }
    n.threads = n.lanes <= 32 && n.cluster == 1 ? 128 : n.lanes;
    n.row_groups = n.threads / n.lanes;
    n.full = n.cols % 8 == 0 && n.wide == kNormWideAll && n.classes == 1;
    // `row_groups` rows of a class, or neighbours where rows share gates
    const int64_t rows = n.classes * (int64_t)(n.gate_rows > 1 ? 1 : n.row_groups);
    const int64_t a = rows * dtype_bytes(p->dtype), r = rows * dtype_bytes(p->residual_dtype);
    const int64_t g = rows * dtype_bytes(p->gate_dtype);
    for (NormRows *t : {&n.z, &n.h, &n.dh, &n.dz})
        t->step = t->stride * a;
    for (NormRows *t : {&n.x, &n.u, &n.du, &n.dx})
        t->step = t->stride * r;
    // the rows of a shared gate are counted, so a step there is one gate
    for (NormRows *t : {&n.gate, &n.dgate})
        t->step = n.gate_rows > 1 ? t->stride * dtype_bytes(p->gate_dtype) : t->stride * g;
    n.flags |= p->gate.data && n.gate_rows >= kNormHeldRows ? kNormGateHeld : 0;
}

// Clusters of a launch: as many as are resident at once (`threads_per_sm` by the
// kernel's register bound, and by the shared memory of their stages), no more than
// there are rows.
void grid(NormParams &n, int threads_per_sm)
{
    n.threads_per_sm = threads_per_sm;
    const int by_registers = std::max(1, threads_per_sm / n.threads);
    const int64_t groups = (n.rows + n.row_groups - 1) / n.row_groups;
    const size_t stage = (size_t)n.threads * 16 * n.units * n.vectors;
    n.smem = 2 * stage;
    const int resident = std::max(1, std::min(by_registers, (int)(kNormSmemPerSm / n.smem)));
    n.ctas = (int)std::max<int64_t>(1, std::min<int64_t>(groups, (int64_t)kNormSms * resident / n.cluster));
    n.ctas = (n.ctas + n.classes - 1) / n.classes * n.classes;      // as many for each class
}

void forward_shape(const rikfad_residual_norm *p, NormParams &n)
{
    const int a = p->dtype == RIKFAD_F32 ? 2 : 1, r = p->residual_dtype == RIKFAD_F32 ? 2 : 1;
    n.units = r + a + (p->gate.data && p->gate_rows < kNormHeldRows ? (p->gate_dtype == RIKFAD_F32 ? 2 : a) : 0);
    const int most = n.flags & kNormSharedGate ? 1 : 2;
    shape(n, p, most, kNormMaxThreads / most, drift_of(n));
    const bool heavy = (n.flags & kNormPost) && n.general;
    grid(n, n.vectors == 1                         ? (heavy ? kNormHeavyForwardThreads1 : kNormForwardThreads1)
            : heavy && p->cols <= kNormHeavyCols ? kNormHeavyThreads
                                                 : kNormForwardThreads2);
}

struct Workspace {
    int64_t weights = 0, gates = 0;     // floats
};

// Partial sums: one row of each kind for every cluster, and two of the gate's for
// every group whose rows share gates with others.
Workspace backward_shape(const rikfad_residual_norm *p, NormParams &n, int drift)
{
    const int a = p->dtype == RIKFAD_F32 ? 2 : 1, r = p->residual_dtype == RIKFAD_F32 ? 2 : 1;
    n.units = 2 * a + 2 * r + (p->gate.data && p->gate_rows < kNormHeldRows ? (p->gate_dtype == RIKFAD_F32 ? 2 : a) : 0);
    const bool shared = (n.flags & kNormSharedGate) && p->dgate.data, heavy = (n.flags & kNormPost) && n.general;
    const int threads = heavy && p->cols <= kNormHeavyCols ? kNormHeavyThreads : kNormBackwardThreads;
    shape(n, p, 1, threads, drift);
    grid(n, threads);
    n.sums = 0;
    for (const void *v : {p->dpre_weight, p->dpost_weight, p->dpre_bias, p->dpost_bias})
        n.sums += v != nullptr;
    // A group leaves partial sums of two gates at most; where its rows of a class reach
    // over more, every tensor's own rows decide.
    if (shared && n.classes > 1) {
        const int64_t workers = (int64_t)(n.ctas / n.classes) * n.row_groups;
        const int64_t rows = (p->rows + n.classes - 1) / n.classes;
        if ((rows + workers - 1) / workers * n.classes > p->gate_rows) {
            NormParams again = params(p, true);
            return backward_shape(p, n = again, 0);
        }
    }
    Workspace w;
    w.weights = (int64_t)n.sums * n.ctas * n.cols;
    w.gates = shared ? (int64_t)2 * n.ctas * n.row_groups * n.cols : 0;
    return w;
}

using Launch = cudaError_t (*)(const NormParams &, cudaStream_t);

cudaError_t launch_norm(const NormParams &n, int dtype, int residual_dtype, bool backward, cudaStream_t s)
{
    // by dtype, residual_dtype == RIKFAD_F32 and direction
    static const Launch table[3][2][2] = {
        {{norm_forward_f32_f32, norm_backward_f32_f32}, {norm_forward_f32_f32, norm_backward_f32_f32}},
        {{norm_forward_bf16_bf16, norm_backward_bf16_bf16}, {norm_forward_bf16_f32, norm_backward_bf16_f32}},
        {{norm_forward_f16_f16, norm_backward_f16_f16}, {norm_forward_f16_f32, norm_backward_f16_f32}},
    };
    return table[dtype][residual_dtype == RIKFAD_F32][backward](n, s);
}

}  // namespace

extern "C" {

RIKFAD_API size_t rikfad_residual_norm_workspace(const rikfad_residual_norm *p)
{
    RK_ENTRY_BEGIN
    if (check_sizes(p))
        return 0;
    report_error(RIKFAD_OK, "");
    if (p->rows == 0)
        return 0;
    // enough for rows that start anywhere
    int64_t floats = 0;
    for (const int drift : {0, 1, 2, 4}) {
        NormParams n = params(p, true);
        const Workspace w = backward_shape(p, n, drift);
        floats = std::max(floats, w.weights + w.gates);
    }
    return (size_t)floats * sizeof(float);
    }
    catch (...)
    {
        return 0;
    }
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
    NormParams n = params(p, false);
    forward_shape(p, n);
    e = launch_norm(n, p->dtype, p->residual_dtype, false, (cudaStream_t)stream);
    return e == cudaSuccess ? RIKFAD_OK : report_cuda(e, "launch of a residual norm's forward kernel");
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
    NormParams n = params(p, true);
    const Workspace w = p->rows > 0 ? backward_shape(p, n, drift_of(n)) : Workspace();
    const int64_t floats = w.weights + w.gates;
    if (p->workspace_bytes / sizeof(float) < (size_t)floats || (floats > 0 && p->workspace == nullptr))
        return bad("the workspace is smaller than rikfad_residual_norm_workspace");
    cudaError_t e = cudaPeekAtLastError();
    if (e != cudaSuccess)
        return report_cuda(e, "earlier CUDA error");
    const cudaStream_t s = (cudaStream_t)stream;
    if (p->rows == 0) {
        for (void *v : {p->dpre_weight, p->dpost_weight, p->dpre_bias, p->dpost_bias})
            if (v && (e = cudaMemsetAsync(v, 0, pb * (size_t)p->cols, s)) != cudaSuccess)
                return report_cuda(e, "cudaMemsetAsync");
        return RIKFAD_OK;
    }
    n.sum_part = static_cast<float *>(p->workspace);
    n.gate_part = n.sum_part + w.weights;
    e = launch_norm(n, p->dtype, p->residual_dtype, true, s);
    return e == cudaSuccess ? RIKFAD_OK : report_cuda(e, "launch of a residual norm's backward kernels");
    RK_ENTRY_END
}

}  // extern "C"
