// rikfad_clip.cu -- norms of a gradient list and clipping:
//   norm_t = ||g_t||_2,  total = sqrt(sum_t norm_t^2),
//   out_t = c g_t,  c = max_norm / total if max_norm < total < inf, else 1.
//
// The list is laid end to end and cut into equal shares, one per block, so that
// a list of a few large and many small tensors keeps every SM busy to the end; a
// share's part of one tensor is a segment.  The first kernel leaves one sum of
// squares per segment, the second joins them in segment order (in float64) into
// the norms and the factor c, the third scales.
#include <cuda_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <new>
#include <string>
#include <vector>

#include "rikfad.h"
#include "rikfad_host.hpp"
#include "rikfad_kernels.cuh"
#include "rikfad_types.cuh"

using namespace rikfad;

namespace {

constexpr int kClipThreads = 256;
constexpr int kClipWarps = kClipThreads / 32;
constexpr int kClipBlocksPerSm = 2048 / kClipThreads;
constexpr int64_t kMinShare = 8192;     // elements of the smallest share
constexpr int64_t kShareStep = 64;      // shares begin at multiples of this within a tensor
constexpr int kMaxTensors = 1024;       // of one launch

// Elements [begin, end) of tensor `tensor` (an index into the launch's pointers).
struct Segment {
    int64_t begin, end;
    int32_t tensor;
    int16_t grad_dtype, out_dtype;
};

// What the kernels of a call leave for one another.
struct ClipResult {
    float scale;
};

struct ClipParams {
    const Segment *segments;
    const int32_t *block_segment;   // first segment of every block of the list, and the end
    int32_t block0;                 // the launch's first block
    double *partial;                // one per segment
    ClipResult *result;
};

// The pointers of a launch's tensors travel in the kernel's parameters: no copy
// is enqueued, and a captured call keeps its own.
template <int CAP> struct ClipPointers {
    const void *grad[CAP];
    void *out[CAP];
};

// Sum of squares of the elements of a segment that this thread reads, times
// mul^2 (mul a power of two).
template <typename T> __device__ float segment_squares(const T *g, int64_t n, float mul)
{
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    int64_t done = 0;
    if (aligned16(g)) {
        const int64_t chunks = n / 8;
        for (int64_t i = threadIdx.x; i < chunks; i += kClipThreads) {
            float v[8];
            unpack8(load_raw8(g + i * 8), v);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] *= mul;
                acc[e & 3] = fmaf(v[e], v[e], acc[e & 3]);
            }
        }
        done = chunks * 8;
    }
    for (int64_t i = done + threadIdx.x; i < n; i += kClipThreads) {
        const float v = to_f32(g[i]) * mul;
        acc[0] = fmaf(v, v, acc[0]);
    }
    return (acc[0] + acc[1]) + (acc[2] + acc[3]);
}

__device__ float segment_squares(const void *grad, const Segment &s, float mul)
{
    const int64_t n = s.end - s.begin;
    if (s.grad_dtype == RIKFAD_F32)
        return segment_squares(static_cast<const float *>(grad) + s.begin, n, mul);
    if (s.grad_dtype == RIKFAD_BF16)
        return segment_squares(static_cast<const __nv_bfloat16 *>(grad) + s.begin, n, mul);
    return segment_squares(static_cast<const __half *>(grad) + s.begin, n, mul);
}

// The block's total of `v`, in every thread: fixed trees in float64.
__device__ double block_total(float v, double *red)
{
    double d = v;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        d += __shfl_xor_sync(0xffffffffu, d, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0)
        red[threadIdx.x >> 5] = d;
    __syncthreads();
    d = 0.0;
#pragma unroll
    for (int w = 0; w < kClipWarps; ++w)
        d += red[w];
    return d;
}

template <int CAP>
__global__ void __launch_bounds__(kClipThreads) rikfad_clip_squares_kernel(ClipParams a, const __grid_constant__ ClipPointers<CAP> ptrs)
{
    __shared__ double red[kClipWarps];
    const int block = a.block0 + blockIdx.x;
    for (int q = a.block_segment[block]; q < a.block_segment[block + 1]; ++q) {
        const Segment s = a.segments[q];
        const void *g = ptrs.grad[s.tensor];
        double sum = block_total(segment_squares(g, s, 1.f), red);
        // Squares that left float32's range (an infinite sum), or may have lost
        // much below it (1e-30 against a smallest square of 1e-45): once more,
        // with elements scaled by a power of two.  A true infinity stays one.
        if (sum > 1e38 || sum < 1e-30) {
            const bool big = sum > 1.0;
            const float mul = big ? 0x1p-80f : 0x1p100f;
            sum = block_total(segment_squares(g, s, mul), red) * (big ? 0x1p160 : 0x1p-200);
        }
        if (threadIdx.x == 0)
            a.partial[q] = sum;
    }
}

// Segment sums to tensor norms, their total and the factor, by one block.
__global__ void __launch_bounds__(kClipThreads) rikfad_clip_join_kernel(ClipParams a, const int32_t *tensor_segment, int ntensors,
                                                                        double max_norm, float *norms)
{
    __shared__ double red[kClipWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    double total = 0.0;             // of the warp's tensors, the same in its lanes
    for (int t = warp; t < ntensors; t += kClipWarps) {
        double d = 0.0;
        for (int q = tensor_segment[t] + lane; q < tensor_segment[t + 1]; q += 32)
            d += a.partial[q];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            d += __shfl_xor_sync(0xffffffffu, d, o);
        if (lane == 0)
            norms[t] = (float)sqrt(d);
        total += d;
    }
    if (lane == 0)
        red[warp] = total;
    __syncthreads();
    if (threadIdx.x == 0) {
        total = 0.0;
        for (int w = 0; w < kClipWarps; ++w)
            total += red[w];
        total = sqrt(total);
        norms[ntensors] = (float)total;
        a.result->scale = total > max_norm && total < (double)INFINITY ? (float)(max_norm / total) : 1.f;
    }
}

template <typename T, typename U> __device__ void scale_segment(const T *g, U *out, int64_t n, float c)
{
    int64_t done = 0;
    if (aligned16(g) && aligned16(out)) {
        const int64_t chunks = n / 8;
        for (int64_t i = threadIdx.x; i < chunks; i += kClipThreads) {
            float v[8];
            unpack8(load_raw8(g + i * 8), v);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e] *= c;
            store_raw8_cs(out + i * 8, pack8(v, U()));
        }
        done = chunks * 8;
    }
    for (int64_t i = done + threadIdx.x; i < n; i += kClipThreads)
        out[i] = from_f32<U>(to_f32(g[i]) * c);
}

template <typename T> __device__ void scale_segment(const T *g, void *out, const Segment &s, float c)
{
    const int64_t n = s.end - s.begin;
    if (s.out_dtype == RIKFAD_F32)
        scale_segment(g + s.begin, static_cast<float *>(out) + s.begin, n, c);
    else if (s.out_dtype == RIKFAD_BF16)
        scale_segment(g + s.begin, static_cast<__nv_bfloat16 *>(out) + s.begin, n, c);
    else
        scale_segment(g + s.begin, static_cast<__half *>(out) + s.begin, n, c);
}

template <int CAP>
__global__ void __launch_bounds__(kClipThreads) rikfad_clip_scale_kernel(ClipParams a, const __grid_constant__ ClipPointers<CAP> ptrs)
{
    const float c = a.result->scale;
    const int block = a.block0 + blockIdx.x;
    for (int q = a.block_segment[block]; q < a.block_segment[block + 1]; ++q) {
        const Segment s = a.segments[q];
        const void *g = ptrs.grad[s.tensor];
        void *out = ptrs.out[s.tensor];
        if (c == 1.f && g == out)
            continue;
        if (s.grad_dtype == RIKFAD_F32)
            scale_segment(static_cast<const float *>(g), out, s, c);
        else if (s.grad_dtype == RIKFAD_BF16)
            scale_segment(static_cast<const __nv_bfloat16 *>(g), out, s, c);
        else
            scale_segment(static_cast<const __half *>(g), out, s, c);
    }
}

// Tensors [tensor0, tensor1) and blocks [block0, block1) of one launch.
struct Part {
    int tensor0, tensor1, block0, block1;
};

}  // namespace

struct rikfad_clip_s {
    int device = 0;
    int ntensors = 0;
    std::vector<int64_t> numel;
    std::vector<int> grad_dtype, out_dtype;
    std::vector<Part> parts;
    std::vector<const void *> seen_grad;    // addresses that passed check_address
    std::vector<void *> seen_out;
    Segment *d_segments = nullptr;
    int32_t *d_block_segment = nullptr;
    int32_t *d_tensor_segment = nullptr;
    double *d_partial = nullptr;
    ClipResult *d_result = nullptr;
    size_t workspace = 0;
};

namespace {

void release(rikfad_clip c)
{
    for (void *p : {(void *)c->d_segments, (void *)c->d_block_segment, (void *)c->d_tensor_segment,
                    (void *)c->d_partial, (void *)c->d_result})
        counted_free(p);
    delete c;
}

template <typename T> int allocate(rikfad_clip c, T **dst, size_t count, const T *src)
{
    const size_t bytes = sizeof(T) * std::max<size_t>(count, 1);
    cudaError_t e = counted_malloc((void **)dst, bytes);
    if (e == cudaErrorMemoryAllocation)
        return report_error(RIKFAD_ERR_OOM, "cudaMalloc of a clipping plan failed: out of memory");
    if (e != cudaSuccess)
        return report_cuda(e, "cudaMalloc of a clipping plan");
    c->workspace += bytes;
    if (src && count && (e = cudaMemcpy(*dst, src, sizeof(T) * count, cudaMemcpyHostToDevice)) != cudaSuccess)
        return report_cuda(e, "cudaMemcpy of a clipping plan");
    return RIKFAD_OK;
}

// Cuts tensors [t0, t1) into at most `most` shares of equal size.
void plan_part(const rikfad_clip c, int t0, int t1, int64_t most, std::vector<Segment> &segments,
               std::vector<int32_t> &block_segment, std::vector<int32_t> &tensor_segment)
{
    double n = 0.0;
    for (int t = t0; t < t1; ++t)
        n += (double)c->numel[t];
    const double want = std::min((double)most, std::ceil(n / (double)kMinShare));
    const int64_t share = std::max<int64_t>(
        kShareStep, (int64_t)std::ceil(n / std::max(want, 1.0) / (double)kShareStep) * kShareStep);
    int64_t room = 0;       // left in the open share
    for (int t = t0; t < t1; ++t) {
        tensor_segment.push_back((int32_t)segments.size());
        for (int64_t at = 0; at < c->numel[t];) {
            if (room <= 0) {
                block_segment.push_back((int32_t)segments.size());
                room = share;
            }
            // a cut at a multiple of kShareStep, or the tensor's end
            const int64_t take = std::min(c->numel[t] - at, (room + kShareStep - 1) / kShareStep * kShareStep);
            segments.push_back({at, at + take, t - t0, (int16_t)c->grad_dtype[t], (int16_t)c->out_dtype[t]});
            at += take;
            room -= take;
        }
    }
}

int create(rikfad_clip c, const int64_t *numel, const int *grad_dtype, const int *out_dtype, int ntensors)
{
    cudaError_t e = cudaGetDevice(&c->device);
    int sms = 0;
    if (e == cudaSuccess)
        e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, c->device);
    if (e != cudaSuccess)
        return report_cuda(e, "rikfad_clip_create");
    c->ntensors = ntensors;
    c->numel.assign(numel, numel + ntensors);
    c->grad_dtype.assign(grad_dtype, grad_dtype + ntensors);
    c->out_dtype.assign(out_dtype ? out_dtype : grad_dtype, (out_dtype ? out_dtype : grad_dtype) + ntensors);
    c->seen_grad.assign(ntensors, nullptr);
    c->seen_out.assign(ntensors, nullptr);
    std::vector<Segment> segments;
    std::vector<int32_t> block_segment, tensor_segment;
    for (int t0 = 0; t0 < ntensors; t0 += kMaxTensors) {
        const int t1 = std::min(ntensors, t0 + kMaxTensors);
        const int b0 = (int)block_segment.size();
        plan_part(c, t0, t1, (int64_t)sms * kClipBlocksPerSm, segments, block_segment, tensor_segment);
        if ((int)block_segment.size() > b0)
            c->parts.push_back({t0, t1, b0, (int)block_segment.size()});
    }
    block_segment.push_back((int32_t)segments.size());
    tensor_segment.push_back((int32_t)segments.size());
    int rc = allocate(c, &c->d_segments, segments.size(), segments.data());
    if (!rc) rc = allocate(c, &c->d_block_segment, block_segment.size(), block_segment.data());
    if (!rc) rc = allocate(c, &c->d_tensor_segment, tensor_segment.size(), tensor_segment.data());
    if (!rc) rc = allocate<double>(c, &c->d_partial, segments.size(), nullptr);
    if (!rc) rc = allocate<ClipResult>(c, &c->d_result, 1, nullptr);
    return rc;
}

template <int CAP> int launch(rikfad_clip c, const Part &part, const ClipParams &a, const void *const *grad,
                              void *const *out, bool scale, cudaStream_t s)
{
    ClipPointers<CAP> ptrs = {};
    for (int t = part.tensor0; t < part.tensor1; ++t) {
        ptrs.grad[t - part.tensor0] = grad[t];
        ptrs.out[t - part.tensor0] = out ? out[t] : nullptr;
    }
    const dim3 blocks((unsigned)(part.block1 - part.block0));
    if (scale)
        rikfad_clip_scale_kernel<CAP><<<blocks, kClipThreads, 0, s>>>(a, ptrs);
    else
        rikfad_clip_squares_kernel<CAP><<<blocks, kClipThreads, 0, s>>>(a, ptrs);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? RIKFAD_OK : report_cuda(e, scale ? "launch rikfad_clip_scale_kernel" : "launch rikfad_clip_squares_kernel");
}

int launch_parts(rikfad_clip c, ClipParams a, const void *const *grad, void *const *out, bool scale, cudaStream_t s)
{
    for (const Part &part : c->parts) {
        a.block0 = part.block0;
        const int n = part.tensor1 - part.tensor0;
        const int rc = n <= 16    ? launch<16>(c, part, a, grad, out, scale, s)
                       : n <= 256 ? launch<256>(c, part, a, grad, out, scale, s)
                                  : launch<kMaxTensors>(c, part, a, grad, out, scale, s);
        if (rc)
            return rc;
    }
    return RIKFAD_OK;
}

int check_pointer(const void *p, int dtype, int device, const char *what, int t)
{
    if (p == nullptr)
        return report_error(RIKFAD_ERR_ARG, std::string(what) + " pointer of tensor " + std::to_string(t) + " is NULL");
    if ((uintptr_t)p % (uintptr_t)dtype_bytes(dtype))
        return report_error(RIKFAD_ERR_ALIGN, std::string(what) + " pointer of tensor " + std::to_string(t) +
                                                  " is not aligned to its element type");
    return check_address(p, device, what, t);
}

}  // namespace

extern "C" {

RIKFAD_API int rikfad_clip_create(const int64_t *numel, const int *grad_dtype, const int *out_dtype, int ntensors,
                                  rikfad_clip *out)
{
    RK_ENTRY_BEGIN
    if (out == nullptr)
        return report_error(RIKFAD_ERR_ARG, "out is NULL");
    *out = nullptr;
    if (ntensors < 0 || (ntensors > 0 && (numel == nullptr || grad_dtype == nullptr)))
        return report_error(RIKFAD_ERR_ARG, "need ntensors >= 0, numel and grad_dtype");
    for (int t = 0; t < ntensors; ++t) {
        if (numel[t] < 0 || numel[t] > (int64_t)1 << 48)
            return report_error(RIKFAD_ERR_ARG, "numel of tensor " + std::to_string(t) + " is out of range");
        if (!dtype_ok(grad_dtype[t]) || (out_dtype && !dtype_ok(out_dtype[t])))
            return report_error(RIKFAD_ERR_ARG, "dtype of tensor " + std::to_string(t) + " is not a rikfad_dtype");
    }
    rikfad_clip c = new rikfad_clip_s();
    int rc = RIKFAD_ERR_OOM;
    try {
        rc = create(c, numel, grad_dtype, out_dtype, ntensors);
    } catch (...) {
        release(c);
        throw;
    }
    if (rc) {
        release(c);
        return rc;
    }
    *out = c;
    return RIKFAD_OK;
    RK_ENTRY_END
}

RIKFAD_API void rikfad_clip_destroy(rikfad_clip c)
{
    if (c == nullptr)
        return;
    int cur = -1;
    cudaGetDevice(&cur);
    if (cur != c->device)
        cudaSetDevice(c->device);
    const int dev = c->device;
    cudaDeviceSynchronize();
    release(c);
    if (cur >= 0 && cur != dev)
        cudaSetDevice(cur);
}

RIKFAD_API size_t rikfad_clip_workspace_bytes(rikfad_clip c) { return c ? c->workspace : 0; }

RIKFAD_API int rikfad_clip_run(rikfad_clip c, const void *const *grad, void *const *out, double max_norm, float *norms,
                               void *stream)
{
    RK_ENTRY_BEGIN
    if (c == nullptr)
        return report_error(RIKFAD_ERR_ARG, "handle is NULL");
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess)
        return report_cuda(e, "cudaGetDevice");
    if (dev != c->device)
        return report_error(RIKFAD_ERR_STATE, "current CUDA device differs from the handle's device");
    if (c->ntensors > 0 && grad == nullptr)
        return report_error(RIKFAD_ERR_ARG, "grad is NULL");
    if (norms == nullptr)
        return report_error(RIKFAD_ERR_ARG, "norms is NULL");
    if ((uintptr_t)norms % sizeof(float))
        return report_error(RIKFAD_ERR_ALIGN, "norms is not aligned");
    if (out && !(max_norm >= 0))
        return report_error(RIKFAD_ERR_ARG, "max_norm must be >= 0");
    int rc = check_address(norms, dev, "norms");
    for (int t = 0; !rc && t < c->ntensors; ++t) {
        if (c->numel[t] == 0)
            continue;
        if (grad[t] == nullptr || grad[t] != c->seen_grad[t]) {
            rc = check_pointer(grad[t], c->grad_dtype[t], dev, "gradient", t);
            c->seen_grad[t] = rc ? nullptr : grad[t];
        }
        if (!rc && out && (out[t] == nullptr || out[t] != c->seen_out[t])) {
            rc = check_pointer(out[t], c->out_dtype[t], dev, "output", t);
            c->seen_out[t] = rc ? nullptr : out[t];
        }
        if (!rc && out && out[t] == grad[t] && c->grad_dtype[t] != c->out_dtype[t])
            rc = report_error(RIKFAD_ERR_ARG, "tensor " + std::to_string(t) + " cannot be clipped in place to another type");
    }
    if (rc)
        return rc;
    if ((e = cudaPeekAtLastError()) != cudaSuccess)
        return report_cuda(e, "earlier CUDA error");
    const cudaStream_t s = (cudaStream_t)stream;
    ClipParams a{};
    a.segments = c->d_segments;
    a.block_segment = c->d_block_segment;
    a.partial = c->d_partial;
    a.result = c->d_result;
    if ((rc = launch_parts(c, a, grad, out, false, s)))
        return rc;
    rikfad_clip_join_kernel<<<1, kClipThreads, 0, s>>>(a, c->d_tensor_segment, c->ntensors, max_norm, norms);
    if ((e = cudaGetLastError()) != cudaSuccess)
        return report_cuda(e, "launch rikfad_clip_join_kernel");
    return out ? launch_parts(c, a, grad, out, true, s) : RIKFAD_OK;
    RK_ENTRY_END
}

}  // extern "C"
