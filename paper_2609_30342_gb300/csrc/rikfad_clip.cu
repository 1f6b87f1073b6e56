// rikfad_clip.cu -- norms of a gradient list and clipping:
//   norm_t = ||g_t||_2,  total = sqrt(sum_t norm_t^2),
//   out_t = c g_t,  c = max_norm / total if max_norm < total < inf, else 1.
//
// The list is laid end to end and cut into equal shares, one per resident block,
// so that a list of a few large and many small tensors keeps every SM busy to the
// end; a share's part of one tensor is a segment.  The first kernel leaves one
// sum of squares per segment.  The block that finishes a tensor's last segment adds
// them up in order (float64), the block that finishes last adds the tensors and
// forms c: one block joining everything would read its sums for tens of
// microseconds after the others.  The second kernel scales.  It walks
// every share from its end, so that what the first one read last is read from the
// L2 cache.
//
// Memory bounds both: every gradient is read twice (the factor is known only when
// all of them have been read once) and written once.  124.4M float32 gradients to
// bfloat16 in 196 tensors take 198 us (1.24 GB, 6.3 TB/s), 1557.6M of bfloat16 in
// 772 tensors 1500 us (9.3 GB, 6.2 TB/s), 30.1M of bfloat16 36 us (the second read
// from L2); 131584 of float32 10 us on the device, the chain from the first load over
// two rounds of counters to the last store, and 13 on the host.
#include <cuda_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstring>
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
constexpr int kClipBlocksPerSm = 6;
// 8-element loads in flight per thread: 64 bytes.
template <typename T> constexpr int kClipUnroll = sizeof(T) == 4 ? 2 : 4;
constexpr int64_t kMinShare = 8192;     // elements of the smallest share
constexpr int64_t kShareStep = 64;      // shares begin at multiples of this within a tensor
constexpr int64_t kMaxShare = 1 << 30;  // elements of the largest share (lists far beyond any memory are refused)
constexpr int kShortSegment = 2048;     // elements of a segment that one warp reads
constexpr int kMaxTensors = 1024;       // of one launch

// Elements [begin, end) of tensor `tensor` (an index into the launch's pointers).
struct Segment {
    int64_t begin, end;
    int32_t tensor;
    int16_t grad_dtype, out_dtype;
    int32_t list_tensor;            // index in the list
    int32_t first, count;           // the tensor's segments
    int32_t unused;                 // to 48 bytes
};

// What the kernels of a call leave for one another.  The factor is shift times scale:
// shift is 1, or for factors near the end of float32's range a power of two that keeps
// scale's 24 bits (an element below 2^-62, whose product with it loses bits, is below
// the range once scaled).
struct ClipResult {
    float scale, shift;
    unsigned int blocks_done;       // of this call; the last block leaves 0
};

struct ClipParams {
    const Segment *segments;
    const int32_t *block_segment;   // first segment of every block of the list, and the end
    int32_t block0;                 // the launch's first block
    double *partial;                // one per segment
    double *tensor_sum;             // one per tensor of the list (empty ones stay 0)
    unsigned int *tensor_done;      // its finished segments of this call; left at 0
    ClipResult *result;
    int32_t ntensors, total_blocks; // of the list
    double max_norm;
    float *norms, *total;
};

// The pointers of a launch's tensors travel in the kernel's parameters: no copy
// is enqueued, and a captured call keeps its own.
template <int CAP> struct ClipPointers {
    const void *grad[CAP];
    void *out[CAP];
};

template <typename T> __device__ __forceinline__ void add_squares(const Raw8<T> &r, float mul, float (&acc)[4])
{
    float v[8];
    unpack8(r, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        v[e] *= mul;
        acc[e & 3] = fmaf(v[e], v[e], acc[e & 3]);
    }
}

// Sum of squares of the elements of a segment that this thread reads, times
// mul^2 (mul a power of two).  The first sums take at most 64 squares before they
// move to the second: an error of a few units of 2^-24 whatever the share's
// length.  Float64 sums would do without, but float64 additions are issued at a
// 64th of the float32 rate: with them in every thread and in the block's tree the
// kernel took 37 us instead of 14 for 60 MB of bfloat16 gradients.
template <typename T> __device__ float segment_squares(const T *g, int n, float mul, int thread, int threads)
{
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    float total = 0.f;
    int done = 0, k = 0;
    if (aligned16(g)) {
        const int chunks = n / 8;
        for (int i = thread; i < chunks; i += kClipUnroll<T> * threads) {
            Raw8<T> r[kClipUnroll<T>] = {};        // a last, partial round is one round trip as well
#pragma unroll
            for (int j = 0; j < kClipUnroll<T>; ++j)
                if (i + j * threads < chunks)
                    r[j] = load_raw8(g + (int64_t)(i + j * threads) * 8);
#pragma unroll
            for (int j = 0; j < kClipUnroll<T>; ++j)
                add_squares(r[j], mul, acc);
            if (++k * kClipUnroll<T> == 32) {
                k = 0;
                total += (acc[0] + acc[1]) + (acc[2] + acc[3]);
                acc[0] = acc[1] = acc[2] = acc[3] = 0.f;
            }
        }
        done = chunks * 8;
        k = 0;
    }
    for (int i = done + thread; i < n; i += threads) {
        const float v = to_f32(g[i]) * mul;
        acc[k & 3] = fmaf(v, v, acc[k & 3]);
        if (++k == 256) {
            k = 0;
            total += (acc[0] + acc[1]) + (acc[2] + acc[3]);
            acc[0] = acc[1] = acc[2] = acc[3] = 0.f;
        }
    }
    return total + ((acc[0] + acc[1]) + (acc[2] + acc[3]));
}

__device__ float segment_squares(const void *grad, const Segment &s, float mul, int thread, int threads)
{
    const int n = (int)(s.end - s.begin);
    if (s.grad_dtype == RIKFAD_F32)
        return segment_squares(static_cast<const float *>(grad) + s.begin, n, mul, thread, threads);
    if (s.grad_dtype == RIKFAD_BF16)
        return segment_squares(static_cast<const __nv_bfloat16 *>(grad) + s.begin, n, mul, thread, threads);
    return segment_squares(static_cast<const __half *>(grad) + s.begin, n, mul, thread, threads);
}

// The sums of a block's segments [q0, q0 + n), n <= 32: lane i of warp 0 stores
// segment q0 + i and, if it is its tensor's last, adds up the tensor.  The order
// of the additions is the segments', whichever block makes them.
__device__ void finish_segments(const ClipParams &a, const Segment *segments, int q0, int n, double sum)
{
    const int lane = threadIdx.x;
    const bool mine = lane < n;
    const int count = mine ? segments[lane].count : 0, tensor = mine ? segments[lane].list_tensor : 0;
    bool last = count == 1;
    if (count > 1) {
        a.partial[q0 + lane] = sum;
        __threadfence();
        last = atomicInc(a.tensor_done + tensor, (unsigned)count - 1) == (unsigned)count - 1;
        __threadfence();
    }
    for (unsigned todo = __ballot_sync(0xffffffffu, last && count > 1); todo; todo &= todo - 1) {
        const int i = __ffs(todo) - 1;
        const int first = segments[i].first, parts = segments[i].count;
        double d = 0.0;
#pragma unroll 4
        for (int k = lane; k < parts; k += 32)
            d += __ldcg(a.partial + first + k);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            d += __shfl_xor_sync(0xffffffffu, d, o);
        if (lane == i)
            sum = d;
    }
    if (last) {
        a.tensor_sum[tensor] = sum;
        a.norms[tensor] = (float)sqrt(sum);
    }
}

// The total and the factor, by the first warp of the block that finishes last.
__device__ void finish_list(const ClipParams &a)
{
    const int lane = threadIdx.x;
    double total = 0.0;
#pragma unroll 8
    for (int t = lane; t < a.ntensors; t += 32)
        total += __ldcg(a.tensor_sum + t);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        total += __shfl_xor_sync(0xffffffffu, total, o);
    if (lane == 0) {
        total = sqrt(total);
        *a.total = (float)total;
        const double c = total > a.max_norm && total < (double)INFINITY ? a.max_norm / total : 1.0;
        const bool low = c < 0x1p-100;
        a.result->scale = (float)(low ? c * 0x1p64 : c);
        a.result->shift = low ? 0x1p-64f : 1.f;
    }
}

// A block walks its segments without a barrier, so that the loads of the next one
// follow at once; every warp leaves its sum of every segment in shared memory, and
// warp 0 joins up to 32 segments at a time.  Short segments (vectors between a
// list's matrices) are one warp's each, all of them under way together: as the
// block's work, one after the other, each costs a round trip to memory.
template <int CAP>
__global__ void __launch_bounds__(kClipThreads, kClipBlocksPerSm)
    rikfad_clip_squares_kernel(const __grid_constant__ ClipParams a, const __grid_constant__ ClipPointers<CAP> ptrs)
{
    __shared__ Segment segments[32];
    __shared__ float red[kClipWarps][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int block = a.block0 + blockIdx.x;
    wait_for_predecessor();
    const int end = a.block_segment[block + 1];
    for (int q0 = a.block_segment[block]; q0 < end; q0 += 32) {
        const int n = min(32, end - q0);
        __syncthreads();
        if (threadIdx.x < n)
            segments[threadIdx.x] = a.segments[q0 + threadIdx.x];
        __syncthreads();
        for (int pass = 0; pass < 2; ++pass)
            for (int i = 0; i < n; ++i) {
                const bool brief = segments[i].end - segments[i].begin <= kShortSegment;
                if (brief != (pass == 0))
                    continue;
                float sum = 0.f;
                if (!brief)
                    sum = warp_sum(segment_squares(ptrs.grad[segments[i].tensor], segments[i], 1.f, threadIdx.x, kClipThreads));
                else if (i % kClipWarps == warp)
                    sum = warp_sum(segment_squares(ptrs.grad[segments[i].tensor], segments[i], 1.f, lane, 32));
                if (lane == 0)
                    red[warp][i] = sum;
            }
        __syncthreads();
        // Squares that left float32's range (an infinite sum), or may have lost
        // much below it (1e-30 against a smallest square of 1e-45): once more, with
        // elements scaled by a power of two.  A true infinity stays one.  Every
        // warp comes to the same verdicts.
        float total = 0.f;
#pragma unroll
        for (int w = 0; w < kClipWarps; ++w)
            total += lane < n ? red[w][lane] : 1.f;
        double sum = total;
        const bool big = total > 1e38f;
        for (unsigned redo = __ballot_sync(0xffffffffu, big || total < 1e-30f); redo; redo &= redo - 1) {
            const int i = __ffs(redo) - 1;
            const bool down = __shfl_sync(0xffffffffu, big, i);
            const float part = warp_sum(segment_squares(ptrs.grad[segments[i].tensor], segments[i], down ? 0x1p-80f : 0x1p100f,
                                                        threadIdx.x, kClipThreads));
            __syncthreads();
            if (lane == 0)
                red[warp][32] = part;
            __syncthreads();
            if (lane == i) {
                total = 0.f;
#pragma unroll
                for (int w = 0; w < kClipWarps; ++w)
                    total += red[w][32];
                sum = total * (down ? 0x1p160 : 0x1p-200);
            }
        }
        if (warp == 0)
            finish_segments(a, segments, q0, n, sum);
    }
    allow_successor_launch();
    if (warp == 0) {
        bool last = false;
        __syncwarp();               // the lanes' stores before lane 0's fence
        if (lane == 0) {
            __threadfence();
            last = atomicInc(&a.result->blocks_done, (unsigned)a.total_blocks - 1) == (unsigned)a.total_blocks - 1;
            __threadfence();
        }
        if (__shfl_sync(0xffffffffu, last, 0))
            finish_list(a);
    }
}

struct Factor {
    float scale, shift;
    __device__ __forceinline__ float operator()(float v) const { return v * shift * scale; }
};

template <typename T, typename U> __device__ __forceinline__ void scale8(const Raw8<T> &r, U *out, const Factor &c)
{
    float v[8];
    unpack8(r, v);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        v[e] = c(v[e]);
    store_raw8_cs(out, pack8(v, U()));
}

// out = c g over a segment, from its end.  The loads and stores are streaming: nothing
// is read again.
template <typename T, typename U> __device__ void scale_segment(const T *g, U *out, int n, const Factor &c)
{
    const bool wide = aligned16(g) && aligned16(out);
    const int chunks = wide ? n / 8 : 0;
    for (int i = n - 1 - (int)threadIdx.x; i >= chunks * 8; i -= kClipThreads)
        out[i] = from_f32<U>(c(to_f32(g[i])));
    g += (int64_t)(chunks - 1 - (int)threadIdx.x) * 8;
    out += (int64_t)(chunks - 1 - (int)threadIdx.x) * 8;
    int left = chunks - (int)threadIdx.x;
    for (; left > (kClipUnroll<T> - 1) * kClipThreads; left -= kClipUnroll<T> * kClipThreads) {
        Raw8<T> r[kClipUnroll<T>];
#pragma unroll
        for (int j = 0; j < kClipUnroll<T>; ++j)
            r[j] = load_raw8_cs(g - j * kClipThreads * 8);
#pragma unroll
        for (int j = 0; j < kClipUnroll<T>; ++j)
            scale8(r[j], out - j * kClipThreads * 8, c);
        g -= kClipUnroll<T> * kClipThreads * 8;
        out -= kClipUnroll<T> * kClipThreads * 8;
    }
    for (; left > 0; left -= kClipThreads) {
        scale8(load_raw8_cs(g), out, c);
        g -= kClipThreads * 8;
        out -= kClipThreads * 8;
    }
}

template <typename T> __device__ void scale_segment(const T *g, void *out, const Segment &s, const Factor &c)
{
    const int n = (int)(s.end - s.begin);
    if (s.out_dtype == RIKFAD_F32)
        scale_segment(g + s.begin, static_cast<float *>(out) + s.begin, n, c);
    else if (s.out_dtype == RIKFAD_BF16)
        scale_segment(g + s.begin, static_cast<__nv_bfloat16 *>(out) + s.begin, n, c);
    else
        scale_segment(g + s.begin, static_cast<__half *>(out) + s.begin, n, c);
}

template <int CAP>
__global__ void __launch_bounds__(kClipThreads, kClipBlocksPerSm)
    rikfad_clip_scale_kernel(const __grid_constant__ ClipParams a, const __grid_constant__ ClipPointers<CAP> ptrs)
{
    wait_for_predecessor();
    const Factor c{a.result->scale, a.result->shift};
    const int block = a.block0 + blockIdx.x;
    for (int q = a.block_segment[block + 1] - 1; q >= a.block_segment[block]; --q) {
        const Segment s = a.segments[q];
        const void *g = ptrs.grad[s.tensor];
        void *out = ptrs.out[s.tensor];
        if (c.scale == 1.f && c.shift == 1.f && g == out)
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
    int blocks = 0;
    std::vector<int64_t> numel;
    std::vector<int> grad_dtype, out_dtype;
    std::vector<Part> parts;
    std::vector<const void *> seen_grad;    // addresses that passed check_address, as in a step's pointer table
    std::vector<void *> seen_out;
    void *memory = nullptr;                 // the plan and what the kernels leave in it, one allocation
    ClipParams params{};                    // pointers into it
    size_t workspace = 0;
};

namespace {

void release(rikfad_clip c)
{
    counted_free(c->memory);
    delete c;
}

// Where `count` elements of T go in an image of the plan's memory, 16-byte aligned.
template <typename T> size_t place(size_t &bytes, size_t count)
{
    const size_t at = bytes;
    bytes += (sizeof(T) * count + 15) / 16 * 16;
    return at;
}

// Cuts tensors [t0, t1) into at most `most` shares of equal size.
bool plan_part(const rikfad_clip c, int t0, int t1, int64_t most, std::vector<Segment> &segments,
               std::vector<int32_t> &block_segment)
{
    double n = 0.0;
    for (int t = t0; t < t1; ++t)
        n += (double)c->numel[t];
    const double want = std::min((double)most, std::ceil(n / (double)kMinShare));
    const int64_t share = std::max<int64_t>(
        kShareStep, (int64_t)std::ceil(n / std::max(want, 1.0) / (double)kShareStep) * kShareStep);
    if (share > kMaxShare)
        return false;
    int64_t room = 0;       // left in the open share
    for (int t = t0; t < t1; ++t) {
        const int32_t first = (int32_t)segments.size();
        int64_t at = 0;
        do {                        // an empty tensor has one empty segment
            if (room <= 0) {
                block_segment.push_back((int32_t)segments.size());
                room = share;
            }
            // a cut at a multiple of kShareStep, or the tensor's end
            const int64_t take = std::min(c->numel[t] - at, (room + kShareStep - 1) / kShareStep * kShareStep);
            segments.push_back({at, at + take, t - t0, (int16_t)c->grad_dtype[t], (int16_t)c->out_dtype[t], t, first, 0, 0});
            at += take;
            room -= take;
        } while (at < c->numel[t]);
        for (size_t q = first; q < segments.size(); ++q)
            segments[q].count = (int32_t)segments.size() - first;
    }
    return true;
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
    std::vector<int32_t> block_segment;
    for (int t0 = 0; t0 < ntensors; t0 += kMaxTensors) {
        const int t1 = std::min(ntensors, t0 + kMaxTensors);
        const int b0 = (int)block_segment.size();
        if (!plan_part(c, t0, t1, (int64_t)sms * kClipBlocksPerSm, segments, block_segment))
            return report_error(RIKFAD_ERR_ARG, "the tensors are too large");
        if ((int)block_segment.size() > b0)
            c->parts.push_back({t0, t1, b0, (int)block_segment.size()});
    }
    if (c->parts.empty()) {         // no tensors: one block without segments
        c->parts.push_back({0, 0, 0, 1});
        block_segment.push_back(0);
    }
    c->blocks = (int)block_segment.size();
    block_segment.push_back((int32_t)segments.size());
    size_t bytes = 0;
    const size_t at_segments = place<Segment>(bytes, segments.size());
    const size_t at_blocks = place<int32_t>(bytes, block_segment.size());
    const size_t at_partial = place<double>(bytes, segments.size());
    const size_t at_sum = place<double>(bytes, ntensors);
    const size_t at_done = place<unsigned int>(bytes, ntensors);
    const size_t at_result = place<ClipResult>(bytes, 1);
    std::vector<char> image(bytes, 0);          // sums and counters start at zero
    if (!segments.empty())
        std::memcpy(&image[at_segments], segments.data(), sizeof(Segment) * segments.size());
    std::memcpy(&image[at_blocks], block_segment.data(), sizeof(int32_t) * block_segment.size());
    e = counted_malloc(&c->memory, bytes);
    if (e == cudaErrorMemoryAllocation)
        return report_error(RIKFAD_ERR_OOM, "cudaMalloc of a clipping plan failed: out of memory");
    if (e == cudaSuccess)
        e = cudaMemcpy(c->memory, image.data(), bytes, cudaMemcpyHostToDevice);
    // From pageable memory the copy returns when its bytes are staged, and a stream that
    // does not wait for the legacy one may run the plan at once.
    if (e == cudaSuccess)
        e = cudaStreamSynchronize(cudaStreamLegacy);
    if (e != cudaSuccess)
        return report_cuda(e, "memory of a clipping plan");
    c->workspace = bytes;
    char *const base = static_cast<char *>(c->memory);
    c->params.segments = reinterpret_cast<const Segment *>(base + at_segments);
    c->params.block_segment = reinterpret_cast<const int32_t *>(base + at_blocks);
    c->params.partial = reinterpret_cast<double *>(base + at_partial);
    c->params.tensor_sum = reinterpret_cast<double *>(base + at_sum);
    c->params.tensor_done = reinterpret_cast<unsigned int *>(base + at_done);
    c->params.result = reinterpret_cast<ClipResult *>(base + at_result);
    c->params.ntensors = ntensors;
    c->params.total_blocks = c->blocks;
    return RIKFAD_OK;
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
    const cudaError_t e = launch_chained(scale ? rikfad_clip_scale_kernel<CAP> : rikfad_clip_squares_kernel<CAP>, blocks,
                                         kClipThreads, 0, s, a, ptrs);
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
                               float *total, void *stream)
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
    if (total == nullptr || (c->ntensors > 0 && norms == nullptr))
        return report_error(RIKFAD_ERR_ARG, "norms or total is NULL");
    if ((uintptr_t)norms % sizeof(float) || (uintptr_t)total % sizeof(float))
        return report_error(RIKFAD_ERR_ALIGN, "norms or total is not aligned");
    if (out && !(max_norm >= 0))
        return report_error(RIKFAD_ERR_ARG, "max_norm must be >= 0");
    int rc = check_address(total, dev, "total");
    if (!rc && c->ntensors > 0)
        rc = check_address(norms, dev, "norms");
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
    ClipParams a = c->params;
    a.max_norm = max_norm;
    a.norms = norms;
    a.total = total;
    if ((rc = launch_parts(c, a, grad, out, false, s))) {
        // the parts that were launched have left their counts
        const char *const end = static_cast<const char *>(c->memory) + c->workspace;
        cudaMemsetAsync(a.tensor_done, 0, (size_t)(end - reinterpret_cast<const char *>(a.tensor_done)), s);
        cudaGetLastError();
        return rc;
    }
    return out ? launch_parts(c, a, grad, out, true, s) : RIKFAD_OK;
    RK_ENTRY_END
}

}  // extern "C"
