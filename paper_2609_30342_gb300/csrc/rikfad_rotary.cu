// rikfad_rotary.cu -- rotary positions: pair (a, b) number i of a head of the
// token at position t turns by t f_i,
//   (a, b) -> magnitude (a cos - b sin, b cos + a sin).
//
// The angle is t times f_i / (2 pi) in 64-bit fixed point: the integer product
// wraps at whole turns, so its high half is the fraction of a turn to 2^-32 at
// any position (a float32 product is off by 0.06 rad at position 1e6).
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <string>

#include "rikfad.h"
#include "rikfad_host.hpp"
#include "rikfad_types.cuh"

using namespace rikfad;

namespace {

constexpr int kRotaryThreads = 256;

struct RotaryParams {
    rikfad_rotary d;
    float magnitude;
};

__device__ __forceinline__ void angle(const RotaryParams &p, int64_t batch, int64_t token, int pair, float &cosine, float &sine)
{
    int64_t position = p.d.start + token;
    if (p.d.positions) {
        const int64_t i = batch * p.d.position_batch + token;
        position = p.d.position_bytes == 4 ? (int64_t)static_cast<const int32_t *>(p.d.positions)[i]
                                           : static_cast<const int64_t *>(p.d.positions)[i];
    }
    // the turn's fraction in [-1/2, 1/2), in half turns for sincospi
    const uint64_t turn = (uint64_t)position * p.d.turns[pair];
    sincospif((float)(int32_t)(turn >> 32) * 0x1p-31f, &sine, &cosine);
    cosine *= p.magnitude;
    sine *= p.d.inverse ? -p.magnitude : p.magnitude;
}

template <typename T> __global__ void __launch_bounds__(kRotaryThreads) rikfad_rotary_kernel(const __grid_constant__ RotaryParams p)
{
    const rikfad_rotary_heads &l = p.d.lists[blockIdx.y];
    const int pairs = p.d.rotary_dim / 2, slots = p.d.head_dim - pairs;     // pairs, then single elements
    const int64_t work = p.d.batch * p.d.tokens * l.heads * slots;
    for (int64_t w = (int64_t)blockIdx.x * kRotaryThreads + threadIdx.x; w < work; w += (int64_t)gridDim.x * kRotaryThreads) {
        const int slot = (int)(w % slots);
        const int64_t head = w / slots % l.heads, at = w / slots / l.heads;
        const int64_t token = at % p.d.tokens, batch = at / p.d.tokens;
        const T *src = static_cast<const T *>(l.src) + batch * l.src_batch + token * l.src_token + head * l.src_head;
        T *dst = static_cast<T *>(l.dst) + batch * l.dst_batch + token * l.dst_token + head * l.dst_head;
        if (slot >= pairs) {
            dst[pairs + slot] = src[pairs + slot];
            continue;
        }
        float c, s;
        angle(p, batch, token, slot, c, s);
        const int i = p.d.layout == RIKFAD_ROTARY_HALF ? slot : 2 * slot;
        const int j = p.d.layout == RIKFAD_ROTARY_HALF ? slot + pairs : 2 * slot + 1;
        const float a = to_f32(src[i]), b = to_f32(src[j]);
        dst[i] = from_f32<T>(fmaf(a, c, -b * s));
        dst[j] = from_f32<T>(fmaf(b, c, a * s));
    }
}

int bad(const std::string &msg) { return report_error(RIKFAD_ERR_ARG, msg); }

int check(const rikfad_rotary *p)
{
    if (p == nullptr)
        return bad("p is NULL");
    if (p->batch < 0 || p->tokens < 0 || p->batch > (int64_t)1 << 40 || p->tokens > (int64_t)1 << 40)
        return bad("batch or tokens is out of range");
    if (p->tokens > 0 && p->batch > ((int64_t)1 << 40) / p->tokens)
        return bad("batch times tokens must be at most 2^40");
    if (p->head_dim < 1 || p->head_dim > 4096)
        return bad("head_dim must be in [1, 4096]");
    if (p->rotary_dim < 0 || p->rotary_dim > p->head_dim || p->rotary_dim % 2)
        return bad("rotary_dim must be even and in [0, head_dim]");
    if (p->layout != RIKFAD_ROTARY_HALF && p->layout != RIKFAD_ROTARY_INTERLEAVED)
        return bad("layout must be a rikfad_rotary_layout");
    if (!dtype_ok(p->dtype))
        return bad("dtype is not a rikfad_dtype");
    if (p->nlists < 0 || p->nlists > 2)
        return bad("nlists must be 0, 1 or 2");
    if (!std::isfinite(p->magnitude))
        return bad("magnitude must be finite");
    if (p->positions && p->position_bytes != 4 && p->position_bytes != 8)
        return bad("position_bytes must be 4 or 8");
    for (int i = 0; i < p->nlists; ++i) {
        const rikfad_rotary_heads &l = p->lists[i];
        if (l.heads < 0 || l.heads > (int64_t)1 << 24)
            return bad("heads is out of range");
    }
    int device = -1;
    const cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess)
        return report_cuda(e, "cudaGetDevice");
    if (p->batch == 0 || p->tokens == 0)
        return RIKFAD_OK;
    int rc = RIKFAD_OK;
    if (p->rotary_dim > 0) {
        if (p->turns == nullptr)
            return bad("turns is NULL");
        if ((uintptr_t)p->turns % 8)
            return report_error(RIKFAD_ERR_ALIGN, "turns is not aligned");
        rc = check_address(p->turns, device, "turns");
    }
    if (!rc && p->positions) {
        if ((uintptr_t)p->positions % (uintptr_t)p->position_bytes)
            return report_error(RIKFAD_ERR_ALIGN, "positions is not aligned");
        rc = check_address(p->positions, device, "positions");
    }
    for (int i = 0; !rc && i < p->nlists; ++i) {
        const rikfad_rotary_heads &l = p->lists[i];
        if (l.heads == 0)
            continue;
        if (l.src == nullptr || l.dst == nullptr)
            return bad("src or dst is NULL");
        if ((uintptr_t)l.src % (uintptr_t)dtype_bytes(p->dtype) || (uintptr_t)l.dst % (uintptr_t)dtype_bytes(p->dtype))
            return report_error(RIKFAD_ERR_ALIGN, "src or dst is not aligned to its element type");
        if (l.src == l.dst && (l.src_batch != l.dst_batch || l.src_token != l.dst_token || l.src_head != l.dst_head))
            return bad("src = dst needs equal strides");
        rc = check_address(l.src, device, "src");
        if (!rc) rc = check_address(l.dst, device, "dst");
    }
    return rc;
}

template <typename T> cudaError_t launch(const RotaryParams &p, cudaStream_t s)
{
    int64_t most = 0;
    for (int i = 0; i < p.d.nlists; ++i)
        most = std::max(most, p.d.lists[i].heads);
    const int64_t work = p.d.batch * p.d.tokens * most * (p.d.head_dim - p.d.rotary_dim / 2);
    if (work == 0)
        return cudaSuccess;
    const dim3 grid((unsigned)std::min<int64_t>((work + kRotaryThreads - 1) / kRotaryThreads, 152 * 16), (unsigned)p.d.nlists);
    rikfad_rotary_kernel<T><<<grid, kRotaryThreads, 0, s>>>(p);
    return cudaGetLastError();
}

}  // namespace

extern "C" {

RIKFAD_API int rikfad_rotary_turns(const double *radians, int64_t n, uint64_t *turns)
{
    if (n < 0 || (n > 0 && (radians == nullptr || turns == nullptr)))
        return bad("need n >= 0, radians and turns");
    for (int64_t i = 0; i < n; ++i) {
        const double t = radians[i] / 6.283185307179586476925;
        if (!std::isfinite(t))
            return bad("radians must be finite");
        const double f = std::ldexp(t - std::floor(t), 64);      // in [0, 2^64]
        turns[i] = f < 0x1p64 ? (uint64_t)f : 0;
    }
    return RIKFAD_OK;
}

RIKFAD_API int rikfad_rotary_apply(const rikfad_rotary *p, void *stream)
{
    RK_ENTRY_BEGIN
    const int rc = check(p);
    if (rc)
        return rc;
    cudaError_t e = cudaPeekAtLastError();
    if (e != cudaSuccess)
        return report_cuda(e, "earlier CUDA error");
    RotaryParams r{};
    r.d = *p;
    r.magnitude = (float)p->magnitude;
    const cudaStream_t s = (cudaStream_t)stream;
    e = p->dtype == RIKFAD_F32    ? launch<float>(r, s)
        : p->dtype == RIKFAD_BF16 ? launch<__nv_bfloat16>(r, s)
                                  : launch<__half>(r, s);
    return e == cudaSuccess ? RIKFAD_OK : report_cuda(e, "launch rikfad_rotary_kernel");
    RK_ENTRY_END
}

}  // extern "C"
