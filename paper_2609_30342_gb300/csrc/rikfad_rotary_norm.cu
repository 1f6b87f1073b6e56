// rikfad_rotary_norm.cu -- norms of queries and keys per head with the rotation by
// position in the same pass:
//   y = x r w,  r = 1 / sqrt(mean(x^2) + eps),  out = R(position) y,
// and from dout, with dy = R^T dout and g = dy w,
//   dx = r (g - x r^2 mean(g x)),  dw = sum dy x r.
//
// Memory bounds both: x is read once and out written once (backward: x and dout read,
// dx written).  A head's elements stay in the registers of the lanes that loaded them;
// its sums are shuffles.  Cosines and sines of a token are formed once for all heads
// of queries and keys.  The weights' gradients stay in registers over all heads of a
// block, leave one partial row a block and are joined by a second kernel in order.
#include <cuda_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <new>
#include <string>

#include "rikfad.h"
#include "rikfad_host.hpp"
#include "rikfad_kernels.cuh"
#include "rikfad_rotary.cuh"
#include "rikfad_types.cuh"

using namespace rikfad;

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kSms = 152;
constexpr int kForwardBlocksPerSm = 4, kBackwardBlocksPerSm = 2;
constexpr int kTablePairs = 4096;           // cosines and sines of a tile of tokens: 32 KB at most
constexpr int kMaxHeadDim = 512;
constexpr int kJoinThreads = 1024;

struct Heads {
    const void *x, *dout, *weight;
    void *out;
    int64_t x_batch, x_token, x_head, out_batch, out_token, out_head, dout_batch, dout_token, dout_head;
    int32_t heads;
};

struct Params {
    Heads lists[2];
    const uint64_t *turns;
    const void *positions;
    int64_t position_batch, start, tokens, tiles_per_sequence, tiles;
    int32_t position_bytes, nlists, head_dim, rotary_dim, pairs;
    int32_t interleaved, param_f32;
    int32_t tile;                       // tokens of a tile
    int32_t lanes, turn_units, units;   // of a head: lanes, units that turn (half layout), all units
    float magnitude, inv_dim, eps;
    float *part;                        // [block][list][head_dim]
};

// A unit is V pairs of one head, as two vectors of V elements: in the half layout
// one vector from each half, in the interleaved layout (and beyond rotary_dim) two
// neighbours.  first < 0: no unit; second < 0: one vector; pair < 0: nothing turns.
struct Place {
    int first, second, pair;
};

template <int V> __device__ __forceinline__ Place place_of(const Params &p, int unit)
{
    Place at;
    if (unit >= p.units)
        return {-1, -1, -1};
    if (p.interleaved) {
        at.first = 2 * unit * V;
        at.second = at.first + V < p.head_dim ? at.first + V : -1;
        at.pair = unit * V < p.pairs ? unit * V : -1;
    } else if (unit < p.turn_units) {
        at.first = unit * V;
        at.second = at.first + p.pairs;
        at.pair = at.first;
    } else {
        at.first = p.rotary_dim + 2 * (unit - p.turn_units) * V;
        at.second = at.first + V < p.head_dim ? at.first + V : -1;
        at.pair = -1;
    }
    return at;
}

template <typename T, int V, int U> struct Raw {
    Vec<T, V> a[U], b[U];

    __device__ __forceinline__ void load(const T *head, const Place (&at)[U])
    {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (at[u].first >= 0)
                a[u].word = __ldcs(reinterpret_cast<const decltype(a[u].word) *>(head + at[u].first));
            if (at[u].second >= 0)
                b[u].word = __ldcs(reinterpret_cast<const decltype(b[u].word) *>(head + at[u].second));
        }
    }
    __device__ __forceinline__ void store(T *head, const Place (&at)[U]) const
    {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (at[u].first >= 0)
                *reinterpret_cast<decltype(a[u].word) *>(head + at[u].first) = a[u].word;
            if (at[u].second >= 0)
                *reinterpret_cast<decltype(b[u].word) *>(head + at[u].second) = b[u].word;
        }
    }
    // Values; zeros where there are none.
    __device__ __forceinline__ void values(float (&v)[U][2 * V], const Place (&at)[U], bool active) const
    {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float x[V], y[V];
            widen(a[u], x);
            widen(b[u], y);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                v[u][e] = active && at[u].first >= 0 ? x[e] : 0.f;
                v[u][V + e] = active && at[u].second >= 0 ? y[e] : 0.f;
            }
        }
    }
    __device__ __forceinline__ void take(const float (&v)[U][2 * V])
    {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float x[V], y[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                x[e] = v[u][e];
                y[e] = v[u][V + e];
            }
            narrow(x, a[u]);
            narrow(y, b[u]);
        }
    }
};

__device__ __forceinline__ void turn_pair(float &x, float &y, const float2 &cs)
{
    const float u = x, v = y;
    x = fmaf(u, cs.x, -v * cs.y);
    y = fmaf(v, cs.x, u * cs.y);
}

// The pairs of the lane's units turned by the token's cosines and sines.
template <int V, int U>
__device__ __forceinline__ void turn(const Params &p, float (&v)[U][2 * V], const Place (&at)[U], const float2 *table)
{
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (at[u].pair < 0)
            continue;
        if (p.interleaved) {            // pair e is elements 2 e and 2 e + 1; the last unit may reach beyond rotary_dim
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (at[u].pair + e < p.pairs)
                    turn_pair(v[u][2 * e], v[u][2 * e + 1], table[at[u].pair + e]);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
                turn_pair(v[u][e], v[u][V + e], table[at[u].pair + e]);
        }
    }
}

// Where a group of lanes is in its tile's heads, and how it goes on.
struct Walk {
    int slot, head, slots, heads;

    __device__ __forceinline__ Walk(int item, int step, int count)
        : slot(item / count), head(item % count), slots(step / count), heads(step % count)
    {
    }
    __device__ __forceinline__ void next(int count)
    {
        head += heads;
        const int over = head >= count;
        head -= over ? count : 0;
        slot += slots + over;
    }
};

template <typename T, int V, int U, bool BACKWARD>
__global__ void __launch_bounds__(kThreads, BACKWARD ? kBackwardBlocksPerSm : kForwardBlocksPerSm)
rikfad_rotary_norm_kernel(const __grid_constant__ Params p)
{
    extern __shared__ float2 table[];
    __shared__ float weights[2][kMaxHeadDim];
    const int groups = kThreads / p.lanes, group = threadIdx.x / p.lanes, lane = threadIdx.x % p.lanes;
    const int warp_group = (threadIdx.x & ~31) / p.lanes;       // the first of the warp
    Place at[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
        at[u] = place_of<V>(p, lane + u * p.lanes);
    float sums[2][U][2 * V];
    if constexpr (BACKWARD)
#pragma unroll
        for (int l = 0; l < 2; ++l)
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < 2 * V; ++e)
                    sums[l][u][e] = 0.f;
    wait_for_predecessor();
    allow_successor_launch();
    for (int i = threadIdx.x; i < 2 * p.head_dim; i += kThreads) {
        const int l = i / p.head_dim, e = i % p.head_dim;
        const void *w = p.lists[l].weight;
        weights[l][e] = w == nullptr ? 1.f : p.param_f32 ? static_cast<const float *>(w)[e] : to_f32(static_cast<const T *>(w)[e]);
    }
    for (int64_t tile = blockIdx.x; tile < p.tiles; tile += gridDim.x) {
        const int64_t batch = p.tiles_per_sequence == p.tiles ? 0 : tile / p.tiles_per_sequence;
        const int64_t token0 = (tile - batch * p.tiles_per_sequence) * p.tile;
        const int here = (int)min((int64_t)p.tile, p.tokens - token0);
        __syncthreads();
        for (int i = threadIdx.x; i < here * p.pairs; i += kThreads) {
            const int64_t position =
                token_position(p.positions, p.position_bytes, p.position_batch, p.start, batch, token0 + i / p.pairs);
            const float2 cs = cosine_sine(position, p.turns[i % p.pairs]);
            table[i] = make_float2(cs.x * p.magnitude, cs.y * (BACKWARD ? -p.magnitude : p.magnitude));
        }
        __syncthreads();
#pragma unroll
        for (int l = 0; l < 2; ++l) {
            const Heads &h = p.lists[l];
            const int items = here * h.heads;
            if (items == 0)
                continue;
            float w[U][2 * V];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    w[u][e] = at[u].first >= 0 ? weights[l][at[u].first + e] : 0.f;
                    w[u][V + e] = at[u].second >= 0 ? weights[l][at[u].second + e] : 0.f;
                }
            const T *x = static_cast<const T *>(h.x) + batch * h.x_batch + token0 * h.x_token;
            const T *dout = static_cast<const T *>(h.dout) + batch * h.dout_batch + token0 * h.dout_token;
            T *out = static_cast<T *>(h.out) + batch * h.out_batch + token0 * h.out_token;
            Walk walk(group, groups, h.heads);
            Raw<T, V, U> in, din;
            if (group < items) {
                in.load(x + walk.slot * h.x_token + walk.head * h.x_head, at);
                if constexpr (BACKWARD)
                    din.load(dout + walk.slot * h.dout_token + walk.head * h.dout_head, at);
            }
            for (int first = warp_group, item = group; first < items; first += groups, item += groups) {
                const bool active = item < items;
                const int slot = walk.slot;
                T *to = out + walk.slot * h.out_token + walk.head * h.out_head;
                Raw<T, V, U> next, dnext;
                walk.next(h.heads);
                if (item + groups < items) {
                    next.load(x + walk.slot * h.x_token + walk.head * h.x_head, at);
                    if constexpr (BACKWARD)
                        dnext.load(dout + walk.slot * h.dout_token + walk.head * h.dout_head, at);
                }
                float v[U][2 * V], squares = 0.f;
                in.values(v, at, active);
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int e = 0; e < 2 * V; ++e)
                        squares = fmaf(v[u][e], v[u][e], squares);
                if constexpr (BACKWARD) {
                    float d[U][2 * V], product = 0.f;
                    din.values(d, at, active);
                    if (active)
                        turn<V, U>(p, d, at, table + slot * p.pairs);
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int e = 0; e < 2 * V; ++e)
                            product = fmaf(d[u][e] * w[u][e], v[u][e], product);
                    for (int s = p.lanes / 2; s > 0; s /= 2) {
                        squares += __shfl_xor_sync(~0u, squares, s);
                        product += __shfl_xor_sync(~0u, product, s);
                    }
                    const float r = active ? rsqrtf(fmaf(squares, p.inv_dim, p.eps)) : 0.f;
                    const float back = product * p.inv_dim * r * r;
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int e = 0; e < 2 * V; ++e) {
                            sums[l][u][e] = fmaf(d[u][e], v[u][e] * r, sums[l][u][e]);
                            v[u][e] = r * fmaf(-back, v[u][e], d[u][e] * w[u][e]);
                        }
                } else {
                    for (int s = p.lanes / 2; s > 0; s /= 2)
                        squares += __shfl_xor_sync(~0u, squares, s);
                    const float r = rsqrtf(fmaf(squares, p.inv_dim, p.eps));
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int e = 0; e < 2 * V; ++e)
                            v[u][e] *= r * w[u][e];
                    if (active)
                        turn<V, U>(p, v, at, table + slot * p.pairs);
                }
                if (active) {
                    in.take(v);
                    in.store(to, at);
                }
                in = next;
                din = dnext;
            }
        }
    }
    if constexpr (BACKWARD) {
        if (p.part == nullptr)
            return;
        float *sum = reinterpret_cast<float *>(table);      // [warp][element]
        const int in_warp = threadIdx.x & 31, warp = threadIdx.x >> 5;
        for (int l = 0; l < p.nlists; ++l) {
            __syncthreads();
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int e = 0; e < 2 * V; ++e) {
                    float s = l == 0 ? sums[0][u][e] : sums[1][u][e];
                    for (int d = 16; d >= p.lanes; d /= 2)
                        s += __shfl_xor_sync(~0u, s, d);
                    const int first = e < V ? at[u].first : at[u].second;
                    if (in_warp < p.lanes && first >= 0)
                        sum[warp * p.head_dim + first + e % V] = s;
                }
            __syncthreads();
            for (int e = threadIdx.x; e < p.head_dim; e += kThreads) {
                float s = 0.f;
                for (int w = 0; w < kWarps; ++w)
                    s += sum[w * p.head_dim + e];
                p.part[((int64_t)blockIdx.x * 2 + l) * p.head_dim + e] = s;
            }
        }
    }
}

// dweight of list blockIdx.y: the blocks' partial rows, each warp every 32nd of them, then
// the warps in order.
template <typename T>
__global__ void __launch_bounds__(kJoinThreads)
rikfad_rotary_norm_join_kernel(const float *part, int blocks, int head_dim, T *dq, T *dk, float *dq32, float *dk32)
{
    __shared__ float sum[kJoinThreads / 32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e = blockIdx.x * 32 + lane;
    wait_for_predecessor();
    allow_successor_launch();
    float s = 0.f;
    if (e < head_dim)
#pragma unroll 4
        for (int b = warp; b < blocks; b += kJoinThreads / 32)
            s += part[((int64_t)b * 2 + blockIdx.y) * head_dim + e];
    sum[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && e < head_dim) {
        s = 0.f;
        for (int w = 0; w < kJoinThreads / 32; ++w)
            s += sum[w][lane];
        T *to = blockIdx.y ? dk : dq;
        float *to32 = blockIdx.y ? dk32 : dq32;
        if (to)
            to[e] = from_f32<T>(s);
        if (to32)
            to32[e] = s;
    }
}

// ------------------------------------------------------------------------ host

int bad(const std::string &msg) { return report_error(RIKFAD_ERR_ARG, msg); }

int check_sizes(const rikfad_rotary_norm *p)
{
    if (p == nullptr)
        return bad("p is NULL");
    if (p->batch < 0 || p->tokens < 0 || p->batch > (int64_t)1 << 40 || p->tokens > (int64_t)1 << 40)
        return bad("batch or tokens is out of range");
    if (p->tokens > 0 && p->batch > ((int64_t)1 << 40) / p->tokens)
        return bad("batch times tokens must be at most 2^40");
    if (p->head_dim < 1 || p->head_dim > kMaxHeadDim)
        return bad("head_dim must be in [1, 512]");
    if (p->rotary_dim < 0 || p->rotary_dim > p->head_dim || p->rotary_dim % 2)
        return bad("rotary_dim must be even and in [0, head_dim]");
    if (p->layout != RIKFAD_ROTARY_HALF && p->layout != RIKFAD_ROTARY_INTERLEAVED)
        return bad("layout must be a rikfad_rotary_layout");
    if (!dtype_ok(p->dtype))
        return bad("dtype is not a rikfad_dtype");
    if (p->param_dtype != RIKFAD_F32 && p->param_dtype != p->dtype)
        return bad("param_dtype must be RIKFAD_F32 or dtype");
    if (p->nlists < 0 || p->nlists > 2)
        return bad("nlists must be 0, 1 or 2");
    if (!std::isfinite(p->magnitude))
        return bad("magnitude must be finite");
    if (!std::isfinite(p->eps) || p->eps < 0)
        return bad("eps must be finite and >= 0");
    if (p->positions && p->position_bytes != 4 && p->position_bytes != 8)
        return bad("position_bytes must be 4 or 8");
    for (int i = 0; i < p->nlists; ++i) {
        const rikfad_rotary_norm_heads &l = p->lists[i];
        if (l.heads < 0 || l.heads > (int64_t)1 << 16)
            return bad("heads is out of range");
        if (l.heads == 0 || p->tokens == 0 || p->batch == 0)
            continue;
        if ((l.heads > 1 && l.out_head == 0) || (p->tokens > 1 && l.out_token == 0) || (p->batch > 1 && l.out_batch == 0))
            return bad("a stride of 0 would write several heads, tokens or sequences to one place");
    }
    return RIKFAD_OK;
}

int check_place(const void *v, const char *name, size_t align, int device)
{
    if (v == nullptr)
        return bad(std::string(name) + " is NULL");
    if ((uintptr_t)v % align)
        return report_error(RIKFAD_ERR_ALIGN, std::string(name) + " is not aligned");
    return check_address(v, device, name);
}

int check(const rikfad_rotary_norm *p, bool backward)
{
    int rc = check_sizes(p);
    if (rc)
        return rc;
    int device = -1;
    const cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess)
        return report_cuda(e, "cudaGetDevice");
    const size_t pb = (size_t)dtype_bytes(p->param_dtype), b = (size_t)dtype_bytes(p->dtype);
    for (int i = 0; !rc && backward && i < p->nlists; ++i)
        if (p->lists[i].dweight)
            rc = check_place(p->lists[i].dweight, "dweight", pb, device);
    if (rc || p->batch == 0 || p->tokens == 0)
        return rc;
    if (p->rotary_dim > 0)
        rc = check_place(p->turns, "turns", 8, device);
    if (!rc && p->positions)
        rc = check_place(p->positions, "positions", (size_t)p->position_bytes, device);
    for (int i = 0; !rc && i < p->nlists; ++i) {
        const rikfad_rotary_norm_heads &l = p->lists[i];
        if (l.heads == 0)
            continue;
        rc = check_place(l.x, "x", b, device);
        if (!rc) rc = check_place(l.out, "out", b, device);
        if (!rc && backward) rc = check_place(l.dout, "dout", b, device);
        if (!rc && l.weight) rc = check_place(l.weight, "weight", pb, device);
        if (!rc && l.x == l.out && (l.x_batch != l.out_batch || l.x_token != l.out_token || l.x_head != l.out_head))
            return bad("x = out needs equal strides");
        if (!rc && backward && l.dout == l.out &&
            (l.dout_batch != l.out_batch || l.dout_token != l.out_token || l.dout_head != l.out_head))
            return bad("dout = dx needs equal strides");
    }
    return rc;
}

size_t workspace_of(const rikfad_rotary_norm *p)
{
    return (size_t)kSms * kBackwardBlocksPerSm * 2 * (size_t)p->head_dim * sizeof(float);
}

template <typename T, int V, int U, bool BACKWARD> cudaError_t launch(Params p, const rikfad_rotary_norm *d, cudaStream_t s)
{
    const int groups = kThreads / p.lanes;
    const int64_t heads = p.lists[0].heads + p.lists[1].heads, tokens = p.tiles * p.tokens;   // p.tiles: sequences, here
    // Heads of a group in a tile: 2 to 16, so that a launch has a dozen rounds of blocks
    // where it can, within the table's size.
    const int64_t share = tokens * heads / ((int64_t)12 * kForwardBlocksPerSm * kSms * groups);
    const int64_t each = std::max<int64_t>(2, std::min<int64_t>(16, share));
    const int64_t most = std::min<int64_t>(p.tokens, p.pairs ? std::max(1, kTablePairs / p.pairs) : 1 << 10);
    p.tile = (int32_t)std::max<int64_t>(1, std::min(most, each * groups / heads));
    while (p.tile > 1 && (tokens + p.tile - 1) / p.tile < 2 * kSms)
        p.tile /= 2;
    p.tiles_per_sequence = (p.tokens + p.tile - 1) / p.tile;
    p.tiles *= p.tiles_per_sequence;
    if (!BACKWARD && p.tiles > INT32_MAX)
        return cudaErrorInvalidConfiguration;
    const int64_t blocks = BACKWARD ? std::min<int64_t>(p.tiles, kSms * kBackwardBlocksPerSm) : p.tiles;
    size_t smem = sizeof(float2) * (size_t)p.tile * p.pairs;
    if (BACKWARD && p.part)
        smem = std::max(smem, sizeof(float) * kWarps * (size_t)p.head_dim);
    const cudaError_t e =
        launch_chained(rikfad_rotary_norm_kernel<T, V, U, BACKWARD>, dim3((unsigned)blocks), kThreads, smem, s, p);
    if (e != cudaSuccess || !BACKWARD || p.part == nullptr)
        return e;
    void *const dq = d->lists[0].dweight, *const dk = d->nlists > 1 ? d->lists[1].dweight : nullptr;
    const bool f32 = p.param_f32;
    return launch_chained(rikfad_rotary_norm_join_kernel<T>, dim3((unsigned)(p.head_dim + 31) / 32, (unsigned)p.nlists), kJoinThreads,
                          0, s, (const float *)p.part, (int)blocks, (int)p.head_dim, f32 ? nullptr : (T *)dq,
                          f32 ? nullptr : (T *)dk, f32 ? (float *)dq : nullptr, f32 ? (float *)dk : nullptr);
}

// Lanes of a head: enough for one unit each, up to a warp.
template <typename T, int V, bool BACKWARD> cudaError_t launch(Params p, const rikfad_rotary_norm *d, cudaStream_t s)
{
    if (p.interleaved) {
        p.units = (p.head_dim + 2 * V - 1) / (2 * V);
    } else {
        p.turn_units = p.pairs / V;
        p.units = p.turn_units + (p.head_dim - p.rotary_dim + 2 * V - 1) / (2 * V);
    }
    p.lanes = 1;
    while (p.lanes < 32 && p.lanes < p.units)
        p.lanes *= 2;
    if constexpr (V <= 1)
        if (p.units > 128)
            return launch<T, V, 8, BACKWARD>(p, d, s);
    if constexpr (V <= 2)
        if (p.units > 64)
            return launch<T, V, 4, BACKWARD>(p, d, s);
    if constexpr (V <= 4)
        if (p.units > 32)
            return launch<T, V, 2, BACKWARD>(p, d, s);
    return launch<T, V, 1, BACKWARD>(p, d, s);
}

template <typename T, bool BACKWARD> cudaError_t launch(const rikfad_rotary_norm *d, cudaStream_t s)
{
    Params p{};
    p.turns = d->turns;
    p.positions = d->positions;
    p.position_batch = d->position_batch;
    p.start = d->start;
    p.position_bytes = d->position_bytes;
    p.nlists = d->nlists;
    p.head_dim = d->head_dim;
    p.rotary_dim = d->rotary_dim;
    p.pairs = d->rotary_dim / 2;
    p.interleaved = d->layout == RIKFAD_ROTARY_INTERLEAVED;
    p.param_f32 = d->param_dtype == RIKFAD_F32;
    p.magnitude = (float)d->magnitude;
    p.inv_dim = 1.f / (float)d->head_dim;
    p.eps = (float)d->eps;
    p.tokens = d->tokens;
    p.tiles = d->batch;
    bool wanted = false;
    // The widest vectors that the heads' layout and addresses allow: every part of a
    // head and every stride is a whole number of vectors, and so are the addresses.
    uint64_t parts = (uint64_t)d->head_dim;
    if (!p.interleaved)
        parts |= (uint64_t)p.pairs | (uint64_t)(d->head_dim - d->rotary_dim);
    bool one = true;            // one run of tokens: every batch stride is `tokens` token strides
    for (int i = 0; i < d->nlists; ++i) {
        const rikfad_rotary_norm_heads &l = d->lists[i];
        wanted = wanted || (BACKWARD && l.dweight);
        Heads &h = p.lists[i];
        h = {l.x, l.dout, l.weight, l.out, l.x_batch, l.x_token, l.x_head, l.out_batch, l.out_token, l.out_head,
             l.dout_batch, l.dout_token, l.dout_head, (int32_t)l.heads};
        if (!BACKWARD) {
            h.dout = nullptr;
            h.dout_batch = h.dout_token = h.dout_head = 0;
        }
        if (l.heads == 0)
            continue;
        parts |= (uint64_t)((uintptr_t)h.x | (uintptr_t)h.out | (uintptr_t)h.dout) / sizeof(T);
        if (l.heads > 1)
            parts |= (uint64_t)h.x_head | (uint64_t)h.out_head | (uint64_t)h.dout_head;
        if (p.tokens > 1)
            parts |= (uint64_t)h.x_token | (uint64_t)h.out_token | (uint64_t)h.dout_token;
        if (d->batch > 1)
            parts |= (uint64_t)h.x_batch | (uint64_t)h.out_batch | (uint64_t)h.dout_batch;
        if (p.tokens == 1) {
            h.x_token = h.x_batch;
            h.out_token = h.out_batch;
            h.dout_token = h.dout_batch;
        }
        one = one && h.x_batch == h.x_token * p.tokens && h.out_batch == h.out_token * p.tokens &&
              h.dout_batch == h.dout_token * p.tokens;
    }
    if (d->batch > 1 && one && p.positions && p.position_batch == p.tokens) {
        p.tokens *= p.tiles;
        p.tiles = 1;
    }
    if (BACKWARD && wanted)
        p.part = static_cast<float *>(d->workspace);
    if constexpr (sizeof(T) == 2)
        if (parts % 8 == 0)
            return launch<T, 8, BACKWARD>(p, d, s);
    return parts % 4 == 0   ? launch<T, 4, BACKWARD>(p, d, s)
           : parts % 2 == 0 ? launch<T, 2, BACKWARD>(p, d, s)
                            : launch<T, 1, BACKWARD>(p, d, s);
}

template <bool BACKWARD> int run(const rikfad_rotary_norm *p, void *stream)
{
    const int rc = check(p, BACKWARD);
    if (rc)
        return rc;
    bool any = false, wanted = false;
    for (int i = 0; i < p->nlists; ++i) {
        any = any || (p->lists[i].heads > 0 && p->batch > 0 && p->tokens > 0);
        wanted = wanted || (BACKWARD && p->lists[i].dweight);
    }
    if (any && wanted) {
        if (p->workspace == nullptr || p->workspace_bytes < workspace_of(p))
            return bad("the workspace is smaller than rikfad_rotary_norm_workspace");
        if ((uintptr_t)p->workspace % 16)
            return report_error(RIKFAD_ERR_ALIGN, "workspace is not aligned");
    }
    cudaError_t e = cudaPeekAtLastError();
    if (e != cudaSuccess)
        return report_cuda(e, "earlier CUDA error");
    const cudaStream_t s = (cudaStream_t)stream;
    if (!any) {
        for (int i = 0; i < p->nlists && wanted; ++i)
            if (p->lists[i].dweight) {
                e = cudaMemsetAsync(p->lists[i].dweight, 0, (size_t)dtype_bytes(p->param_dtype) * (size_t)p->head_dim, s);
                if (e != cudaSuccess)
                    return report_cuda(e, "cudaMemsetAsync");
            }
        return RIKFAD_OK;
    }
    e = p->dtype == RIKFAD_F32    ? launch<float, BACKWARD>(p, s)
        : p->dtype == RIKFAD_BF16 ? launch<__nv_bfloat16, BACKWARD>(p, s)
                                  : launch<__half, BACKWARD>(p, s);
    return e == cudaSuccess ? RIKFAD_OK : report_cuda(e, "launch of the rotary norm's kernels");
}

}  // namespace

extern "C" {

RIKFAD_API size_t rikfad_rotary_norm_workspace(const rikfad_rotary_norm *p)
{
    RK_ENTRY_BEGIN
    if (check_sizes(p))
        return 0;
    report_error(RIKFAD_OK, "");
    return workspace_of(p);
    }
    catch (...)
    {
        return 0;
    }
}

RIKFAD_API int rikfad_rotary_norm_forward(const rikfad_rotary_norm *p, void *stream)
{
    RK_ENTRY_BEGIN
    return run<false>(p, stream);
    RK_ENTRY_END
}

RIKFAD_API int rikfad_rotary_norm_backward(const rikfad_rotary_norm *p, void *stream)
{
    RK_ENTRY_BEGIN
    return run<true>(p, stream);
    RK_ENTRY_END
}

}  // extern "C"
