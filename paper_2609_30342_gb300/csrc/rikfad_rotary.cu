// rikfad_rotary.cu -- rotary positions: pair (a, b) number i of a head of the
// token at position t turns by t f_i,
//   (a, b) -> magnitude (a cos - b sin, b cos + a sin).
//
// The angle is t times f_i / (2 pi) in 64-bit fixed point: the integer product
// wraps at whole turns, so its high half is the fraction of a turn to 2^-32 at
// any position (a float32 product is off by 0.06 rad at position 1e6).
//
// Memory bounds it: every element is read once and written once, and the cosines
// and sines of a token are formed once for all heads of queries and keys.  131072
// tokens of 40 heads of 128 take 430 us (2.7 GB, 6.2 TB/s), 16384 tokens of 24 heads
// of 64 about 23 us (101 MB, 4.3 TB/s; a copy of as many bytes takes 22).
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

constexpr int kRotaryThreads = 256;
constexpr int kSms = 152;
constexpr int kRotaryBlocksPerSm = 5;
constexpr int kTableFloats = 8192;      // cosines and sines of a tile of tokens: 32 KB at most

struct RotaryParams {
    rikfad_rotary d;
    float magnitude, sine_sign;
    int32_t tile;                       // tokens of one block
    int32_t turn_units, units;          // of a head: units that turn, all units
    int32_t heads;                      // of both lists
    bool copy;                          // elements beyond rotary_dim are copied
};

// V elements as one load.
template <int BYTES> struct Word;
template <> struct Word<2> { using type = uint16_t; };
template <> struct Word<4> { using type = uint32_t; };
template <> struct Word<8> { using type = uint2; };
template <> struct Word<16> { using type = uint4; };

template <typename T, int V> union Vec {
    typename Word<V * sizeof(T)>::type word;
    uint32_t pairs[V * sizeof(T) >= 4 ? V * sizeof(T) / 4 : 1];
    T v[V];
    __device__ __forceinline__ Vec() {}
};

template <typename T, int V> __device__ __forceinline__ void widen(const Vec<T, V> &r, float (&f)[V])
{
    if constexpr (sizeof(T) == 2 && V > 1) {
#pragma unroll
        for (int i = 0; i < V / 2; ++i)
            unpack2(r.pairs[i], f[2 * i], f[2 * i + 1], T());
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            f[i] = to_f32(r.v[i]);
    }
}

template <typename T, int V> __device__ __forceinline__ void narrow(const float (&f)[V], Vec<T, V> &r)
{
    if constexpr (sizeof(T) == 2 && V > 1) {
#pragma unroll
        for (int i = 0; i < V / 2; ++i)
            r.pairs[i] = pack2(f[2 * i], f[2 * i + 1], T());
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            r.v[i] = from_f32<T>(f[i]);
    }
}

// Where a thread is in its tile, and how it goes on: divisions once, not per unit.
struct Walk {
    int slot, head, unit;       // token within the tile, head of both lists, unit of the head
    int slots, heads, units;    // of one step

    __device__ __forceinline__ Walk(const RotaryParams &p, int w, int step)
    {
        unit = w % p.units;
        head = w / p.units % p.heads;
        slot = w / p.units / p.heads;
        units = step % p.units;
        heads = step / p.units % p.heads;
        slots = step / p.units / p.heads;
    }
    __device__ __forceinline__ void next(const RotaryParams &p)
    {
        unit += units;
        const int carry = unit >= p.units;
        unit -= carry ? p.units : 0;
        head += heads + carry;
        const int over = head >= p.heads;
        head -= over ? p.heads : 0;
        slot += slots + over;
    }
};

// A unit is V pairs of one head, as two vectors of V elements: in the half layout
// one vector from each half, in the interleaved layout two neighbours.  Beyond
// the turning units, a unit is up to two vectors of elements that are copied.
template <typename T, int V> struct Unit {
    const T *src;
    T *dst;
    int first, second;      // elements of the head; second < 0: none
    int pair;               // first pair, in the tile's table; < 0: copy
    Vec<T, V> a, b;

    __device__ __forceinline__ void locate(const RotaryParams &p, int64_t token0, const Walk &w)
    {
        const int64_t at = token0 + w.slot;
        const int64_t batch = p.d.batch == 1 ? 0 : at / p.d.tokens, token = at - batch * p.d.tokens;
        const int list = w.head >= (int)p.d.lists[0].heads;
        const int head = w.head - (list ? (int)p.d.lists[0].heads : 0);
        const rikfad_rotary_heads &l = p.d.lists[list];
        src = static_cast<const T *>(l.src) + batch * l.src_batch + token * l.src_token + head * l.src_head;
        dst = static_cast<T *>(l.dst) + batch * l.dst_batch + token * l.dst_token + head * l.dst_head;
        if (w.unit < p.turn_units) {
            const bool half = p.d.layout == RIKFAD_ROTARY_HALF;
            first = half ? w.unit * V : 2 * w.unit * V;
            second = first + (half ? p.d.rotary_dim / 2 : V);
            pair = w.slot * (p.d.rotary_dim / 2) + w.unit * V;
        } else {
            first = p.d.rotary_dim + 2 * (w.unit - p.turn_units) * V;
            second = first + V < p.d.head_dim ? first + V : -1;
            pair = -1;
        }
    }

    __device__ __forceinline__ void load()
    {
        a.word = __ldcs(reinterpret_cast<const decltype(a.word) *>(src + first));
        if (second >= 0)
            b.word = __ldcs(reinterpret_cast<const decltype(b.word) *>(src + second));
    }

    __device__ __forceinline__ void turn(const RotaryParams &p, const float2 *table)
    {
        if (pair < 0)
            return;
        float x[V], y[V];
        widen(a, x);
        widen(b, y);
        if (p.d.layout == RIKFAD_ROTARY_HALF) {
#pragma unroll
            for (int e = 0; e < V; ++e)
                turn(x[e], y[e], table[pair + e]);
        } else {                // pair e is elements 2 e and 2 e + 1 of the two vectors together
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float &even = 2 * e < V ? x[2 * e % V] : y[2 * e % V];
                float &odd = 2 * e + 1 < V ? x[(2 * e + 1) % V] : y[(2 * e + 1) % V];
                turn(even, odd, table[pair + e]);
            }
        }
        narrow(x, a);
        narrow(y, b);
    }

    __device__ __forceinline__ static void turn(float &x, float &y, const float2 &cs)
    {
        const float u = x, v = y;
        x = fmaf(u, cs.x, -v * cs.y);
        y = fmaf(v, cs.x, u * cs.y);
    }

    __device__ __forceinline__ void store() const
    {
        *reinterpret_cast<decltype(a.word) *>(dst + first) = a.word;
        if (second >= 0)
            *reinterpret_cast<decltype(b.word) *>(dst + second) = b.word;
    }
};

// A block takes `tile` tokens: it forms their cosines and sines once, for all
// heads, and its threads walk the tile's units, the next one's loads ahead of the
// present one's arithmetic and the first one's ahead of the table.  blockIdx.y
// splits the units of a tile where tokens are few.
template <typename T, int V>
__global__ void __launch_bounds__(kRotaryThreads) rikfad_rotary_kernel(const __grid_constant__ RotaryParams p)
{
    extern __shared__ float2 table[];
    const int64_t tokens = p.d.batch * p.d.tokens, token0 = (int64_t)blockIdx.x * p.tile;
    const int here = (int)min((int64_t)p.tile, tokens - token0);
    const int work = here * p.heads * p.units, step = kRotaryThreads * gridDim.y;
    int w = blockIdx.y * kRotaryThreads + threadIdx.x;
    Walk walk(p, w, step);
    wait_for_predecessor();
    Unit<T, V> unit;
    if (w < work) {
        unit.locate(p, token0, walk);
        unit.load();
    }
    const int pairs = p.d.rotary_dim / 2;
    for (int i = threadIdx.x; i < here * pairs; i += kRotaryThreads) {
        const int64_t at = token0 + i / pairs;
        const int64_t batch = p.d.batch == 1 ? 0 : at / p.d.tokens, token = at - batch * p.d.tokens;
        int64_t position = p.d.start + token;
        if (p.d.positions) {
            const int64_t k = batch * p.d.position_batch + token;
            position = p.d.position_bytes == 4 ? (int64_t)static_cast<const int32_t *>(p.d.positions)[k]
                                               : static_cast<const int64_t *>(p.d.positions)[k];
        }
        // the turn's fraction in [-1/2, 1/2), in half turns for sincospi
        const uint64_t turn = (uint64_t)position * p.d.turns[i % pairs];
        float c, s;
        sincospif((float)(int32_t)(turn >> 32) * 0x1p-31f, &s, &c);
        table[i] = make_float2(c * p.magnitude, s * p.sine_sign);
    }
    __syncthreads();
    allow_successor_launch();
    while (w < work) {
        Unit<T, V> next;
        w += step;
        if (w < work) {
            walk.next(p);
            next.locate(p, token0, walk);
            next.load();
        }
        unit.turn(p, table);
        unit.store();
        unit = next;
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
        if (l.heads < 0 || l.heads > (int64_t)1 << 16)
            return bad("heads is out of range");
        if (l.heads == 0 || p->tokens == 0 || p->batch == 0)
            continue;
        if ((l.heads > 1 && l.dst_head == 0) || (p->tokens > 1 && l.dst_token == 0) || (p->batch > 1 && l.dst_batch == 0))
            return bad("a stride of 0 would write several heads, tokens or sequences to one place");
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

template <typename T, int V> cudaError_t launch(RotaryParams p, cudaStream_t s)
{
    const int rest = p.copy ? p.d.head_dim - p.d.rotary_dim : 0, pairs = p.d.rotary_dim / 2;
    p.turn_units = pairs / V;
    p.units = p.turn_units + (rest + 2 * V - 1) / (2 * V);
    const int64_t per_token = (int64_t)p.heads * p.units, tokens = p.d.batch * p.d.tokens;
    if (per_token == 0 || tokens == 0)
        return cudaSuccess;
    // Units of a thread: 2 to 16, so that a launch has a dozen rounds of blocks where it
    // can (16384 tokens of 24 x 64: 45 us for two calls with 2, 77 with 16; 131072 tokens of
    // 40 x 128: 448 us with 16, 530 with 2), within the table's size.
    const int64_t share = tokens * per_token / ((int64_t)12 * kRotaryBlocksPerSm * kSms * kRotaryThreads);
    const int64_t each = std::max<int64_t>(2, std::min<int64_t>(16, share));
    const int64_t most = pairs ? std::max(1, kTableFloats / 2 / pairs) : 1 << 10;
    p.tile = (int32_t)std::max<int64_t>(1, std::min(most, each * kRotaryThreads / per_token));
    // Few tokens: smaller tiles, then several blocks for a tile, until the SMs have work.
    while (p.tile > 1 && (tokens + p.tile - 1) / p.tile < 2 * kSms)
        p.tile /= 2;
    const int64_t tiles = (tokens + p.tile - 1) / p.tile;
    const int64_t want = (p.tile * per_token + kRotaryThreads - 1) / kRotaryThreads;    // blocks of one unit a thread
    const int64_t splits = std::max<int64_t>(1, std::min<int64_t>(want, 2 * kSms / tiles));
    if (tiles > INT32_MAX || p.tile * per_token > INT32_MAX / 2)
        return cudaErrorInvalidConfiguration;
    return launch_chained(rikfad_rotary_kernel<T, V>, dim3((unsigned)tiles, (unsigned)splits), kRotaryThreads,
                          sizeof(float2) * (size_t)p.tile * pairs, s, p);
}

// The widest vectors that the heads' layout and addresses allow: every part of a
// head (half of the pairs, the elements beyond them) and every stride is a whole
// number of vectors, and so are the addresses.
template <typename T> cudaError_t launch(RotaryParams p, cudaStream_t s)
{
    uint64_t parts = (uint64_t)(p.d.rotary_dim / 2) | (uint64_t)(p.d.head_dim - p.d.rotary_dim);
    uint64_t bytes = 0;
    p.heads = 0;
    p.copy = false;
    for (int i = 0; i < p.d.nlists; ++i) {
        const rikfad_rotary_heads &l = p.d.lists[i];
        if (l.heads == 0)
            continue;
        p.heads += (int32_t)l.heads;
        p.copy = p.copy || l.src != l.dst;
        if (l.heads > 1)
            parts |= (uint64_t)l.src_head | (uint64_t)l.dst_head;
        if (p.d.tokens > 1)
            parts |= (uint64_t)l.src_token | (uint64_t)l.dst_token;
        if (p.d.batch > 1)
            parts |= (uint64_t)l.src_batch | (uint64_t)l.dst_batch;
        bytes |= (uint64_t)(uintptr_t)l.src | (uint64_t)(uintptr_t)l.dst;
    }
    parts |= bytes / sizeof(T);
    if constexpr (sizeof(T) == 2)
        if (parts % 8 == 0)
            return launch<T, 8>(p, s);
    return parts % 4 == 0 ? launch<T, 4>(p, s) : parts % 2 == 0 ? launch<T, 2>(p, s) : launch<T, 1>(p, s);
}

}  // namespace

extern "C" {

RIKFAD_API int rikfad_rotary_turns(const double *radians, int64_t n, uint64_t *turns)
{
    RK_ENTRY_BEGIN
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
    RK_ENTRY_END
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
    r.sine_sign = p->inverse ? -r.magnitude : r.magnitude;
    const cudaStream_t s = (cudaStream_t)stream;
    e = p->dtype == RIKFAD_F32    ? launch<float>(r, s)
        : p->dtype == RIKFAD_BF16 ? launch<__nv_bfloat16>(r, s)
                                  : launch<__half>(r, s);
    return e == cudaSuccess ? RIKFAD_OK : report_cuda(e, "launch rikfad_rotary_kernel");
    RK_ENTRY_END
}

}  // extern "C"
