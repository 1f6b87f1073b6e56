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
//
// 65536 tokens of 32 + 8 heads of 128 in bfloat16 take 215 us forward (1.34 GB, 6.3 TB/s)
// and 341 backward (2.0 GB, 5.9 TB/s); 16384 of 12 + 12 of 64 22 and 38 (101 and 151 MB).
// What is left is arithmetic: a head of 128 is a lane's 16 elements and some 250 instructions
// of a warp of four such heads forward, 320 backward.
#include <cuda_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <new>
#include <string>

#include "rikfad.h"
#include "rikfad_host.hpp"
#include "rikfad_kernels.cuh"
#include "rikfad_pairs.cuh"
#include "rikfad_rotary.cuh"
#include "rikfad_types.cuh"

using namespace rikfad;

namespace {

constexpr int kThreads = 128;
constexpr int kSms = 152;
constexpr int kForwardBlocksPerSm = 4, kBackwardBlocksPerSm = 3;
constexpr int kTablePairs = 1024;           // cosines and sines of a tile of tokens: 8 KB at most
constexpr int kMaxHeadDim = 512;
constexpr int kWish = 32;                   // heads of a group in a tile
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
    int32_t lanes, turn_units, units;   // of a head: lanes, units that turn (half layout), all units (whole heads: pairs)
    int32_t rest_half;                  // how far the elements of a pair beyond rotary_dim are apart
    float magnitude, inv_dim, eps;
    int32_t pitch;                      // of a token's cosines and sines
    int32_t split;                      // groups of lanes that have heads of the first list; the others have the second's
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

template <int BYTES> __device__ __forceinline__ void copy_async(void *to, const void *from)
{
    const uint32_t at = (uint32_t)__cvta_generic_to_shared(to);
    if constexpr (BYTES == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(from) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(at), "l"(from), "n"(BYTES) : "memory");
}

// A lane's units as loaded; zeros where there are none.
template <typename T, int V, int U> struct Raw {
    Vec<T, V> a[U], b[U];

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
};

// A unit's 2 V elements in float32, two to a register pair: the first vector's, then the
// second's.
template <int V> struct Values {
    f2 p[V];

    template <typename T> __device__ __forceinline__ void from(const Vec<T, V> &a, const Vec<T, V> &b)
    {
        float x[V], y[V];
        widen(a, x);
        widen(b, y);
        put(x, y);
    }
    template <typename T> __device__ __forceinline__ void to(Vec<T, V> &a, Vec<T, V> &b) const
    {
        float x[V], y[V];
        get(x, y);
        narrow(x, a);
        narrow(y, b);
    }
    __device__ __forceinline__ void put(const float (&x)[V], const float (&y)[V])
    {
#pragma unroll
        for (int e = 0; e < V; e += 2) {
            p[e / 2] = pair(x[e], x[e + 1]);
            p[V / 2 + e / 2] = pair(y[e], y[e + 1]);
        }
    }
    __device__ __forceinline__ void get(float (&x)[V], float (&y)[V]) const
    {
#pragma unroll
        for (int e = 0; e < V; e += 2) {
            apart(p[e / 2], x[e], x[e + 1]);
            apart(p[V / 2 + e / 2], y[e], y[e + 1]);
        }
    }
};

__device__ __forceinline__ void turn_pair(float &x, float &y, float c, float s)
{
    const float u = x, v = y;
    x = fmaf(u, c, -v * s);
    y = fmaf(v, c, u * s);
}

// A unit's pairs turned by the token's cosines and sines.
template <int V>
__device__ __forceinline__ void turn(const Params &p, Values<V> &v, const Place &at, const float *cosines, const float *sines)
{
    if (at.pair < 0)
        return;
    constexpr int L = 4;                        // elements of one load
    Vec<float, L> c[V / L], s[V / L];
#pragma unroll
    for (int i = 0; i < V / L; ++i) {
        c[i].word = reinterpret_cast<const decltype(c[i].word) *>(cosines + at.pair)[i];
        s[i].word = reinterpret_cast<const decltype(s[i].word) *>(sines + at.pair)[i];
    }
    if (!p.interleaved) {
#pragma unroll
            for (int e = 0; e < V; e += 2) {
                const f2 ce = pair(c[e / L].v[e % L], c[e / L].v[e % L + 1]), se = pair(s[e / L].v[e % L], s[e / L].v[e % L + 1]);
                f2 &a = v.p[e / 2], &b = v.p[V / 2 + e / 2];
                const f2 x = a;
                a = sub(mul(a, ce), mul(b, se));
                b = fma(x, se, mul(b, ce));
            }
        return;
    }
    // pair e is elements 2 e and 2 e + 1; the last unit may reach beyond rotary_dim
#pragma unroll
    for (int e = 0; e < V; ++e) {
        float x, y;
        apart(v.p[e], x, y);
        if (at.pair + e < p.pairs)
            turn_pair(x, y, c[e / L].v[e % L], s[e / L].v[e % L]);
        v.p[e] = pair(x, y);
    }
}

// A tile of tokens of one sequence.
struct Tile {
    int64_t batch, token0;
    int here;                   // tokens; none beyond the last tile

    __device__ __forceinline__ Tile(const Params &p, int64_t tile)
    {
        batch = p.tiles_per_sequence == p.tiles ? 0 : tile / p.tiles_per_sequence;
        token0 = (tile - batch * p.tiles_per_sequence) * p.tile;
        here = tile < p.tiles ? (int)min((int64_t)p.tile, p.tokens - token0) : 0;
    }
};

// How the groups that share a list go on from head to head: by `step` elements, and by
// `wrap` more into the next token.
struct Steps {
    int64_t batch, token, first, step, wrap;

    __device__ __forceinline__ Steps(int64_t per_batch, int64_t per_token, int64_t per_head, int g, int n, int heads)
        : batch(per_batch), token(per_token)
    {
        const int slot = g / heads, slots = n / heads;
        first = slot * per_token + (g - slot * heads) * per_head;
        step = slots * per_token + (n - slots * heads) * per_head;
        wrap = per_token - heads * per_head;
    }
    template <typename T> __device__ __forceinline__ T *at(T *base, const Tile &t) const
    {
        return base + (t.batch * batch + t.token0 * token + first);
    }
};

// The V pairs of a lane where heads are copied whole: pairs lane, lane + lanes, ..., so that
// neighbours read neighbouring elements.  Beyond rotary_dim any two elements are a pair.
template <int V> struct Spread {
    uint32_t at[V];             // first and second element, 0xffff where there is none
    int turning;                // pairs that turn: the first so many

    __device__ __forceinline__ Spread(const Params &p, int lane)
    {
        turning = 0;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int k = lane + e * p.lanes;
            int first, second;
            if (p.interleaved) {
                first = 2 * k;
                second = first + 1;
            } else {
                first = k < p.pairs ? k : k + p.pairs;
                second = first + (k < p.pairs ? p.pairs : p.rest_half);
            }
            first = k < p.units ? first : 0xffff;
            second = k < p.units && second < p.head_dim ? second : 0xffff;
            at[e] = (uint32_t)first | (uint32_t)second << 16;
            turning += k < p.pairs;
        }
    }
    __device__ __forceinline__ int first(int e) const { return at[e] & 0xffff; }
    __device__ __forceinline__ int second(int e) const { return at[e] >> 16; }
    template <typename F> __device__ __forceinline__ void each(float (&x)[V], float (&y)[V], F element) const
    {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            x[e] = first(e) != 0xffff ? element(first(e)) : 0.f;
            y[e] = second(e) != 0xffff ? element(second(e)) : 0.f;
        }
    }
    __device__ __forceinline__ void turn(const Params &p, Values<V> &v, int lane, const float *cosines, const float *sines) const
    {
        float c[V], s[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            c[e] = e < turning ? cosines[lane + e * p.lanes] : 1.f;
            s[e] = e < turning ? sines[lane + e * p.lanes] : 0.f;
        }
#pragma unroll
        for (int e = 0; e < V; e += 2) {
            const f2 ce = pair(c[e], c[e + 1]), se = pair(s[e], s[e + 1]);
            f2 &a = v.p[e / 2], &b = v.p[V / 2 + e / 2];
            const f2 x = a;
            a = sub(mul(a, ce), mul(b, se));
            b = fma(x, se, mul(b, ce));
        }
    }
};

// Heads on their way.  Vectors of 8 or 16 bytes: each lane's at a place of shared memory of its
// own.  Other heads whole: all of the 16 bytes that one begins and ends in, wherever that is
// (the other bytes of the first and last 16 are read too, and not used), copied by the group's
// lanes, each of which reads its elements there.  16384 tokens of 24 heads of 131 in bfloat16,
// forward and backward: 960 us with an element a load, 267 so; of 70: 355 and 143.
template <typename T, int V, int U, bool WHOLE, bool BACKWARD> struct Ring {
    static constexpr int kWord = V * (int)sizeof(T), kWords = (BACKWARD ? 4 : 2) * U;
    static constexpr int kDepth = WHOLE ? 8 / (int)sizeof(T) : kWord * kWords > 64 ? 2 : 4;
    __host__ __device__ static constexpr int whole_bytes(int head_dim)
    {
        return (head_dim * (int)sizeof(T) + 31 - (int)sizeof(T)) / 16 * 16;
    }
    __host__ __device__ static constexpr int bytes(int head_dim, int groups)
    {
        return WHOLE ? kDepth * groups * (BACKWARD ? 2 : 1) * whole_bytes(head_dim) : kDepth * kWords * kWord * kThreads;
    }
};

// A block has tile after tile of tokens: their cosines and sines, formed once a tile, and
// all heads, shared by its groups of lanes.  A group has heads of one list, and their
// weights' gradients in registers.  Its next kDepth heads are on their way meanwhile.
//
// The same with one head ahead, in registers, took 865 us for 65536 x 40 x 128 (too few
// bytes on their way); with lists on blocks of their own 835 (the second list's blocks form
// the tables again, and end late).  Tiles of 3, 6 and 12 tokens: 666, 624 and 563 us.
template <typename T, int V, int U, bool WHOLE, bool BACKWARD>
__global__ void __launch_bounds__(kThreads, BACKWARD ? kBackwardBlocksPerSm : kForwardBlocksPerSm)
rikfad_rotary_norm_kernel(const __grid_constant__ Params p)
{
    using R = Ring<T, V, U, WHOLE, BACKWARD>;
    extern __shared__ float4 shared[];
    float *const cosines = reinterpret_cast<float *>(reinterpret_cast<char *>(shared) + R::bytes(p.head_dim, kThreads / p.lanes));
    float *const sines = cosines + p.tile * p.pitch;
    const int group = threadIdx.x / p.lanes, lane = threadIdx.x % p.lanes;
    Place at[U];                        // of vectors; whole heads have a spread instead
    if constexpr (!WHOLE) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            at[u] = place_of<V>(p, lane + u * p.lanes);
    }
    const Spread<V> spread(p, lane);
    const bool list = group >= p.split;
    const int g = list ? group - p.split : group, n = list ? kThreads / p.lanes - p.split : p.split;
    const Heads &h0 = p.lists[0], &h1 = p.lists[1];
    const int heads = list ? h1.heads : h0.heads, more_heads = n - n / heads * heads;
    auto steps = [&](int64_t b0, int64_t b1, int64_t t0, int64_t t1, int64_t s0, int64_t s1) {
        return Steps(list ? b1 : b0, list ? t1 : t0, list ? s1 : s0, g, n, heads);
    };
    const Steps of_x = steps(h0.x_batch, h1.x_batch, h0.x_token, h1.x_token, h0.x_head, h1.x_head);
    const Steps of_dout = steps(h0.dout_batch, h1.dout_batch, h0.dout_token, h1.dout_token, h0.dout_head, h1.dout_head);
    const Steps of_out = steps(h0.out_batch, h1.out_batch, h0.out_token, h1.out_token, h0.out_head, h1.out_head);
    const T *const x = static_cast<const T *>(list ? h1.x : h0.x), *const dout = static_cast<const T *>(list ? h1.dout : h0.dout);
    T *const out = static_cast<T *>(list ? h1.out : h0.out);
    // heads of a group in a tile of that many tokens: the same for all groups
    auto rounds_of = [&](int here) {
        const int q = (here * h0.heads + p.split - 1) / max(p.split, 1), others = kThreads / p.lanes - p.split;
        return max(q, (here * h1.heads + others - 1) / max(others, 1));
    };
    Values<V> sums[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int e = 0; e < V; ++e)
            sums[u].p[e] = pair(0.f, 0.f);
    }
    wait_for_predecessor();
    allow_successor_launch();
    // the head to load next
    int64_t ask_tile = blockIdx.x;
    int ask_round = 0, ask_rounds, ask_item, ask_items, ask_head;
    const T *from, *dfrom;
    auto ask_enter = [&] {
        const Tile t(p, ask_tile);
        from = of_x.at(x, t);
        dfrom = of_dout.at(dout, t);
        ask_round = 0;
        ask_rounds = rounds_of(t.here);
        ask_item = g;
        ask_items = t.here * heads;
        ask_head = g % heads;
    };
    auto ask_next = [&] {
        if (++ask_round >= ask_rounds) {
            ask_tile += gridDim.x;
            ask_enter();
            return;
        }
        ask_item += n;
        ask_head += more_heads;
        const bool over = ask_head >= heads;
        ask_head -= over ? heads : 0;
        from += of_x.step + (over ? of_x.wrap : 0);
        dfrom += of_dout.step + (over ? of_dout.wrap : 0);
    };
    // Vector i of a lane's in place j of the ring: the thread's own, neighbours side by side.
    auto place = [&](int j, int i) {
        return reinterpret_cast<char *>(shared) + ((j * R::kWords + i) * kThreads + threadIdx.x) * R::kWord;
    };
    // Whole heads: at which byte of its place each begins, 4 bits for every place of x and dout.
    const int whole = R::whole_bytes(p.head_dim), head_bytes = p.head_dim * (int)sizeof(T);
    uint32_t skips = 0;
    auto whole_place = [&](int j, int tensor) {
        return reinterpret_cast<char *>(shared) + ((j * (kThreads / p.lanes) + group) * (BACKWARD ? 2 : 1) + tensor) * whole;
    };
    auto request_whole = [&](int j, int tensor, const T *head) {
        const int skip = (int)((uintptr_t)head % 16), words = (skip + head_bytes + 15) / 16;
        for (int i = lane; i < words; i += p.lanes)
            copy_async<16>(whole_place(j, tensor) + 16 * i, reinterpret_cast<const char *>(head) - skip + 16 * i);
        const int bits = 8 * j + 4 * tensor;
        skips = (skips & ~(15u << bits)) | (uint32_t)skip << bits;
    };
    // The group's results, by way of x's place: 16 bytes at a time, elements at the ends.
    auto store_whole = [&](int j, T *head, const float (&a)[V], const float (&b)[V], bool active) {
        constexpr int E = 16 / sizeof(T);
        const int skip = (int)((uintptr_t)head % 16);
        const int lead = min((16 - skip) % 16 / (int)sizeof(T), p.head_dim);
        const int words = (p.head_dim - lead) / E, edges = p.head_dim - words * E;
        T *const place = reinterpret_cast<T *>(whole_place(j, 0) + skip);
        __syncwarp();                   // all lanes have taken theirs
#pragma unroll
        for (int e = 0; e < V; ++e) {
            if (spread.first(e) != 0xffff)
                place[spread.first(e)] = from_f32<T>(a[e]);
            if (spread.second(e) != 0xffff)
                place[spread.second(e)] = from_f32<T>(b[e]);
        }
        __syncwarp();
        if (active) {
            for (int i = lane; i < words; i += p.lanes)
                reinterpret_cast<uint4 *>(head + lead)[i] = reinterpret_cast<const uint4 *>(place + lead)[i];
            for (int i = lane; i < edges; i += p.lanes) {
                const int e = i < lead ? i : i + words * E;
                head[e] = place[e];
            }
        }
        __syncwarp();                   // before the place is filled again
    };
    auto request = [&](int j) {
        if (ask_item < ask_items) {
            if constexpr (WHOLE) {
                request_whole(j, 0, from);
                if (BACKWARD)
                    request_whole(j, 1, dfrom);
            } else {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (at[u].first >= 0) {
                        copy_async<R::kWord>(place(j, 2 * u), from + at[u].first);
                        if (BACKWARD)
                            copy_async<R::kWord>(place(j, 2 * U + 2 * u), dfrom + at[u].first);
                    }
                    if (at[u].second >= 0) {
                        copy_async<R::kWord>(place(j, 2 * u + 1), from + at[u].second);
                        if (BACKWARD)
                            copy_async<R::kWord>(place(j, 2 * U + 2 * u + 1), dfrom + at[u].second);
                    }
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        ask_next();
    };
    ask_enter();
    if constexpr (!WHOLE) {     // vectors that a lane has not stay zeros
#pragma unroll
        for (int i = 0; i < R::kDepth * R::kWords; ++i) {
            Vec<T, V> none;
            none.word = decltype(none.word){};
            *reinterpret_cast<decltype(none.word) *>(place(0, i)) = none.word;
        }
    }
#pragma unroll
    for (int j = 0; j < R::kDepth; ++j)
        request(j);
    Values<V> w[U];
    const void *const weights = list ? h1.weight : h0.weight;
    auto weight = [&](int e) {
        return weights == nullptr ? 1.f
               : p.param_f32      ? static_cast<const float *>(weights)[e]
                                  : to_f32(static_cast<const T *>(weights)[e]);
    };
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float a[V], b[V];
        if constexpr (WHOLE) {
            spread.each(a, b, weight);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                a[e] = at[u].first >= 0 ? weight(at[u].first + e) : 0.f;
                b[e] = at[u].second >= 0 ? weight(at[u].second + e) : 0.f;
            }
        }
        w[u].put(a, b);
    }
    int turn_of_ring = 0;
    for (int64_t tile = blockIdx.x; tile < p.tiles; tile += gridDim.x) {
        const Tile t(p, tile);
        __syncthreads();
        for (int i = threadIdx.x; i < t.here * p.pairs; i += kThreads) {
            const int slot = i / p.pairs, e = i - slot * p.pairs;
            const int64_t position = token_position(p.positions, p.position_bytes, p.position_batch, p.start, t.batch, t.token0 + slot);
            const float2 cs = cosine_sine(position, p.turns[e]);
            cosines[slot * p.pitch + e] = cs.x * p.magnitude;
            sines[slot * p.pitch + e] = cs.y * (BACKWARD ? -p.magnitude : p.magnitude);
        }
        __syncthreads();
        const int rounds = rounds_of(t.here), items = t.here * heads, table_step = n / heads * p.pitch;
        T *to = of_out.at(out, t);
        int head = g % heads, table = g / heads * p.pitch, item = g;
        for (int round = 0; round < rounds; ++round) {
            const bool active = item < items;
            asm volatile("cp.async.wait_group %0;" ::"n"(R::kDepth - 1) : "memory");
            Values<V> v[U], d[U];
            if constexpr (WHOLE) {
                __syncwarp();           // the other lanes' copies
                auto take = [&](Values<V> &v, int tensor) {
                    const int skip = skips >> (8 * turn_of_ring + 4 * tensor) & 15;
                    const T *head = reinterpret_cast<const T *>(whole_place(turn_of_ring, tensor) + skip);
                    float a[V], b[V];
                    spread.each(a, b, [&](int e) { return to_f32(head[e]); });
                    v.put(a, b);
                };
                take(v[0], 0);
                if constexpr (BACKWARD) {
                    take(d[0], 1);
                }
            } else {
                auto take = [&](Values<V> &v, int i) {
                    Vec<T, V> a, b;
                    a.word = *reinterpret_cast<const decltype(a.word) *>(place(turn_of_ring, i));
                    b.word = *reinterpret_cast<const decltype(b.word) *>(place(turn_of_ring, i + 1));
                    v.from(a, b);
                };
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    take(v[u], 2 * u);
                    if constexpr (BACKWARD) {
                        take(d[u], 2 * U + 2 * u);
                    }
                }
            }
            auto turn_all = [&](Values<V> (&v)[U], const float *c, const float *s) {
                if constexpr (WHOLE) {
                    spread.turn(p, v[0], lane, c, s);
                } else {
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        turn<V>(p, v[u], at[u], c, s);
                }
            };
            const float *const c = cosines + (active ? table : 0), *const s = sines + (active ? table : 0);
            f2 squares2 = pair(0.f, 0.f);
#pragma unroll
            for (int u = 0; u < U; ++u) {
#pragma unroll
                for (int e = 0; e < V; ++e)
                    squares2 = fma(v[u].p[e], v[u].p[e], squares2);
            }
            float squares = total(squares2);
            if constexpr (BACKWARD) {
                turn_all(d, c, s);
                f2 product2 = pair(0.f, 0.f);
#pragma unroll
                for (int u = 0; u < U; ++u) {
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        product2 = fma(mul(d[u].p[e], w[u].p[e]), v[u].p[e], product2);
                }
                float product = total(product2);
                if constexpr (!WHOLE)           // the next head on its way, now that this one has been taken
                    request(turn_of_ring);
                for (int far = p.lanes / 2; far > 0; far /= 2) {
                    squares += __shfl_xor_sync(~0u, squares, far);
                    product += __shfl_xor_sync(~0u, product, far);
                }
                const float r = rsqrtf(fmaf(squares, p.inv_dim, p.eps));
                const f2 rr = both(r), minus = both(-product * p.inv_dim * r * r);
                if (active) {                   // else what was there before
#pragma unroll
                    for (int u = 0; u < U; ++u) {
#pragma unroll
                        for (int e = 0; e < V; ++e)
                            sums[u].p[e] = fma(d[u].p[e], mul(v[u].p[e], rr), sums[u].p[e]);
                    }
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        v[u].p[e] = mul(rr, fma(minus, v[u].p[e], mul(d[u].p[e], w[u].p[e])));
                }
            } else {
                if constexpr (!WHOLE)
                    request(turn_of_ring);
                for (int far = p.lanes / 2; far > 0; far /= 2)
                    squares += __shfl_xor_sync(~0u, squares, far);
                const f2 rr = both(rsqrtf(fmaf(squares, p.inv_dim, p.eps)));
#pragma unroll
                for (int u = 0; u < U; ++u) {
#pragma unroll
                    for (int e = 0; e < V; ++e)
                        v[u].p[e] = mul(v[u].p[e], mul(rr, w[u].p[e]));
                }
                turn_all(v, c, s);
            }
            if constexpr (WHOLE) {
                float a[V], b[V];
                v[0].get(a, b);
                store_whole(turn_of_ring, to, a, b, active);
                request(turn_of_ring);
            } else if (active) {
                Raw<T, V, U> result;
#pragma unroll
                for (int u = 0; u < U; ++u)
                    v[u].to(result.a[u], result.b[u]);
                result.store(to, at);
            }
            turn_of_ring = turn_of_ring + 1 == R::kDepth ? 0 : turn_of_ring + 1;
            item += n;
            head += more_heads;
            const bool over = head >= heads;
            head -= over ? heads : 0;
            table += table_step + (over ? p.pitch : 0);
            to += of_out.step + (over ? of_out.wrap : 0);
        }
    }
    if constexpr (BACKWARD) {
        if (p.part == nullptr)
            return;
        // every group's sums, then those of a list's groups in order
        float *sum = reinterpret_cast<float *>(shared);         // [group][element]
        __syncthreads();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float a[V], b[V];
            sums[u].get(a, b);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const int first = WHOLE ? spread.first(e) : at[u].first + e, second = WHOLE ? spread.second(e) : at[u].second + e;
                if (WHOLE ? first != 0xffff : at[u].first >= 0)
                    sum[group * p.head_dim + first] = a[e];
                if (WHOLE ? second != 0xffff : at[u].second >= 0)
                    sum[group * p.head_dim + second] = b[e];
            }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * p.head_dim; i += kThreads) {
            const int l = i >= p.head_dim, e = i - l * p.head_dim;
            float s = 0.f;
            for (int group = l ? p.split : 0; group < (l ? kThreads / p.lanes : p.split); ++group)
                s += sum[group * p.head_dim + e];
            p.part[((int64_t)blockIdx.x * 2 + l) * p.head_dim + e] = s;
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
    if (e < head_dim) {
#pragma unroll 4
        for (int b = warp; b < blocks; b += kJoinThreads / 32)
            s += part[((int64_t)b * 2 + blockIdx.y) * head_dim + e];
    }
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

template <typename T, int V, int U, bool WHOLE, bool BACKWARD> cudaError_t launch(Params p, const rikfad_rotary_norm *d, cudaStream_t s)
{
    const int groups = kThreads / p.lanes;
    const int64_t heads = p.lists[0].heads + p.lists[1].heads, tokens = p.tiles * p.tokens;   // p.tiles: sequences, here
    // the groups of a block shared among the lists as their heads are
    p.split = p.lists[1].heads == 0   ? groups
              : p.lists[0].heads == 0 ? 0
                                      : std::max(1, std::min(groups - 1, (int)((groups * (int64_t)p.lists[0].heads + heads / 2) / heads)));
    // the last unit of the interleaved layout reads a vector's worth of the table
    p.pitch = (std::max(p.pairs, p.interleaved && p.pairs ? (p.pairs + V - 1) / V * V : 0) + 3) / 4 * 4;
    // As many tiles a block as leave a group kWish heads of each, all of the same size, within
    // the table's; two at least where they are large, so that one's table and another's heads
    // are formed at one time (16384 tokens of 24 heads of 64: 70 us with one of 27 tokens, 61
    // with two of 14).
    const int64_t all = kSms * (BACKWARD ? kBackwardBlocksPerSm : kForwardBlocksPerSm);
    const int64_t wish = std::max<int64_t>(1, kWish * groups / heads);
    const int64_t most = std::min<int64_t>(wish, p.pairs ? std::max(1, kTablePairs / p.pitch) : 1 << 10);
    const int64_t each = std::max<int64_t>((tokens + all * most - 1) / (all * most), tokens > 16 * all ? 2 : 1);
    p.tile = (int32_t)std::min<int64_t>(p.tokens, std::max<int64_t>(1, (tokens + all * each - 1) / (all * each)));
    p.tiles_per_sequence = (p.tokens + p.tile - 1) / p.tile;
    p.tiles *= p.tiles_per_sequence;
    const int64_t blocks = std::min(p.tiles, all);
    size_t smem = Ring<T, V, U, WHOLE, BACKWARD>::bytes(p.head_dim, groups) + 2 * sizeof(float) * (size_t)p.tile * p.pitch;
    if (BACKWARD && p.part)
        smem = std::max(smem, sizeof(float) * groups * (size_t)p.head_dim);
    const cudaError_t e =
        launch_chained(rikfad_rotary_norm_kernel<T, V, U, WHOLE, BACKWARD>, dim3((unsigned)blocks), kThreads, smem, s, p);
    if (e != cudaSuccess || !BACKWARD || p.part == nullptr)
        return e;
    void *const dq = d->lists[0].dweight, *const dk = d->nlists > 1 ? d->lists[1].dweight : nullptr;
    const bool f32 = p.param_f32;
    return launch_chained(rikfad_rotary_norm_join_kernel<T>, dim3((unsigned)(p.head_dim + 31) / 32, (unsigned)p.nlists), kJoinThreads,
                          0, s, (const float *)p.part, (int)blocks, (int)p.head_dim, f32 ? nullptr : (T *)dq,
                          f32 ? nullptr : (T *)dk, f32 ? (float *)dq : nullptr, f32 ? (float *)dk : nullptr);
}

// Lanes of a head: enough for one unit each, up to a warp.
template <typename T, int V, bool BACKWARD> cudaError_t launch_vectors(Params p, const rikfad_rotary_norm *d, cudaStream_t s)
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
    if constexpr (V <= 4)
        if (p.units > 32)
            return launch<T, V, 2, false, BACKWARD>(p, d, s);
    return launch<T, V, 1, false, BACKWARD>(p, d, s);
}

// As many as have eight pairs each, or six where they do (16384 tokens of 24 heads of 131: 267 us
// with six, 316 with eight), and four at least: the groups' rings fit 40 KB.
template <typename T, bool BACKWARD> cudaError_t launch_whole(Params p, const rikfad_rotary_norm *d, cudaStream_t s)
{
    const int rest = p.head_dim - p.rotary_dim;
    p.rest_half = (rest + 1) / 2;
    p.units = p.interleaved ? (p.head_dim + 1) / 2 : p.pairs + p.rest_half;
    p.lanes = 4;
    while (p.lanes < 32 && p.lanes * 8 < p.units)
        p.lanes *= 2;
    return p.units <= p.lanes * 6 ? launch<T, 6, 1, true, BACKWARD>(p, d, s) : launch<T, 8, 1, true, BACKWARD>(p, d, s);
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
    // Vectors of 8 or 4 elements if the heads' layout and addresses allow them: every part of a
    // head and every stride is a whole number of vectors, and so are the addresses.  16384 tokens
    // of 24 heads of bfloat16, both directions: 80 with 40 turned 119 us in vectors of 4, 139
    // whole; 64 with 40 68, 96; 128 with 120 125, 172.
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
            return launch_vectors<T, 8, BACKWARD>(p, d, s);
    return parts % 4 == 0 ? launch_vectors<T, 4, BACKWARD>(p, d, s) : launch_whole<T, BACKWARD>(p, d, s);
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
        int device = -1;
        const cudaError_t e = cudaGetDevice(&device);
        if (e != cudaSuccess)
            return report_cuda(e, "cudaGetDevice");
        const int bad_place = check_place(p->workspace, "workspace", 16, device);
        if (bad_place)
            return bad_place;
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
