// Host-side check of the residual norm's launches: the C entries' host code with the
// kernels' launches replaced by a look at the parameters they would get and the CUDA
// runtime by host memory (tests/host_runtime.cpp).  Compiled by
// tests/test_norm_launch.py; the argument names the check.  Prints "OK" or the first
// violation.
//
//   copies  every 16-byte asynchronous copy, those of no bytes too, starts on 16 bytes
//   shapes  every width at every drift of its rows has a launch that the kernels run
#include "rikfad_norm.cu"

#include <cstdio>
#include <cstring>

static NormParams g_launched;
static int g_launches = 0;
static std::string g_error;

namespace rikfad {

int report_error(int code, const std::string &msg)
{
    g_error = msg;
    return code;
}
int check_address(const void *, int, const char *, int64_t) { return RIKFAD_OK; }

static cudaError_t look(const NormParams &n)
{
    g_launched = n;
    ++g_launches;
    return cudaSuccess;
}
#define STUB(name) \
    cudaError_t norm_forward_##name(const NormParams &n, cudaStream_t) { return look(n); } \
    cudaError_t norm_backward_##name(const NormParams &n, cudaStream_t) { return look(n); }
STUB(f32_f32)
STUB(bf16_bf16)
STUB(bf16_f32)
STUB(f16_f16)
STUB(f16_f32)

}  // namespace rikfad

static uint64_t g_random = 88172645463325252ull;
static int64_t below(int64_t n)
{
    g_random ^= g_random << 13;
    g_random ^= g_random >> 7;
    g_random ^= g_random << 17;
    return (int64_t)(g_random % (uint64_t)n);
}
static bool chance() { return below(2); }

// A tensor somewhere of its own: on 16 bytes or `offset` elements beyond.
static rikfad_rows somewhere(int which, int64_t stride, int dtype, int64_t offset)
{
    return {reinterpret_cast<void *>(((uintptr_t)(which + 1) << 40) + (uintptr_t)(offset * dtype_bytes(dtype))), stride};
}

static int fail(const rikfad_residual_norm &p, const char *what, long long a, long long b)
{
    std::printf("FAIL %s (%lld, %lld): rows %lld cols %lld gate_rows %lld dtypes %d %d\n", what, a, b, (long long)p.rows,
                (long long)p.cols, (long long)p.gate_rows, p.dtype, p.residual_dtype);
    return 1;
}

// A random call: tensors dense or in wider rows, aligned or not, some absent.
static rikfad_residual_norm draw(bool backward)
{
    rikfad_residual_norm p{};
    p.dtype = (int)below(3);
    p.residual_dtype = chance() ? RIKFAD_F32 : p.dtype;
    p.gate_dtype = chance() ? RIKFAD_F32 : p.dtype;
    p.param_dtype = chance() ? RIKFAD_F32 : p.dtype;
    p.cols = below(4) ? 1 + below(2048) : 1 + below(32768);
    const int64_t few[] = {1, 1, 2, 3, 15, 16, 17, 600};
    p.gate_rows = few[below(8)];
    p.rows = p.gate_rows * (1 + below(3000));
    p.post_eps = p.pre_eps = 1e-6;
    p.post = (int)below(3);
    p.pre = (int)below(3);
    const bool z = below(4) || p.post, dense = below(3), drift = chance();
    const int64_t pad = below(10);
    auto tensor = [&](int which, int dtype) {
        const int64_t stride = p.cols + (dense ? 0 : drift ? pad : below(10));
        return somewhere(which, stride, dtype, below(8) ? 0 : below(16));
    };
    p.x = tensor(0, p.residual_dtype);
    if (z) p.z = tensor(1, p.dtype);
    if (z && chance()) p.gate = tensor(2, p.gate_dtype);
    void *const vec = reinterpret_cast<void *>((uintptr_t)1 << 50);
    p.stats = static_cast<float *>(vec);
    if (p.pre && chance()) p.pre_weight = vec;
    if (p.pre && chance()) p.pre_bias = vec;
    if (p.post && chance()) p.post_weight = vec;
    if (p.post && chance()) p.post_bias = vec;
    if (!backward) {
        if (below(4)) p.u = tensor(3, p.residual_dtype);
        if (below(4)) p.h = tensor(4, p.dtype);
        return p;
    }
    if (chance()) p.du = tensor(5, p.residual_dtype);
    if (chance()) p.dh = tensor(6, p.dtype);
    if (below(4)) p.dx = tensor(7, p.residual_dtype);
    if (z && below(4)) p.dz = tensor(8, p.dtype);
    if (p.gate.data && below(4)) p.dgate = tensor(9, p.gate_dtype);
    if (p.pre_weight && chance()) p.dpre_weight = vec;
    if (p.pre_bias && chance()) p.dpre_bias = vec;
    if (p.post_weight && chance()) p.dpost_weight = vec;
    if (p.post_bias && chance()) p.dpost_bias = vec;
    return p;
}

// Launches p; its workspace is as large as the query says.
static int run(rikfad_residual_norm &p, bool backward)
{
    if (!backward)
        return rikfad_residual_norm_forward(&p, nullptr);
    p.workspace_bytes = rikfad_residual_norm_workspace(&p);
    p.workspace = reinterpret_cast<void *>((uintptr_t)1 << 51);
    return rikfad_residual_norm_backward(&p, nullptr);
}

// The kernels' copies of a row start at its first column less the class's shift (a
// whole number of vectors on), in every class.  An absent gradient's copies of no
// bytes start where x's do.
static int check_copies(const rikfad_residual_norm &p, const NormParams &n, bool backward)
{
    const int a = dtype_bytes(p.dtype), r = dtype_bytes(p.residual_dtype), g = dtype_bytes(p.gate_dtype);
    const struct {
        const NormRows *rows;
        uint32_t wide;
        int bytes;
        bool gate;
    } all[] = {{&n.x, kNormWideX, r, false}, {&n.z, kNormWideZ, a, false}, {&n.gate, kNormWideGate, g, true},
               {&n.u, kNormWideU, r, false}, {&n.h, kNormWideH, a, false}, {&n.du, kNormWideDu, r, false},
               {&n.dh, kNormWideDh, a, false}, {&n.dx, kNormWideDx, r, false}, {&n.dz, kNormWideDz, a, false},
               {&n.dgate, kNormWideDgate, g, true}};
    for (const auto &t : all) {
        if (!(t.wide & n.wide))
            continue;
        const bool gradient = t.rows == &n.du || t.rows == &n.dh;
        if (t.rows->data == nullptr && !(backward && gradient))
            continue;               // absent: no copy
        const NormRows &at = t.rows->data ? *t.rows : n.x;
        const int bytes = t.rows->data ? t.bytes : r;
        const bool shared = t.gate && n.gate_rows > 1;
        if (shared && n.classes > 1)
            return fail(p, "wide rows of a shared gate in classes", t.wide, n.classes);
        const int64_t rows = shared ? n.rows / n.gate_rows : n.rows;
        for (int64_t row = 0; row < std::min<int64_t>(rows, 17); ++row) {
            const int64_t shift = row % n.classes * n.drift % 8;
            const uintptr_t from = (uintptr_t)at.data + (uintptr_t)((row * at.stride - shift) * bytes);
            if (from % 16)
                return fail(p, "a copy that does not start on 16 bytes", t.wide, row);
        }
    }
    return 0;
}

static int copies()
{
    for (int i = 0; i < 400000; ++i) {
        const bool backward = below(3) > 0;
        rikfad_residual_norm p = draw(backward);
        const int before = g_launches;
        if (run(p, backward) || g_launches != before + 1)
            return fail(p, g_error.c_str(), i, 0);
        if (check_copies(p, g_launched, backward))
            return 1;
    }
    return 0;
}

// What the kernels take: up to 8 blocks of a cluster of up to 16 warps each, whole
// rows of a warp or warps of a row, and columns for every element of a row wherever
// it starts.
static int check_shape(const rikfad_residual_norm &p, const NormParams &n)
{
    if (n.cluster != 1 && n.cluster != 2 && n.cluster != 4 && n.cluster != 8)
        return fail(p, "blocks of a cluster", n.cluster, n.drift);
    if (n.threads < 32 || n.threads > kNormMaxThreads || n.threads % 32 || n.threads > n.threads_per_sm)
        return fail(p, "threads of a block", n.threads, n.threads_per_sm);
    if (n.row_groups * n.lanes != n.threads || (n.lanes < 32 ? 32 % n.lanes : n.lanes % 32) ||
        (n.row_groups > 1 && (n.lanes > 32 || n.cluster > 1)))
        return fail(p, "lanes of a row", n.lanes, n.row_groups);
    const int most_shift = n.classes > 1 ? 7 : 0;
    if (n.vectors < 1 || n.vectors > 2 || n.lanes * n.vectors * 8 < n.cta_cols || n.cta_cols % 8 ||
        (int64_t)n.cta_cols * n.cluster < n.cols + most_shift)
        return fail(p, "columns of a block", n.cta_cols, n.cluster);
    if (n.classes > 1 && (n.classes * n.drift % 8 || n.drift < 1 || n.drift > 7))
        return fail(p, "classes of rows", n.classes, n.drift);
    if (n.full && (n.cols % 8 || n.classes > 1 || n.wide != kNormWideAll))
        return fail(p, "whole vectors", n.classes, n.wide);
    if (n.smem != (size_t)2 * n.threads * 16 * n.units * n.vectors || n.smem > kNormSmemPerSm)
        return fail(p, "shared memory", (long long)n.smem, n.units);
    if (n.ctas < 1 || n.ctas % n.classes || (int64_t)n.ctas * n.cluster > kNormSms * 64 + 8)
        return fail(p, "clusters of a launch", n.ctas, n.classes);
    return 0;
}

static int shapes()
{
    const int64_t some_rows[] = {1, 2, 5, 4096};
    for (int64_t cols = 1; cols <= 32768; ++cols)
        for (int pad = 0; pad < 8; ++pad)
            for (int kind = 0; kind < 8; ++kind) {
                const bool backward = kind & 1, general = kind & 2, shared = kind & 4;
                rikfad_residual_norm p{};
                p.dtype = (int)below(3);
                p.residual_dtype = chance() ? RIKFAD_F32 : p.dtype;
                p.rows = some_rows[below(4)] * (shared ? 3 : 1);
                p.cols = cols;
                p.gate_rows = shared ? 3 : 1;
                p.post = general ? RIKFAD_NORM_LAYER : RIKFAD_NORM_RMS;
                p.pre = RIKFAD_NORM_RMS;
                const int64_t stride = cols + pad;
                p.x = somewhere(0, stride, p.residual_dtype, 0);
                p.z = somewhere(1, stride, p.dtype, 0);
                p.gate = somewhere(2, stride, p.gate_dtype, 0);
                void *const vec = reinterpret_cast<void *>((uintptr_t)1 << 50);
                p.stats = static_cast<float *>(vec);
                p.pre_weight = p.post_weight = vec;
                if (backward) {
                    p.du = somewhere(3, stride, p.residual_dtype, 0);
                    p.dh = somewhere(4, stride, p.dtype, 0);
                    p.dx = somewhere(5, stride, p.residual_dtype, 0);
                    p.dz = somewhere(6, stride, p.dtype, 0);
                    p.dgate = somewhere(7, stride, p.gate_dtype, 0);
                    p.dpre_weight = p.dpost_weight = vec;
                } else {
                    p.u = somewhere(3, stride, p.residual_dtype, 0);
                    p.h = somewhere(4, stride, p.dtype, 0);
                }
                if (run(p, backward))
                    return fail(p, g_error.c_str(), pad, kind);
                if (check_shape(p, g_launched) || check_copies(p, g_launched, backward))
                    return 1;
            }
    return 0;
}

int main(int argc, char **argv)
{
    const char *what = argc > 1 ? argv[1] : "";
    const int rc = !std::strcmp(what, "copies") ? copies() : !std::strcmp(what, "shapes") ? shapes() : 2;
    if (rc == 0)
        std::printf("OK\n");
    return rc;
}
