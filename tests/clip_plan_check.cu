// Host-side check of the clipping plan: the C entries' host code with the CUDA
// runtime replaced by host memory and a record of what is still under way
// (tests/host_runtime.cpp).  Compiled by tests/test_clip_plan.py; the argument names the check.  Prints "OK"
// or the first violation.
//
//   upload  a plan that create returns has arrived: no stream has to wait for it
//   shares  the shares' segments cover every element once, in order
#include "rikfad_clip.cu"

#include <cstdio>
#include <cstdlib>

extern bool g_under_way;        // host_runtime.cpp: a copy that the device may not have yet
static std::string g_error;

namespace rikfad {

int report_error(int code, const std::string &msg)
{
    g_error = msg;
    return code;
}
int check_address(const void *, int, const char *, int64_t) { return RIKFAD_OK; }
cudaError_t counted_malloc(void **p, size_t bytes)
{
    *p = std::malloc(bytes);
    return *p ? cudaSuccess : cudaErrorMemoryAllocation;
}
void counted_free(void *p) { std::free(p); }

}  // namespace rikfad

static int fail(const char *what, long long a, long long b)
{
    std::printf("FAIL %s (%lld, %lld) %s\n", what, a, b, g_error.c_str());
    return 1;
}

static const std::vector<std::vector<int64_t>> &lists()
{
    static std::vector<std::vector<int64_t>> all;
    if (all.empty()) {
        all = {{}, {0}, {1}, {0, 1, 0}, {7, 64, 65, 8191}, {256 * 512, 512}, {(int64_t)1 << 31, 9, (int64_t)1 << 33},
               std::vector<int64_t>(1024, 130), std::vector<int64_t>(1025, 1), std::vector<int64_t>(3000, 0)};
        uint64_t r = 88172645463325252ull;
        auto next = [&](int64_t n) {
            r ^= r << 13, r ^= r >> 7, r ^= r << 17;
            return (int64_t)(r % (uint64_t)n);
        };
        for (int i = 0; i < 300; ++i) {
            std::vector<int64_t> v((size_t)next(next(4) ? 40 : 2600));
            for (int64_t &n : v)
                n = next(5) ? next((int64_t)1 << (1 + next(26))) : next(200);
            all.push_back(v);
        }
    }
    return all;
}

static int upload()
{
    for (const auto &numel : lists()) {
        const std::vector<int> types(numel.size(), RIKFAD_F32);
        rikfad_clip c = nullptr;
        if (rikfad_clip_create(numel.data(), types.data(), nullptr, (int)numel.size(), &c))
            return fail("create", (long long)numel.size(), 0);
        if (g_under_way)
            return fail("create returned before its plan had arrived", (long long)numel.size(), 0);
        rikfad_clip_destroy(c);
    }
    return 0;
}

static int check_shares(rikfad_clip c, const std::vector<int64_t> &numel, const std::vector<int> &in, const std::vector<int> &out)
{
    const ClipParams &a = c->params;
    if (a.ntensors != (int)numel.size() || a.total_blocks != c->blocks || a.block_segment[0] != 0)
        return fail("head", a.ntensors, a.total_blocks);
    int tensor = 0, block = 0, q = 0;
    int64_t at = 0;
    for (const Part &p : c->parts) {
        if (p.tensor0 != tensor || p.block0 != block || p.tensor1 - p.tensor0 > kMaxTensors || p.block1 <= p.block0 ||
            p.block1 - p.block0 > 152 * kClipBlocksPerSm)
            return fail("part", p.tensor0, p.block0);
        for (; block < p.block1; ++block) {
            if (a.block_segment[block] != q || (numel.size() && a.block_segment[block + 1] <= q))
                return fail("a block's segments", block, q);
            for (; q < a.block_segment[block + 1]; ++q) {
                const Segment &s = a.segments[q];
                if (s.list_tensor != tensor || s.tensor != tensor - p.tensor0 || tensor >= p.tensor1)
                    return fail("a segment's tensor", q, tensor);
                if (s.begin != at || s.end < at || s.end > numel[tensor] || s.end - s.begin > kMaxShare + kShareStep ||
                    s.begin % kShareStep || (s.begin == s.end && numel[tensor]))
                    return fail("a segment's elements", q, at);
                if (s.grad_dtype != in[tensor] || s.out_dtype != out[tensor])
                    return fail("a segment's types", q, tensor);
                if (q < s.first || q >= s.first + s.count || a.segments[s.first].begin != 0 ||
                    a.segments[s.first].list_tensor != tensor || a.segments[s.first + s.count - 1].end != numel[tensor])
                    return fail("a tensor's first segment and their number", q, tensor);
                at = s.end;
                if (at == numel[tensor])
                    ++tensor, at = 0;
            }
        }
        if (tensor != p.tensor1)
            return fail("a part's tensors", tensor, p.tensor1);
    }
    if (tensor != (int)numel.size() || block != c->blocks || a.block_segment[block] != q)
        return fail("end", tensor, block);
    for (int t = 0; t < (int)numel.size(); ++t)
        if (a.tensor_sum[t] != 0.0 || a.tensor_done[t] != 0)
            return fail("a counter that is not zero", t, 0);
    return a.result->blocks_done == 0 ? 0 : fail("blocks_done", 0, 0);
}

static int shares()
{
    int kind = 0;
    for (const auto &numel : lists()) {
        std::vector<int> in, out;
        for (size_t t = 0; t < numel.size(); ++t)
            in.push_back(kind++ % 3), out.push_back(kind % 3);
        rikfad_clip c = nullptr;
        if (rikfad_clip_create(numel.data(), in.data(), out.data(), (int)numel.size(), &c))
            return fail("create", (long long)numel.size(), 0);
        if (check_shares(c, numel, in, out))
            return 1;
        rikfad_clip_destroy(c);
    }
    return 0;
}

int main(int argc, char **argv)
{
    const std::string what = argc > 1 ? argv[1] : "";
    const int rc = what == "upload" ? upload() : what == "shares" ? shares() : 2;
    if (rc == 0)
        std::printf("OK\n");
    return rc;
}
