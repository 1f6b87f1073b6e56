// rikfad_norm.hpp -- parameters and launches of the residual norm's kernels, shared
// by the host code and the instantiations per element type.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "rikfad.h"

namespace rikfad {

// A thread owns 8 neighbouring columns of a row (two times 8 forward, where a row has
// enough of them).  A row is one to 32 lanes', then up to 16 warps' (a block's), then a
// cluster's of up to 8 blocks, which exchange their sums through distributed shared
// memory.
constexpr int kNormMaxThreads = 512;
constexpr int kNormMaxWarps = kNormMaxThreads / 32;
constexpr int kNormMaxCluster = 8;              // what every launch may ask for
// Threads of an SM, by the registers that the kernels are given: 80 with one vector
// forward, 128 with two and backward.
constexpr int kNormForwardThreads1 = 768, kNormForwardThreads2 = 512, kNormBackwardThreads = 512;
// With a post norm and layer norms or biases ("heavy"), fewer threads with more
// registers: 128 with one vector forward (8192 x 1600 with a shared gate: 47 us, 60 with
// 80), 168 with two (8192 x 1600: 36 us, 42 with 128) and backward (72 us, 99 with 128) for
// rows of up to kNormHeavyCols columns.  Wider ones would leave an SM one block, or take
// two blocks a row (4096 x 4096: forward 52 us instead of 47, backward 141 instead of 117).
constexpr int kNormHeavyForwardThreads1 = 512, kNormHeavyThreads = 384;
constexpr int kNormHeavyCols = 8 * kNormHeavyThreads - 8;      // a shifted row may need one vector more
constexpr int norm_registers(int threads) { return threads <= 256 ? 248 : 65536 / threads / 8 * 8; }
// Rows of a gate from which it is kept in registers, not staged for every row (8192 x
// 1600, 1024 rows a gate: forward 30 us, 50 staged; 16 rows: 30 and 33; 4 rows: 33 both).
constexpr int64_t kNormHeldRows = 16;
constexpr int kNormSms = 152;
constexpr size_t kNormSmemPerSm = 200 << 10;    // for the stages; a block keeps 1 KB more
constexpr size_t kNormSmemDefault = 40 << 10;   // a block may have as much unasked (48 KB, less the row sums' slots)

enum : uint32_t {
    kNormBranch = 1u << 0,          // z is there
    kNormGated = 1u << 1,
    kNormGateF32 = 1u << 2,
    kNormParamF32 = 1u << 3,
    kNormPost = 1u << 4,
    kNormPostLayer = 1u << 5,
    kNormPostWeight = 1u << 6,
    kNormPostBias = 1u << 7,
    kNormPre = 1u << 8,
    kNormPreLayer = 1u << 9,
    kNormPreWeight = 1u << 10,
    kNormPreBias = 1u << 11,
    kNormU = 1u << 12,
    kNormH = 1u << 13,
    kNormStats = 1u << 14,
    kNormDu = 1u << 15,
    kNormDh = 1u << 16,
    kNormDx = 1u << 17,
    kNormDz = 1u << 18,
    kNormDgate = 1u << 19,
    kNormSharedGate = 1u << 20,     // a gate serves several rows
    kNormDpreWeight = 1u << 21,
    kNormDpostWeight = 1u << 22,
    kNormDpreBias = 1u << 23,
    kNormDpostBias = 1u << 24,
    kNormGateHeld = 1u << 25,       // a gate lasts so long that it is kept in registers
};

// Tensors whose vectors all start on 16 bytes.
enum : uint32_t {
    kNormWideX = 1u << 0,
    kNormWideZ = 1u << 1,
    kNormWideGate = 1u << 2,
    kNormWideU = 1u << 3,
    kNormWideH = 1u << 4,
    kNormWideDu = 1u << 5,
    kNormWideDh = 1u << 6,
    kNormWideDx = 1u << 7,
    kNormWideDz = 1u << 8,
    kNormWideDgate = 1u << 9,
    kNormWideAll = (1u << 10) - 1,
};

// Rows of `cols` elements, and the bytes from a thread's row to its next one.
struct NormRows {
    void *data;
    int64_t stride, step;
};

struct NormParams {
    int64_t rows, gate_rows;
    int32_t cols;
    float inv_cols, a, b, post_eps, pre_eps;
    // Rows of class c (c, c + classes, ...) start c * drift % 8 elements after a vector.
    int32_t classes, drift;
    NormRows x, z, gate;
    const void *post_weight, *post_bias, *pre_weight, *pre_bias;
    float4 *stats;              // mean, 1/deviation of post; the same of pre
    NormRows u, h;
    NormRows du, dh, dx, dz, dgate;
    void *dpost_weight, *dpost_bias, *dpre_weight, *dpre_bias;
    uint32_t flags, wide;
    // the launch
    bool full, general;                     // only whole vectors; a layer norm, a bias or its gradient
    int32_t vectors;                        // of a thread
    int32_t threads, lanes, row_groups;     // of a block; of a row within it; rows of a block at a time
    int32_t cluster, cta_cols;              // blocks of a row; columns of each
    int32_t ctas;                           // clusters of the launch
    int32_t threads_per_sm;                 // by the kernel's registers
    int32_t units;                          // 16-byte units of a vector
    int32_t join_rows;                      // of the join kernel (join_gate)
    bool join_bounds;
    size_t smem;
    // backward: partial sums
    int32_t sums;
    float *sum_part;            // sums x ctas x cols, in the order dpre_weight, dpost_weight, dpre_bias, dpost_bias
    float *gate_part;           // ctas x row_groups x 2 x cols
};

// One translation unit each (types of the activations and of the residual stream).
cudaError_t norm_forward_f32_f32(const NormParams &n, cudaStream_t s);
cudaError_t norm_backward_f32_f32(const NormParams &n, cudaStream_t s);
cudaError_t norm_forward_bf16_bf16(const NormParams &n, cudaStream_t s);
cudaError_t norm_backward_bf16_bf16(const NormParams &n, cudaStream_t s);
cudaError_t norm_forward_bf16_f32(const NormParams &n, cudaStream_t s);
cudaError_t norm_backward_bf16_f32(const NormParams &n, cudaStream_t s);
cudaError_t norm_forward_f16_f16(const NormParams &n, cudaStream_t s);
cudaError_t norm_backward_f16_f16(const NormParams &n, cudaStream_t s);
cudaError_t norm_forward_f16_f32(const NormParams &n, cudaStream_t s);
cudaError_t norm_backward_f16_f32(const NormParams &n, cudaStream_t s);

}  // namespace rikfad
