// rikfad_norm.hpp -- parameters and launches of the residual norm's kernels, shared
// by the host code and the instantiations per element type.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "rikfad.h"

namespace rikfad {

// A row of up to 4096 columns is one block's (or, up to 256 columns, 8, 16 or 32
// lanes of one): every thread owns 8 neighbouring columns, so that a block of 512
// threads may use 128 registers each.  Wider rows are split over a cluster of up to
// 8 blocks, which exchange their sums through distributed shared memory.
constexpr int kNormMaxThreads = 512;
constexpr int kNormMaxWarps = kNormMaxThreads / 32;
constexpr int kNormRows = 2;                // rows of a thread at a time (1 where rows are few)
// Threads of an SM by the kernels' register bounds: 80; 168 with two rows and
// biases, else 128.
constexpr int kNormForwardThreads = 768;
template <bool WIDE> constexpr int kNormBackwardThreads = WIDE ? 384 : 512;
constexpr int kNormSms = 152;
constexpr size_t kNormSmemPerSm = 200 << 10;    // for the stages; a block keeps 4 KB more

// Rows of `cols` elements, and the bytes from a thread's row to its next one.
struct NormRows {
    void *data;
    int64_t stride, step;
};

struct NormParams {
    int64_t rows, gate_rows;
    int32_t cols, post, pre;
    float inv_cols, a, b, post_eps, pre_eps;
    int32_t gate_period;        // gate_rows, within int
    NormRows x, z, gate;
    const void *post_weight, *post_bias, *pre_weight, *pre_bias;
    float4 *stats;              // mean, 1/deviation of post; the same of pre
    NormRows u, h;
    NormRows du, dh, dx, dz, dgate;
    void *dpost_weight, *dpost_bias, *dpre_weight, *dpre_bias;
    bool gate_f32, param_f32;
    // rows that start on 16 bytes
    bool wide_x, wide_z, wide_gate, wide_params, wide_u, wide_h, wide_du, wide_dh, wide_dx, wide_dz, wide_dgate;
    // the launch
    int32_t at_once;                        // rows of a thread: 1 or kNormRows
    bool full, bias;                        // no ragged row; gradients of biases
    int32_t threads, lanes, row_groups;     // of a block; of a row within it; rows of a block at a time
    int32_t cluster, cta_cols;              // blocks of a row; columns of each
    int32_t ctas;                           // clusters of the launch
    int32_t units, stages;                  // 16-byte units of 8 columns of a row; rounds in flight and in use
    size_t smem;
    // backward: partial sums
    int32_t sums;
    float *sum_part;            // sums x ctas x cols, in the order dpre_weight, dpost_weight, dpre_bias, dpost_bias
    float *gate_part;           // ctas x row_groups x 2 x cols
};

cudaError_t launch_norm_f32(const NormParams &n, bool backward, cudaStream_t s);
cudaError_t launch_norm_bf16(const NormParams &n, bool residual_f32, bool backward, cudaStream_t s);
cudaError_t launch_norm_f16(const NormParams &n, bool residual_f32, bool backward, cudaStream_t s);

}  // namespace rikfad
