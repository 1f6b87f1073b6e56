// The residual norm's backward kernels for bf16 activations and a f32 residual stream.
#include "rikfad_norm_kernels.cuh"

namespace rikfad {

cudaError_t norm_backward_bf16_f32(const NormParams &n, cudaStream_t s) { return norm_backward<__nv_bfloat16, float>(n, s); }

}  // namespace rikfad
