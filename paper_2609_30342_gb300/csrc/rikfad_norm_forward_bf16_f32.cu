// The residual norm's forward kernels for bf16 activations and a f32 residual stream.
#include "rikfad_norm_kernels.cuh"

namespace rikfad {

cudaError_t norm_forward_bf16_f32(const NormParams &n, cudaStream_t s) { return norm_forward<__nv_bfloat16, float>(n, s); }

}  // namespace rikfad
