// The residual norm's forward kernels for f32 activations and a f32 residual stream.
#include "rikfad_norm_kernels.cuh"

namespace rikfad {

cudaError_t norm_forward_f32_f32(const NormParams &n, cudaStream_t s) { return norm_forward<float, float>(n, s); }

}  // namespace rikfad
