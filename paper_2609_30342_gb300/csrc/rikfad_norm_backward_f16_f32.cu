// The residual norm's backward kernels for f16 activations and a f32 residual stream.
#include "rikfad_norm_kernels.cuh"

namespace rikfad {

cudaError_t norm_backward_f16_f32(const NormParams &n, cudaStream_t s) { return norm_backward<__half, float>(n, s); }

}  // namespace rikfad
