// The residual norm's backward kernels for f16 activations and a f16 residual stream.
#include "rikfad_norm_kernels.cuh"

namespace rikfad {

cudaError_t norm_backward_f16_f16(const NormParams &n, cudaStream_t s) { return norm_backward<__half, __half>(n, s); }

}  // namespace rikfad
