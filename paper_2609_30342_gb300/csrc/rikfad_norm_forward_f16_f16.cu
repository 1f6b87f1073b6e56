// The residual norm's forward kernels for f16 activations and a f16 residual stream.
#include "rikfad_norm_kernels.cuh"

namespace rikfad {

cudaError_t norm_forward_f16_f16(const NormParams &n, cudaStream_t s) { return norm_forward<__half, __half>(n, s); }

}  // namespace rikfad
