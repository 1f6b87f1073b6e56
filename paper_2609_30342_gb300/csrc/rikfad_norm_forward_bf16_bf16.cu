// The residual norm's forward kernels for bf16 activations and a bf16 residual stream.
#include "rikfad_norm_kernels.cuh"

namespace rikfad {

cudaError_t norm_forward_bf16_bf16(const NormParams &n, cudaStream_t s) { return norm_forward<__nv_bfloat16, __nv_bfloat16>(n, s); }

}  // namespace rikfad
