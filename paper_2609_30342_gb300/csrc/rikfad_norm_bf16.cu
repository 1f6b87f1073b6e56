// The residual norm's kernels for bfloat16 activations.
#include "rikfad_norm_kernels.cuh"

namespace rikfad {

cudaError_t launch_norm_bf16(const NormParams &n, bool residual_f32, bool backward, cudaStream_t s)
{
    return residual_f32 ? launch_norm<__nv_bfloat16, float>(n, backward, s) : launch_norm<__nv_bfloat16, __nv_bfloat16>(n, backward, s);
}

}  // namespace rikfad
