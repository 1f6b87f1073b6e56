// The residual norm's kernels for float16 activations.
#include "rikfad_norm_kernels.cuh"

namespace rikfad {

cudaError_t launch_norm_f16(const NormParams &n, bool residual_f32, bool backward, cudaStream_t s)
{
    return residual_f32 ? launch_norm<__half, float>(n, backward, s) : launch_norm<__half, __half>(n, backward, s);
}

}  // namespace rikfad
