// The residual norm's kernels for float32 activations.
#include "rikfad_norm_kernels.cuh"

namespace rikfad {

cudaError_t launch_norm_f32(const NormParams &n, bool backward, cudaStream_t s)
{
    return launch_norm<float, float>(n, backward, s);
}

}  // namespace rikfad
