// Residual norm kernels for fp32 activations.
#include "norm_kernels.cuh"

namespace molt {

cudaError_t launch_norm_fp32(const NormArgs& a, const NormShape& s, int grid, bool bwd, cudaStream_t stream) {
  return bwd ? launch_norm_bwd_typed<float, float>(a, s, grid, stream) : launch_norm_fwd_typed<float, float>(a, s, grid, stream);
}

}  // namespace molt
