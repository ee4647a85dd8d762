// Residual norm kernels for fp32 activations.
#include "norm_kernels.cuh"

namespace molt {

cudaError_t launch_norm_fp32(const NormArgs& a, const NormShape& s, int n_sm, int* grid, bool bwd, cudaStream_t stream) {
  return launch_norm_typed<float, float>(a, s, n_sm, grid, bwd, stream);
}

}  // namespace molt
