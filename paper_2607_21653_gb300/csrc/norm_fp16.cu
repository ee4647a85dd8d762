// Residual norm kernels for fp16 activations.
#include "norm_kernels.cuh"

namespace molt {

cudaError_t launch_norm_fp16(const NormArgs& a, const NormShape& s, int n_sm, int* grid, bool r_f32, bool bwd, cudaStream_t stream) {
  using X = __half;
  return r_f32 ? launch_norm_typed<X, float>(a, s, n_sm, grid, bwd, stream) : launch_norm_typed<X, X>(a, s, n_sm, grid, bwd, stream);
}

}  // namespace molt
