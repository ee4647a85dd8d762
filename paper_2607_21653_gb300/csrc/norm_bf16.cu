// Residual norm kernels for bf16 activations.
#include "norm_kernels.cuh"

namespace molt {

cudaError_t launch_norm_bf16(const NormArgs& a, const NormShape& s, int grid, bool r_f32, bool bwd, cudaStream_t stream) {
  using X = __nv_bfloat16;
  if (bwd) return r_f32 ? launch_norm_bwd_typed<X, float>(a, s, grid, stream) : launch_norm_bwd_typed<X, X>(a, s, grid, stream);
  return r_f32 ? launch_norm_fwd_typed<X, float>(a, s, grid, stream) : launch_norm_fwd_typed<X, X>(a, s, grid, stream);
}

}  // namespace molt
