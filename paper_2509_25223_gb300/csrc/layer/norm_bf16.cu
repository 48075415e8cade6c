// norm_bf16.cu -- the norm kernels (norm.cuh) for f, z and h in bf16.
#include "norm.cuh"

namespace rdn {
namespace norm {
cudaError_t run_bf16(const NormP &p, const Launch &l, bool x_f32, bool bwd, cudaStream_t s) {
  return x_f32 ? run_x<__nv_bfloat16, float>(p, l, bwd, s) : run_x<__nv_bfloat16, __nv_bfloat16>(p, l, bwd, s);
}
}  // namespace norm
}  // namespace rdn
