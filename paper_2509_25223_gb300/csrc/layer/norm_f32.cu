// norm_f32.cu -- the norm kernels (norm.cuh) for f, z and h in f32.
#include "norm.cuh"

namespace rdn {
namespace norm {
cudaError_t run_f32(const NormP &p, const Launch &l, bool x_f32, bool bwd, cudaStream_t s) {
  return x_f32 ? run_x<float, float>(p, l, bwd, s) : run_x<float, __nv_bfloat16>(p, l, bwd, s);
}
}  // namespace norm
}  // namespace rdn
