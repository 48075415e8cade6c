// norm.cu -- the norms around a block (norm.cuh): plan, dispatch and the join of
// the parameter gradients.
#include "norm.cuh"

namespace rdn {
namespace {

using norm::Launch;
using norm::NormP;

// dw [heads, D] = scale q and dscale [D] = w q, dw_next [D], from the row slots'
// partials, in order: 16 interleaved sums, joined in order.
__global__ void __launch_bounds__(512) norm_grad_kernel(const NormP p, int slots, float *dw, float *dscale,
                                                        float *dw_next) {
  __shared__ float sh[16][32];
  const int which = blockIdx.z, head = blockIdx.y, i = blockIdx.x * 32 + threadIdx.x;
  if (which ? !dw_next || head : !dw) return;
  const int stride = which ? 1 : p.heads;
  float a = 0.f;
  if (i < p.D)
    for (long long q = (which ? 0 : head) + (long long)threadIdx.y * stride; q < slots; q += 16ll * stride)
      a += p.part[((size_t)q * 2 + which) * p.D + i];
  sh[threadIdx.y][threadIdx.x] = a;
  __syncthreads();
  if (threadIdx.y || i >= p.D) return;
#pragma unroll
  for (int y = 1; y < 16; ++y) a += sh[y][threadIdx.x];
  if (which) {
    dw_next[i] = a;
    return;
  }
  const bool x = p.mode & norm::kX;
  dw[(size_t)head * p.D + i] = !x ? a : a * (p.scale ? p.scale[i] : p.scale_const);
  if (dscale) dscale[i] = a * p.w[i];
}

int gcd(int a, int b) { return b ? gcd(b, a % b) : a; }

struct NormPlan : Launch {
  int tpr, slots;   // threads per row and CTA, row slots of the grid
  int split, cols;  // CTAs per row, columns of each
};
// CTAs of up to 256 threads (of 384 where that is the most; a row's, if it needs
// more), as many as are resident, so that they stay for many rows; their slots a
// multiple of the heads, so that a slot's rows share a row of w.
NormPlan norm_plan(const rdn_norm_args &a, bool bwd, bool vec) {
  constexpr int kSMs = 152, E = 8;
  NormPlan pl;
  pl.vec = vec;
  const int most = !vec ? norm::kFewThreads : bwd ? norm::kThreads : norm::kMostThreads;
  pl.split = a.D <= most * E ? 1 : (a.D + norm::kFewThreads * E - 1) / (norm::kFewThreads * E);
  pl.cols = pl.split == 1 ? a.D : ((a.D + pl.split - 1) / pl.split + 7) / 8 * 8;
  pl.tpr = (pl.cols + E - 1) / E;
  pl.tpr = pl.split == 1 && pl.tpr <= 8 ? 8 : pl.split == 1 && pl.tpr <= 16 ? 16 : (pl.tpr + 31) / 32 * 32;
  const bool any_f32 = a.dtype == RDN_F32 || (a.x && a.x_dtype == RDN_F32);
  const bool few = pl.split > 1 || norm::few_threads(vec, bwd, any_f32, pl.tpr);
  // (rows of 5 warps and more have a CTA each)
  const int per = pl.split > 1 || pl.tpr > 128 ? 1 : (few ? norm::kFewThreads : 256) / pl.tpr;
  pl.threads = pl.tpr * per;
  const int step = a.heads / gcd(a.heads, per);
  const long long need = ((a.rows + per - 1) / per + step - 1) / step * step;
  const int threads = few ? norm::kFewThreads : bwd ? norm::kThreads : 2 * norm::kThreads;
  const int resident = threads / pl.threads > 1 ? threads / pl.threads : 1;
  // (clusters of more than two leave SMs unused; one more than fits would take as long as all)
  const long long at_once = pl.split == 1 ? kSMs * resident : pl.split == 2 ? kSMs / 2 : (kSMs - 16) / pl.split;
  const long long rows = (at_once + step - 1) / step * step;
  const long long units = (rows < need ? rows : need);
  pl.ctas = (int)(units * pl.split);
  pl.slots = (int)(units * per);
  return pl;
}

bool norm_vec(const rdn_norm_args &a, bool bwd) {
  if (a.D % 8) return false;  // (rows on 16 bytes in either type)
  const size_t es = a.dtype == RDN_BF16 ? 2 : 4, xs = a.x_dtype == RDN_BF16 ? 2 : 4;
  auto on = [](const void *p, size_t bytes) { return !p || (((uintptr_t)p | bytes) & 15) == 0; };
  if (!on(a.f, a.f_ld * es) || !on(a.z, a.z_ld * es) || !on(a.x, a.x_ld * xs)) return false;
  if (!on(a.w, 0) || !on(a.scale, 0) || !on(a.w_next, 0)) return false;
  if (!bwd) return on(a.r_out, 0) && on(a.h, 0);
  return on(a.dr, 0) && on(a.dh, 0) && on(a.df, 0) && on(a.dz, 0) && on(a.dx, 0);
}

}  // namespace

size_t norm_bwd_bytes(const rdn_norm_args &a) {
  // (the larger of the two accesses' plans: the query sees no pointers)
  const int v = norm_plan(a, true, true).slots, e = norm_plan(a, true, false).slots;
  return round256(sizeof(float) * 2 * (size_t)(v > e ? v : e) * a.D);
}

cudaError_t launch_norm(const rdn_norm_args &a, bool bwd, cudaStream_t s) {
  const NormPlan pl = norm_plan(a, bwd, norm_vec(a, bwd));
  NormP p{};
  p.rows = a.rows; p.D = a.D; p.heads = a.heads; p.tpr = pl.tpr;
  p.split = pl.split; p.cols = pl.cols;
  p.mode = (a.f ? norm::kF : 0) | (a.x ? norm::kX : 0) | (a.w_next ? norm::kH : 0) | (a.f && a.z ? 1 + a.gate : 0);
  p.eps = a.eps; p.scale_const = a.scale_const;
  p.f_ld = a.f_ld; p.z_ld = a.z_ld; p.x_ld = a.x_ld;
  p.f = a.f; p.z = a.z; p.x = a.x; p.dr = a.dr; p.dh = a.dh;
  p.w = a.w; p.scale = a.f && a.x ? a.scale : nullptr; p.w_next = a.w_next;
  p.r_out = a.f ? a.r_out : nullptr; p.h = a.h;
  p.df = a.df; p.dz = a.dz; p.dx = a.dx;
  p.part = static_cast<float *>(a.workspace);
  const bool xf = a.x_dtype == RDN_F32;
  const cudaError_t e = a.dtype == RDN_BF16 ? norm::run_bf16(p, pl, xf, bwd, s) : norm::run_f32(p, pl, xf, bwd, s);
  if (e != cudaSuccess || !bwd) return e;
  const dim3 grid((a.D + 31) / 32, a.heads, 2);
  RDN_LAUNCH("norm_grad", s,
             (norm_grad_kernel<<<grid, dim3(32, 16), 0, s>>>(p, pl.slots, a.f ? a.dw : nullptr,
                                                             p.scale ? a.dscale : nullptr,
                                                             a.w_next ? a.dw_next : nullptr)));
  return cudaGetLastError();
}

}  // namespace rdn
