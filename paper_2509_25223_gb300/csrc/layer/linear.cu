// linear.cu -- the matrix product with bias, activation and residual (include/rdn.h,
// rdn_linear_*): the tensor maps, the choice of the kernel, and what the backward does
// besides its two products: dp = dy act'(pre) and the bias's gradient.
#include "linear.cuh"
#include "maps.cuh"

#include <cuda.h>
#include <cudaTypedefs.h>

namespace rdn {
namespace lin {
namespace {

PFN_cuTensorMapEncodeTiled_v12000 encoder() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
    void *f = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess)
      f = nullptr;
    return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f);
  }();
  return fn;
}

}  // namespace

bool make_map(Map *m, const Operand &o, int elem, int box) {
  const auto enc = encoder();
  if (!enc) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)(o.mn ? o.rows : o.k), (cuuint64_t)(o.mn ? o.k : o.rows)};
  const cuuint64_t strides[1] = {(cuuint64_t)o.ld * elem};
  const cuuint32_t boxes[2] = {(cuuint32_t)(128 / elem), (cuuint32_t)(o.mn ? 64 : box)};
  const cuuint32_t one[2] = {1, 1};
  return enc(reinterpret_cast<CUtensorMap *>(m),
             elem == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(o.p),
             dims, strides, boxes, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace lin

bool make_rows_map(void *map128, const void *p, int cols, int rows, int depth, long long ld, int box_cols,
                   int box_rows) {
  const auto enc = lin::encoder();
  if (!enc) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)depth};
  const cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)ld * 2 * rows};
  const cuuint32_t boxes[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1};
  const cuuint32_t one[3] = {1, 1, 1};
  return enc(reinterpret_cast<CUtensorMap *>(map128), CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(p), dims,
             strides, boxes, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

namespace lin {

cudaError_t run_product(const Operand &a, const Operand &b, GemmP p, bool fp8, cudaStream_t s) {
  p.status = status_word();
  const int per = fp8 ? 128 : 64;  // elements of 128 bytes
  p.kblocks = (int)((a.k + per - 1) / per);
  return split_fits(a, b, p.kblocks) ? run_split(a, b, p, fp8, s) : run_tiles(a, b, p, fp8, s);
}

namespace {

// dp = dy act'(pre), rounded to bf16 as the tensor core takes its operands (at most 2^-8 of a term, 0.17 % of the
// products' RMS beside the 0.17 % of their own rounding; two bf16 parts would double the products), and its column
// sums over the CTA's rows, which a kernel of its own joins or (kJoin: one cluster of up to 8 CTAs has all rows)
// this one.  A thread has 8 columns; the 8 warps of a CTA take rows in turn.
// 16384 x 4096 with SiLU: 60 to 68 us, 5.9 to 6.7 TB/s.
struct DpP {
  long long M, dy_ld;
  int N, act;
  const __nv_bfloat16 *dy, *pre;
  __nv_bfloat16 *dp;
  float *part;  // [gridDim.y][N], or NULL
  void *dbias;  // or NULL
  int bias_f32;
};
template <int kAct>
__device__ __forceinline__ void scale_by_grad(float (&g)[8], const float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) g[j] *= act_grad(kAct, v[j]);
}
__device__ __forceinline__ void put_bias(void *dbias, int f32, long long n, float a) {
  if (f32) static_cast<float *>(dbias)[n] = a;
  else static_cast<__nv_bfloat16 *>(dbias)[n] = from_f32<__nv_bfloat16>(a);
}
template <bool kJoin>
__global__ void __launch_bounds__(256) dp_kernel(const DpP p) {
  using P8 = Pack<__nv_bfloat16, 8>;
  __shared__ float sh[8][32 * 8 + 8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (kJoin) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  const long long n = (long long)blockIdx.x * 256 + lane * 8;
  const bool live = n < p.N;
  float sum[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) sum[j] = 0.f;
  if (live) {
    // two rows at a time: their loads are in flight together
    const long long stride = (long long)gridDim.y * 8;
    auto put = [&](long long m, const typename P8::Raw &gy, const typename P8::Raw &gp) {
      float g[8];
      P8::get(gy, g);
      if (p.act) {
        float v[8];
        P8::get(gp, v);
        if (p.act == 1) scale_by_grad<1>(g, v);
        else if (p.act == 2) scale_by_grad<2>(g, v);
        else scale_by_grad<3>(g, v);
        if (p.dp) P8::st(p.dp + m * p.N + n, P8::put(g));
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j] += g[j];
    };
    for (long long m = (long long)blockIdx.y * 8 + warp; m < p.M; m += 2 * stride) {
      const bool two = m + stride < p.M;
      const typename P8::Raw g0 = P8::ld(p.dy + m * p.dy_ld + n);
      const typename P8::Raw g1 = two ? P8::ld(p.dy + (m + stride) * p.dy_ld + n) : P8::zero();
      const typename P8::Raw v0 = p.act ? P8::ld(p.pre + m * p.N + n) : P8::zero();
      const typename P8::Raw v1 = p.act && two ? P8::ld(p.pre + (m + stride) * p.N + n) : P8::zero();
      put(m, g0, v0);
      if (two) put(m + stride, g1, v1);
    }
  }
  if (!kJoin && !p.part) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) sh[warp][j * 33 + lane] = sum[j];
  __syncthreads();
  const int c = threadIdx.x;  // a column each
  const long long at = (long long)blockIdx.x * 256 + c;
  float a = 0.f;
#pragma unroll
  for (int w = 0; w < 8; ++w) a += sh[w][(c & 7) * 33 + (c >> 3)];
  if constexpr (kJoin) {
    __shared__ float joined[8][256];
    const uint32_t to = tc::map_rank(&joined[blockIdx.y][c], 0);
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");  // every CTA of the cluster runs
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to), "f"(a) : "memory");
    tc::cluster_sync();
    if (blockIdx.y || at >= p.N) return;
    a = joined[0][c];
    for (int q = 1; q < (int)gridDim.y; ++q) a += joined[q][c];
    put_bias(p.dbias, p.bias_f32, at, a);
  } else if (at < p.N) {
    p.part[(size_t)blockIdx.y * p.N + at] = a;
  }
}
// dbias: the CTAs' sums, in order: 16 interleaved sums, joined in order.
__global__ void __launch_bounds__(512) dbias_kernel(const float *part, int parts, int N, void *dbias, int f32) {
  __shared__ float sh[16][32];
  const int n = blockIdx.x * 32 + threadIdx.x;
  float a = 0.f;
  if (n < N)
    for (int q = threadIdx.y; q < parts; q += 16) a += part[(size_t)q * N + n];
  sh[threadIdx.y][threadIdx.x] = a;
  __syncthreads();
  if (threadIdx.y || n >= N) return;
#pragma unroll
  for (int y = 1; y < 16; ++y) a += sh[y][threadIdx.x];
  put_bias(dbias, f32, n, a);
}

// CTAs over the rows: about 8 a SM in all.
int dp_parts(const rdn_linear_args &a) {
  const long long cols = (a.N + 255) / 256, rows = (a.M + 7) / 8, want = (152 * 8 + cols - 1) / cols;
  return (int)(rows < want ? (rows < 1 ? 1 : rows) : want);
}
size_t dp_bytes(const rdn_linear_args &a) { return a.act ? round256((size_t)a.M * a.N * 2) : 0; }
// Rows whose sums one cluster joins: a launch less, where a warp has up to 8 rows all the same (forward and
// backward of 1024 x 1024 by 512 rows called one by one 54 -> 47 us, in a graph 27.2 -> 28.6; 173 rows 23.9 -> 23.7).
bool joins(const rdn_linear_args &a) { return a.M <= 512; }

cudaError_t run_dp(const DpP &d, int parts, bool join, cudaStream_t s) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((d.N + 255) / 256, parts);
  cfg.blockDim = dim3(256);
  cfg.stream = s;
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = at.val.clusterDim.z = 1;
  at.val.clusterDim.y = join ? parts : 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  cudaError_t e = cudaSuccess;
  RDN_LAUNCH("linear_dp", s, (e = cudaLaunchKernelEx(&cfg, join ? dp_kernel<true> : dp_kernel<false>, d)));
  return e;
}

}  // namespace
}  // namespace lin

// (the query sees no pointers, and allows for dbias)
size_t linear_bwd_bytes(const rdn_linear_args &a, bool dbias) {
  return lin::dp_bytes(a) +
         (dbias && !lin::joins(a) ? round256(sizeof(float) * (size_t)lin::dp_parts(a) * a.N) : 0);
}

cudaError_t launch_linear_fwd(const rdn_linear_args &a, cudaStream_t s) {
  if (a.M == 0) return cudaSuccess;
  lin::GemmP p{};
  p.M = a.M; p.N = a.N;
  p.e.xs = a.x_scale; p.e.ws = a.w_scale; p.e.bias = a.bias; p.e.res = a.res; p.e.y = a.y;
  p.e.pre = static_cast<__nv_bfloat16 *>(a.pre);
  p.e.res_ld = a.res_ld; p.e.y_ld = a.y_ld; p.e.pre_ld = a.N;
  p.e.act = a.act; p.e.bias_f32 = a.bias_dtype == RDN_F32; p.e.out_f32 = a.y_dtype == RDN_F32;
  p.inject = fault_injection() == 3;
  return lin::run_product({a.x, a.M, a.K, a.x_ld, false}, {a.w, a.N, a.K, a.w_ld, false}, p, a.dtype == RDN_E4M3, s);
}

cudaError_t launch_linear_bwd(const rdn_linear_args &a, cudaStream_t s) {
  const size_t be = a.bias_dtype == RDN_F32 ? 4 : 2, we = a.dw_dtype == RDN_F32 ? 4 : 2;
  cudaError_t e = cudaSuccess;
  if (a.M == 0) {  // sums of nothing
    if (a.dw) e = cudaMemsetAsync(a.dw, 0, (size_t)a.N * a.K * we, s);
    if (e == cudaSuccess && a.dbias) e = cudaMemsetAsync(a.dbias, 0, (size_t)a.N * be, s);
    return e;
  }
  lin::DpP d{};
  d.M = a.M; d.dy_ld = a.dy_ld; d.N = a.N; d.act = a.act;
  d.dy = static_cast<const __nv_bfloat16 *>(a.dy);
  d.pre = static_cast<const __nv_bfloat16 *>(a.pre);
  d.dp = a.dx || a.dw ? static_cast<__nv_bfloat16 *>(a.workspace) : nullptr;
  const bool join = a.dbias && lin::joins(a);
  d.part = a.dbias && !join ? reinterpret_cast<float *>(static_cast<char *>(a.workspace) + lin::dp_bytes(a)) : nullptr;
  d.dbias = a.dbias;
  d.bias_f32 = be == 4;
  const int inject = fault_injection() == 4;
  const void *dp = a.dy;
  long long dp_ld = a.dy_ld;
  if ((a.act && d.dp) || a.dbias) {
    const int parts = join ? (int)(a.M < 64 ? (a.M + 7) / 8 : 8) : lin::dp_parts(a);
    if ((e = lin::run_dp(d, parts, join, s)) != cudaSuccess) return e;
    if (d.part) {
      RDN_LAUNCH("linear_dbias", s,
                 (lin::dbias_kernel<<<(a.N + 31) / 32, dim3(32, 16), 0, s>>>(d.part, parts, a.N, a.dbias, be == 4)));
      if ((e = cudaGetLastError()) != cudaSuccess) return e;
    }
    if (a.act) {
      dp = d.dp;
      dp_ld = a.N;
    }
  }
  if (a.dx) {
    lin::GemmP p{};
    p.M = a.M; p.N = a.K;
    p.inject = inject;
    p.e.y = a.dx; p.e.y_ld = a.K;
    e = lin::run_product({dp, a.M, a.N, dp_ld, false}, {a.w, a.K, a.N, a.w_ld, true}, p, false, s);
    if (e != cudaSuccess) return e;
  }
  if (a.dw) {
    lin::GemmP p{};
    p.M = a.N; p.N = a.K;
    p.inject = inject;
    p.e.y = a.dw; p.e.y_ld = a.K; p.e.out_f32 = we == 4;
    e = lin::run_product({dp, a.N, a.M, dp_ld, true}, {a.x, a.K, a.M, a.x_ld, true}, p, false, s);
  }
  return e;
}

}  // namespace rdn
