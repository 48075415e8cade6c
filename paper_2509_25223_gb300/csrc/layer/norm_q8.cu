// norm_q8.cu -- the residual's addition and the norm before a block, with an output in
// 8 bits and a scale per row (include/rdn.h, rdn_norm_q8):
//     r = x + f,  h = r / rms(r) w,  scale = max |h| / 448,  q = e4m3(h / scale).
// One pass: a row stays in the registers of its warps between the sum of squares, the
// maximum and the codes, so x and f are read once and r, q written once; it is bound by
// HBM.  A row has as few warps as hold it in 64 elements a lane (one warp to 2048
// elements), which need no barrier; where there are fewer rows than warps resident on
// the GPU a lane has 8, for then latency counts.
#include <cuda_fp8.h>

#include "rows.cuh"

namespace rdn {
namespace {

constexpr float kTop = 448.f, kFloor = 0x1p-100f;

struct Q8P {
  long long rows, x_ld, f_ld;
  int D, warps;  // warps of a row
  float eps;
  const void *x, *f;
  const float *w;
  void *r, *q;
  float *scale;
};

// 8 consecutive elements from index i of a row of D
template <typename T, bool kVec>
__device__ __forceinline__ void load8(const T *row, int i, int D, float (&v)[8]) {
  if constexpr (kVec) {
    if (i < D) {
      if constexpr (sizeof(T) == 2) {
        Pack<T, 8>::get(Pack<T, 8>::ld(row + i), v);
      } else {
        float a[4], b[4];
        Pack<T, 4>::get(Pack<T, 4>::ld(row + i), a);
        Pack<T, 4>::get(Pack<T, 4>::ld(row + i + 4), b);
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[e + 4] = b[e]; }
      }
      return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.f;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = i + e < D ? to_f32<T>(row[i + e]) : 0.f;
  }
}
template <typename T, bool kVec>
__device__ __forceinline__ void store8(T *row, int i, int D, const float (&v)[8]) {
  if constexpr (kVec) {
    if (i >= D) return;
    if constexpr (sizeof(T) == 2) {
      Pack<T, 8>::st(row + i, Pack<T, 8>::put(v));
    } else {
      *reinterpret_cast<float4 *>(row + i) = make_float4(v[0], v[1], v[2], v[3]);
      *reinterpret_cast<float4 *>(row + i + 4) = make_float4(v[4], v[5], v[6], v[7]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (i + e < D) row[i + e] = from_f32<T>(v[e]);
  }
}
template <bool kVec>
__device__ __forceinline__ void store_codes(uint8_t *row, int i, int D, const float (&v)[8]) {
  uint32_t c[2] = {0u, 0u};
#pragma unroll
  for (int e = 0; e < 8; e += 2)
    c[e / 4] |= (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(v[e], v[e + 1]), __NV_SATFINITE, __NV_E4M3)
                << (e % 4 * 8);
  if constexpr (kVec) {
    if (i < D) *reinterpret_cast<uint2 *>(row + i) = make_uint2(c[0], c[1]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (i + e < D) row[i + e] = (uint8_t)(c[e / 4] >> (e % 4 * 8));
  }
}

template <bool kMax>
__device__ __forceinline__ float both(float a, float b) { return kMax ? fmaxf(a, b) : a + b; }
// Over the row's warps (in order), for every thread of the row.
template <bool kMax>
__device__ __forceinline__ float over_row(float a, float *sh, int warps) {
#pragma unroll
  for (int o = 16; o; o >>= 1) a = both<kMax>(a, __shfl_xor_sync(0xffffffffu, a, o));
  if (warps == 1) return a;
  const int warp = threadIdx.x >> 5, first = warp / warps * warps;
  if ((threadIdx.x & 31) == 0) sh[warp] = a;
  __syncthreads();
  a = sh[first];
  for (int w = 1; w < warps; ++w) a = both<kMax>(a, sh[first + w]);
  return a;
}

// (a row of 16384 elements has 64 groups of 8 elements a lane)
template <typename XT, typename FT, int NV, bool kVec>
__global__ void __launch_bounds__(NV == 8 ? 256 : NV == 4 ? 512 : 1024) norm_q8_kernel(const Q8P p) {
  __shared__ float sh[2][32];
  const int per = blockDim.x / (32 * p.warps);  // rows of a CTA
  const int mine = threadIdx.x / (32 * p.warps), t = threadIdx.x % (32 * p.warps);
  const XT *x = static_cast<const XT *>(p.x);
  const FT *f = static_cast<const FT *>(p.f);
  for (long long first = (long long)blockIdx.x * per; first < p.rows; first += (long long)gridDim.x * per) {
    const long long row = first + mine;
    const bool live = row < p.rows;
    float r[NV][8], s = 0.f;
#pragma unroll
    for (int n = 0; n < NV; ++n) load8<XT, kVec>(x + (live ? row * p.x_ld : 0), (n * 32 * p.warps + t) * 8, live ? p.D : 0, r[n]);
    if (f) {
#pragma unroll
      for (int n = 0; n < NV; ++n) {
        float g[8];
        load8<FT, kVec>(f + (live ? row * p.f_ld : 0), (n * 32 * p.warps + t) * 8, live ? p.D : 0, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) r[n][e] += g[e];
      }
    }
    if (p.r && live) {
#pragma unroll
      for (int n = 0; n < NV; ++n)
        store8<XT, kVec>(static_cast<XT *>(p.r) + row * p.D, (n * 32 * p.warps + t) * 8, p.D, r[n]);
    }
    if (p.w) {
#pragma unroll
      for (int n = 0; n < NV; ++n)
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf(r[n][e], r[n][e], s);
      s = over_row<false>(s, sh[0], p.warps);
      const float inv = __frsqrt_rn(__fdiv_rn(s, (float)p.D) + p.eps);
#pragma unroll
      for (int n = 0; n < NV; ++n) {
        float w[8];
        load8<float, kVec>(p.w, (n * 32 * p.warps + t) * 8, p.D, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) r[n][e] = r[n][e] * inv * w[e];
      }
    }
    float m = 0.f;
#pragma unroll
    for (int n = 0; n < NV; ++n)
#pragma unroll
      for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(r[n][e]));
    m = fmaxf(over_row<true>(m, sh[1], p.warps), kFloor);
    const float up = __fdiv_rn(kTop, m);
    if (live) {
#pragma unroll
      for (int n = 0; n < NV; ++n) {
#pragma unroll
        for (int e = 0; e < 8; ++e) r[n][e] *= up;
        store_codes<kVec>(static_cast<uint8_t *>(p.q) + row * p.D, (n * 32 * p.warps + t) * 8, p.D, r[n]);
      }
      if (t == 0) p.scale[row] = m * (1.f / kTop);
    }
    // (the two sums' places are written again only behind the other's barrier; without the
    // norm there is no other)
    if (!p.w && p.warps > 1) __syncthreads();
  }
}

template <typename XT, typename FT, bool kVec>
cudaError_t run(const Q8P &p, int nv, int ctas, int threads, cudaStream_t s) {
  auto kern = nv == 8   ? norm_q8_kernel<XT, FT, kVec ? 8 : 4, kVec>
              : nv == 4 ? norm_q8_kernel<XT, FT, 4, kVec>
              : nv == 2 ? norm_q8_kernel<XT, FT, 2, kVec>
                        : norm_q8_kernel<XT, FT, 1, kVec>;
  RDN_LAUNCH("norm_q8", s, (kern<<<ctas, threads, 0, s>>>(p)));
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_norm_q8(const rdn_norm_q8_args &a, cudaStream_t s) {
  if (a.rows == 0) return cudaSuccess;
  constexpr int kSMs = 152;
  Q8P p{};
  p.rows = a.rows; p.x_ld = a.x_ld; p.f_ld = a.f_ld; p.D = a.D; p.eps = a.eps;
  p.x = a.x; p.f = a.f; p.w = a.w; p.r = a.r_out; p.q = a.q; p.scale = a.scale;
  const size_t xe = a.x_dtype == RDN_BF16 ? 2 : 4, fe = a.f_dtype == RDN_BF16 ? 2 : 4;
  auto on = [](const void *q, size_t bytes) { return !q || (((uintptr_t)q | bytes) & 15) == 0; };
  const bool vec = a.D % 8 == 0 && on(a.x, a.x_ld * xe) && on(a.f, a.f_ld * fe) && on(a.w, 0) && on(a.r_out, 0) &&
                   ((uintptr_t)a.q & 7) == 0;
  // the fewest elements a lane that need no more than 32 warps a row; more, up to 8 groups of 8
  // (4 for rows on single elements), where the rows fill the GPU all the same
  const int groups = (a.D + 255) / 256;
  int nv = 1;
  while (nv < (vec ? 8 : 4) && (groups > 32 * nv || (a.rows * groups > kSMs * 16 * nv && groups > nv))) nv *= 2;
  p.warps = (groups + nv - 1) / nv;
  const int per = p.warps >= 4 ? 1 : 4 / p.warps;
  const int threads = 32 * p.warps * per;
  const long long need = (a.rows + per - 1) / per, most = (long long)kSMs * 4;
  const int ctas = (int)(need < most ? need : most);
  const bool xb = a.x_dtype == RDN_BF16, fb = a.f ? a.f_dtype == RDN_BF16 : xb;
  typedef __nv_bfloat16 bf;
  if (vec)
    return xb ? (fb ? run<bf, bf, true>(p, nv, ctas, threads, s) : run<bf, float, true>(p, nv, ctas, threads, s))
              : (fb ? run<float, bf, true>(p, nv, ctas, threads, s) : run<float, float, true>(p, nv, ctas, threads, s));
  return xb ? (fb ? run<bf, bf, false>(p, nv, ctas, threads, s) : run<bf, float, false>(p, nv, ctas, threads, s))
            : (fb ? run<float, bf, false>(p, nv, ctas, threads, s) : run<float, float, false>(p, nv, ctas, threads, s));
}

}  // namespace rdn
