// norm_q8.cu -- the residual's addition and the norm before a block, with an output in
// 8 bits and a scale per row (include/rdn.h, rdn_norm_q8):
//     r = x + f,  h = r / rms(r) w,  scale = max |h| / 448,  q = e4m3(h / scale).
// One pass: a row stays in the registers of its lanes between the sum of squares, the
// maximum and the codes, so x and f are read once and r, q written once; it is bound by
// HBM.  Where rows are many, a lane has 64 elements: of one row (2048 elements and up, by
// one warp and more), or 8 to 32 of each of 8 to 2 rows, whose loads are then in flight
// together (rows of up to 128 elements have 8 or 16 lanes).  Where there are fewer rows than
// fill the GPU a lane has 8, for then latency counts.
// 32768 rows of 2048 in bf16: 77 us, 6.1 TB/s.
#include <cuda_fp8.h>

#include "q8_rows.cuh"
#include "rows.cuh"

namespace rdn {
namespace {

constexpr float kTop = 448.f, kFloor = 0x1p-100f;

struct Q8P {
  long long rows, x_ld, f_ld;
  long long inner;  // rows before the last near_end_rows(D)
  int D, lanes;     // of a row: 8, 16, or a multiple of 32
  float eps;
  const void *x, *f;
  const float *w;
  void *r, *q;
  float *scale;
};

// 8 elements as loaded
template <typename T>
struct Raw8;
template <>
struct Raw8<__nv_bfloat16> {
  uint4 a;
  __device__ void zero() { a = make_uint4(0u, 0u, 0u, 0u); }
  __device__ void load(const __nv_bfloat16 *p) { a = Pack<__nv_bfloat16, 8>::ld(p); }
  __device__ void get(float (&v)[8]) const { Pack<__nv_bfloat16, 8>::get(a, v); }
  __device__ void put(const float (&v)[8]) { a = Pack<__nv_bfloat16, 8>::put(v); }
};
template <>
struct Raw8<float> {
  float4 a, b;
  __device__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ void load(const float *p) { a = Pack<float, 4>::ld(p); b = Pack<float, 4>::ld(p + 4); }
  __device__ void get(float (&v)[8]) const {
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
  __device__ void put(const float (&v)[8]) {
    a = make_float4(v[0], v[1], v[2], v[3]);
    b = make_float4(v[4], v[5], v[6], v[7]);
  }
};
template <typename T, int kLie>
__device__ __forceinline__ void load8(const T *row, int i, int D, bool near_end, Raw8<T> &raw) {
  raw.zero();
  const Read how = read_of<kLie>(i, D, near_end);
  if (how == kGroup) {
    raw.load(row + i);
    if (kLie == kShifted && (i < 0 || i + 8 > D)) {
      float v[8];
      raw.get(v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = i + e >= 0 && i + e < D ? v[e] : 0.f;
      raw.put(v);
    }
  } else if (how == kElements) {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = i + e >= 0 && i + e < D ? to_f32<T>(row[i + e]) : 0.f;
    raw.put(v);
  }
}
// (the weight is on 16 bytes where all the rows are; elsewhere what is outside the row is not used)
template <int kLie>
__device__ __forceinline__ void load_weight(const float *w, int i, int D, float (&v)[8]) {
  if (kLie == kVectors) {
    Raw8<float> raw;
    load8<float, kVectors>(w, i, D, true, raw);
    raw.get(v);
  } else if (kLie == kShifted && i >= 0 && i + 8 <= D) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __ldg(w + i + e);
  } else if (i < D && i > -8) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __ldg(w + min(max(i + e, 0), D - 1));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.f;
  }
}
template <typename T, int kLie>
__device__ __forceinline__ void store8(T *row, int i, int D, const float (&v)[8]) {
  if (kLie != kSingle && whole<kLie>(i, D)) {
    if constexpr (sizeof(T) == 2) {
      Pack<T, 8>::st(row + i, Pack<T, 8>::put(v));
    } else {
      *reinterpret_cast<float4 *>(row + i) = make_float4(v[0], v[1], v[2], v[3]);
      *reinterpret_cast<float4 *>(row + i + 4) = make_float4(v[4], v[5], v[6], v[7]);
    }
  } else if (kLie != kVectors && i < D && i > -8) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (i + e >= 0 && i + e < D) row[i + e] = from_f32<T>(v[e]);
  }
}
template <int kLie>
__device__ __forceinline__ void store_codes(uint8_t *row, int i, int D, const float (&v)[8]) {
  uint32_t c[2] = {0u, 0u};
#pragma unroll
  for (int e = 0; e < 8; e += 2)
    c[e / 4] |= (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(v[e], v[e + 1]), __NV_SATFINITE, __NV_E4M3)
                << (e % 4 * 8);
  if (kLie != kSingle && whole<kLie>(i, D)) {
    *reinterpret_cast<uint2 *>(row + i) = make_uint2(c[0], c[1]);
  } else if (kLie != kVectors && i < D && i > -8) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (i + e >= 0 && i + e < D) row[i + e] = (uint8_t)(c[e / 4] >> (e % 4 * 8));
  }
}

template <bool kMax>
__device__ __forceinline__ float both(float a, float b) { return kMax ? fmaxf(a, b) : a + b; }
// Over the row's lanes (its warps in order), for every one of them.
template <bool kMax>
__device__ __forceinline__ float over_row(float a, float *sh, int lanes) {
#pragma unroll
  for (int o = 16; o; o >>= 1)
    if (o < lanes) a = both<kMax>(a, __shfl_xor_sync(0xffffffffu, a, o));
  if (lanes <= 32) return a;
  const int warps = lanes / 32, warp = threadIdx.x >> 5, first = warp / warps * warps;
  if ((threadIdx.x & 31) == 0) sh[warp] = a;
  __syncthreads();
  a = sh[first];
  for (int w = 1; w < warps; ++w) a = both<kMax>(a, sh[first + w]);
  return a;
}

// R rows of a lane, NV groups of 8 elements each.  (A row of 16384 elements has 64 groups a lane of one warp, a
// shifted one 65.)
template <typename XT, typename FT, int NV, int R, int kLie>
__global__ void __launch_bounds__(R > 1 ? 128 : NV == 8 ? 256 : NV >= 3 ? 544 : 1024, R > 1 ? 4 : NV == 8 ? 2 : 1)
    norm_q8_kernel(const Q8P p) {
  __shared__ float sh[2][32];
  const int lanes = p.lanes, per = blockDim.x / lanes;  // rows of a CTA at one time, R times
  const int mine = threadIdx.x / lanes, t = threadIdx.x % lanes;
  const XT *x = static_cast<const XT *>(p.x);
  const FT *f = static_cast<const FT *>(p.f);
  for (long long first = (long long)blockIdx.x * per * R; first < p.rows; first += (long long)gridDim.x * per * R) {
    auto row_of = [&](int k) { return first + k * per + mine; };
    auto i_of = [&](int k, int n) {
      return place<kLie>(n, t, lanes, kLie == kShifted ? (int)(row_of(k) * p.D & 7) : 0);
    };
    // the rows' loads go out before the first is waited for (fp32 rows leave no registers for f's beside them)
    constexpr bool kAhead = sizeof(XT) == 2;
    Raw8<XT> rx[R][NV];
    Raw8<FT> rf[kAhead ? R : 1][kAhead ? NV : 1];
    auto load_f = [&](int k, int n, Raw8<FT> &raw) {
      const bool live = row_of(k) < p.rows;
      load8<FT, kLie>(f + (live ? row_of(k) * p.f_ld : 0), i_of(k, n), live ? p.D : -8, row_of(k) >= p.inner, raw);
    };
#pragma unroll
    for (int k = 0; k < R; ++k) {
      const bool live = row_of(k) < p.rows;
      const XT *row = x + (live ? row_of(k) * p.x_ld : 0);
#pragma unroll
      for (int n = 0; n < NV; ++n)
        load8<XT, kLie>(row, i_of(k, n), live ? p.D : -8, row_of(k) >= p.inner, rx[k][n]);
    }
    if (kAhead && f) {
#pragma unroll
      for (int k = 0; k < R; ++k)
#pragma unroll
        for (int n = 0; n < NV; ++n) load_f(k, n, rf[kAhead ? k : 0][kAhead ? n : 0]);
    }
    float r[R][NV][8];
#pragma unroll
    for (int k = 0; k < R; ++k)
#pragma unroll
      for (int n = 0; n < NV; ++n) {
        rx[k][n].get(r[k][n]);
        if (kAhead && f) {
          float g[8];
          rf[kAhead ? k : 0][kAhead ? n : 0].get(g);
#pragma unroll
          for (int e = 0; e < 8; ++e) r[k][n][e] += g[e];
        }
      }
    if (!kAhead && f) {
#pragma unroll
      for (int k = 0; k < R; ++k)
#pragma unroll
        for (int n = 0; n < NV; ++n) {
          float g[8];
          load_f(k, n, rf[0][0]);
          rf[0][0].get(g);
#pragma unroll
          for (int e = 0; e < 8; ++e) r[k][n][e] += g[e];
        }
    }
    if (p.r) {
#pragma unroll
      for (int k = 0; k < R; ++k)
        if (row_of(k) < p.rows) {
          XT *rr = static_cast<XT *>(p.r) + row_of(k) * p.D;
#pragma unroll
          for (int n = 0; n < NV; ++n) store8<XT, kLie>(rr, i_of(k, n), p.D, r[k][n]);
        }
    }
    if (p.w) {
      float inv[R];
#pragma unroll
      for (int k = 0; k < R; ++k) {
        float s = 0.f;
#pragma unroll
        for (int n = 0; n < NV; ++n)
#pragma unroll
          for (int e = 0; e < 8; ++e) s = fmaf(r[k][n][e], r[k][n][e], s);
        s = over_row<false>(s, sh[0], lanes);
        inv[k] = __frsqrt_rn(__fdiv_rn(s, (float)p.D) + p.eps);
      }
#pragma unroll
      for (int n = 0; n < NV; ++n) {
        float w[8];
        if (kLie != kShifted) load_weight<kLie>(p.w, i_of(0, n), p.D, w);
#pragma unroll
        for (int k = 0; k < R; ++k) {
          if (kLie == kShifted) load_weight<kLie>(p.w, i_of(k, n), p.D, w);  // (each row's place is its own)
#pragma unroll
          for (int e = 0; e < 8; ++e) r[k][n][e] = r[k][n][e] * inv[k] * w[e];
        }
      }
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
      float m = 0.f;
#pragma unroll
      for (int n = 0; n < NV; ++n)
#pragma unroll
        for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(r[k][n][e]));
      m = fmaxf(over_row<true>(m, sh[1], lanes), kFloor);
      const float up = __fdiv_rn(kTop, m);
      if (row_of(k) < p.rows) {
        uint8_t *qr = static_cast<uint8_t *>(p.q) + row_of(k) * p.D;
#pragma unroll
        for (int n = 0; n < NV; ++n) {
#pragma unroll
          for (int e = 0; e < 8; ++e) r[k][n][e] *= up;
          store_codes<kLie>(qr, i_of(k, n), p.D, r[k][n]);
        }
        if (t == 0) p.scale[row_of(k)] = m * (1.f / kTop);
      }
    }
    // (rows of several warps, R = 1: the two sums' places are written again only behind the other's
    // barrier; without the norm there is no other)
    if (!p.w && lanes > 32) __syncthreads();
  }
}

struct Shape {
  int nv, r;
};
template <typename XT, typename FT, int kLie>
cudaError_t run(const Q8P &p, Shape h, int ctas, int threads, cudaStream_t s) {
  auto kern = norm_q8_kernel<XT, FT, 1, 1, kLie>;
  if (h.nv == 2) kern = norm_q8_kernel<XT, FT, 2, 1, kLie>;
  if (h.nv == 4) kern = norm_q8_kernel<XT, FT, 4, 1, kLie>;
  if constexpr (kLie == kShifted)
    if (h.nv == 3) kern = norm_q8_kernel<XT, FT, 3, 1, kLie>;
  if constexpr (kLie == kVectors) {
    if (h.nv == 8) kern = norm_q8_kernel<XT, FT, 8, 1, kVectors>;
    if (h.r == 2) kern = norm_q8_kernel<XT, FT, 4, 2, kVectors>;
    if (h.r == 4) kern = norm_q8_kernel<XT, FT, 2, 4, kVectors>;
    if (h.r == 8) kern = norm_q8_kernel<XT, FT, 1, 8, kVectors>;
  }
  RDN_LAUNCH("norm_q8", s, (kern<<<ctas, threads, 0, s>>>(p)));
  return cudaGetLastError();
}
template <typename XT, typename FT>
cudaError_t run(const Q8P &p, int lie, Shape h, int ctas, int threads, cudaStream_t s) {
  return lie == kVectors ? run<XT, FT, kVectors>(p, h, ctas, threads, s)
         : lie == kShifted ? run<XT, FT, kShifted>(p, h, ctas, threads, s)
                           : run<XT, FT, kSingle>(p, h, ctas, threads, s);
}

}  // namespace

cudaError_t launch_norm_q8(const rdn_norm_q8_args &a, cudaStream_t s) {
  if (a.rows == 0) return cudaSuccess;
  constexpr int kSMs = 152;
  Q8P p{};
  p.rows = a.rows; p.inner = a.rows - near_end_rows(a.D); p.x_ld = a.x_ld; p.f_ld = a.f_ld; p.D = a.D; p.eps = a.eps;
  p.x = a.x; p.f = a.f; p.w = a.w; p.r = a.r_out; p.q = a.q; p.scale = a.scale;
  const size_t xe = a.x_dtype == RDN_BF16 ? 2 : 4, fe = a.f_dtype == RDN_BF16 ? 2 : 4;
  auto on = [](const void *q, size_t bytes) { return !q || (((uintptr_t)q | bytes) & 15) == 0; };
  const bool bases = on(a.x, 0) && on(a.f, 0) && on(a.r_out, 0) && ((uintptr_t)a.q & 7) == 0;
  const bool vec = bases && a.D % 8 == 0 && on(a.x, a.x_ld * xe) && on(a.f, a.f_ld * fe) && on(a.w, 0);
  const bool shifted = bases && (a.x_ld - a.D) % 8 == 0 && (!a.f || (a.f_ld - a.D) % 8 == 0);
  const int lie = vec ? kVectors : shifted ? kShifted : kSingle;
  // few rows: 8 elements a lane, or what it takes to need no more than 32 warps a row; more, up to 64 (32 on
  // single elements), where the rows fill the GPU's 152 x 16 warps all the same, and then several rows a lane
  const int span = a.D + (lie == kShifted ? 7 : 0), groups = (span + 255) / 256;  // (groups of 8 that a row touches)
  Shape h{1, 1};
  while (h.nv < (vec ? 8 : 4) && (groups > 32 * h.nv || (a.rows * groups > kSMs * 16 * h.nv && groups > h.nv)))
    h.nv *= 2;
  // (of a shifted row of 2055 elements four groups a lane would leave three of twelve without any: 231 us, with
  // three 203; wider rows, 17 groups and more, have few idle ones: 4097 elements 214 and 213, 8191 224 and 258)
  if (lie == kShifted && h.nv == 4 && groups <= 16 && (groups + 2) / 3 * 3 < (groups + 3) / 4 * 4) h.nv = 3;
  p.lanes = 32 * ((groups + h.nv - 1) / h.nv);
  if (groups == 1) p.lanes = span <= 64 ? 8 : span <= 128 ? 16 : 32;
  if (vec && p.lanes <= 32 && h.nv < 8 && a.rows * p.lanes / 32 * h.nv >= kSMs * 16 * 8) h.r = 8 / h.nv;
  const int per = p.lanes >= 128 ? 1 : 128 / p.lanes;
  const int threads = p.lanes * per;
  // (512 threads an SM with 64 elements a lane, 128 registers; else more)
  const int fit = (vec && h.nv * h.r == 8 ? 512 : 1024) / threads;
  const long long need = (a.rows + per * h.r - 1) / (per * h.r), most = (long long)kSMs * (fit > 1 ? fit : 1);
  const int ctas = (int)(need < most ? need : most);
  const bool xb = a.x_dtype == RDN_BF16, fb = a.f ? a.f_dtype == RDN_BF16 : xb;
  typedef __nv_bfloat16 bf;
  if (xb) return fb ? run<bf, bf>(p, lie, h, ctas, threads, s) : run<bf, float>(p, lie, h, ctas, threads, s);
  return fb ? run<float, bf>(p, lie, h, ctas, threads, s) : run<float, float>(p, lie, h, ctas, threads, s);
}

}  // namespace rdn
