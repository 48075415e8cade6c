// norm.cu -- the norms after and before a block with its gate and its scaled
// residual, per row of D elements (rms(t) = sqrt(mean(t^2) + eps)):
//     u = f / rms(f) w act(z),   r = x + scale u,   h = r / rms(r) w_next
// and the backward, with i1 = 1 / rms(f), i2 = 1 / rms(r), everything
// recomputed from f, z and x:
//     gr = dr + i2 (w_next dh - r i2^2 mean(w_next dh r));   dx = gr
//     dscale += gr u,  dw_next += dh r i2,  du = scale gr
//     dz = du f i1 w act'(z),  dn = du act(z),  dw += dn f i1
//     df = i1 (w dn - f i1^2 mean(w dn f))
//
// Memory-bound: every operand is read once and every result written once, in
// one pass: a row lives in the registers of TPR = 8 .. 1024 threads, E
// elements each, and its sums go through shuffles and, above a warp, shared
// memory.  Short rows share a CTA.  The backward's CTAs stay for many rows and
// keep their parameter gradients in registers; one partial per row slot goes to
// the workspace and a second kernel joins them in order.
#include "rows.cuh"

namespace rdn {
namespace {

constexpr int kRowThreads = 256;  // threads of a CTA, but for rows that need more

struct NormP {
  long long rows;
  int D, heads, tpr;  // tpr: threads per row (a power of two)
  int gate;
  float eps, scale_const;
  long long f_ld, z_ld, x_ld;
  const void *f, *z, *x, *dr, *dh;
  const float *w, *scale, *w_next;
  void *r_out, *h, *df, *dz, *dx;
  float *part;  // backward: [row slots][3][D]: dw, dscale, dw_next
};

// E elements of a row: element e of thread t.  Vector accesses: groups of V
// consecutive elements, the groups dealt round over the threads; else single
// elements dealt round.
template <int V>
__device__ __forceinline__ int elem(int e, int t, int tpr) { return (e / V * tpr + t) * V + e % V; }

// V fixes the elements a thread holds (the vector of the 2-byte operands, so
// that operands of both sizes agree); a 4-byte operand takes two accesses.
template <typename T, int V, int E>
__device__ __forceinline__ void load_row(const T *row, int D, int t, int tpr, float (&v)[E]) {
  constexpr int A = V == 1 ? 1 : kVec<T> < V ? kVec<T> : V;  // elements per access
  using K = Pack<T, A>;
#pragma unroll
  for (int e = 0; e < E; e += A) {
    const int i = elem<V>(e, t, tpr);
    float a[A];
    K::get(row && i < D ? K::ld(row + i) : K::zero(), a);
#pragma unroll
    for (int k = 0; k < A; ++k) v[e + k] = a[k];
  }
}
template <typename T, int V, int E>
__device__ __forceinline__ void store_row(T *row, int D, int t, int tpr, const float (&v)[E]) {
  constexpr int A = V == 1 ? 1 : kVec<T> < V ? kVec<T> : V;
  using K = Pack<T, A>;
#pragma unroll
  for (int e = 0; e < E; e += A) {
    const int i = elem<V>(e, t, tpr);
    if (i >= D) continue;
    float a[A];
#pragma unroll
    for (int k = 0; k < A; ++k) a[k] = v[e + k];
    K::st(row + i, K::put(a));
  }
}

// Sum over the tpr threads of a row, in every one of them.  `sh`: 32 floats;
// two calls in a row take different ones (the barrier of the second separates
// the reads of the first from the next write there).
__device__ __forceinline__ float row_sum(float v, int tpr, float *sh) {
  for (int o = min(tpr, 32) / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (tpr <= 32) return v;
  const int warp = threadIdx.x >> 5, per = tpr >> 5, first = warp / per * per;
  if ((threadIdx.x & 31) == 0) sh[warp] = v;
  __syncthreads();
  v = sh[first];
  for (int k = 1; k < per; ++k) v += sh[first + k];
  return v;
}

__device__ __forceinline__ float gate_fn(int gate, float z, float s) { return gate ? s : z * s; }
__device__ __forceinline__ float gate_grad(int gate, float z, float s) {
  return gate ? s * (1.f - s) : silu_grad(z, s);
}

template <typename T, typename XT, int V, int E, int THREADS>
__global__ void __launch_bounds__(THREADS) norm_fwd_kernel(NormP p) {
  __shared__ float sh[2][32];
  const int tpr = p.tpr, t = threadIdx.x % tpr, per = blockDim.x / tpr;
  const long long row = (long long)blockIdx.x * per + threadIdx.x / tpr;
  const bool on = row < p.rows;
  const long long r0 = on ? row : 0;
  float f[E], z[E], x[E];
  const float invD = 1.f / (float)p.D;
  if (p.x) load_row<XT, V>((const XT *)p.x + r0 * p.x_ld, p.D, t, tpr, x);
  if (p.f) {
    load_row<T, V>((const T *)p.f + r0 * p.f_ld, p.D, t, tpr, f);
    if (p.z) load_row<T, V>((const T *)p.z + r0 * p.z_ld, p.D, t, tpr, z);
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) ss = fmaf(f[e], f[e], ss);
    const float inv = rsqrtf(fmaf(row_sum(ss, tpr, sh[0]), invD, p.eps));
    const float *w = p.w + (p.heads > 1 ? r0 % p.heads * p.D : 0);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int i = elem<V>(e, t, tpr);
      if (i >= p.D) continue;
      float u = f[e] * inv * __ldg(w + i);
      if (p.z) u *= gate_fn(p.gate, z[e], sigmoidf(z[e]));
      if (p.x) u = fmaf(p.scale ? __ldg(p.scale + i) : p.scale_const, u, x[e]);
      f[e] = u;
    }
    if (on) {
      if (p.x) {
        if (p.r_out) store_row<XT, V>((XT *)p.r_out + row * p.D, p.D, t, tpr, f);
      } else {
        store_row<T, V>((T *)p.r_out + row * p.D, p.D, t, tpr, f);
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = x[e];
  }
  if (!p.h) return;
  float ss = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) ss = fmaf(f[e], f[e], ss);  // (zero past D)
  const float inv = rsqrtf(fmaf(row_sum(ss, tpr, sh[1]), invD, p.eps));
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int i = elem<V>(e, t, tpr);
    if (i < p.D) f[e] *= inv * __ldg(p.w_next + i);
  }
  if (on) store_row<T, V>((T *)p.h + row * p.D, p.D, t, tpr, f);
}

template <typename T, typename XT, int V, int E, int THREADS>
__global__ void __launch_bounds__(THREADS) norm_bwd_kernel(NormP p) {
  __shared__ float sh[4][32];
  const int tpr = p.tpr, t = threadIdx.x % tpr, per = blockDim.x / tpr;
  const long long slot = (long long)blockIdx.x * per + threadIdx.x / tpr;
  const long long slots = (long long)gridDim.x * per;  // (a multiple of heads)
  const float invD = 1.f / (float)p.D;
  const float *w = p.w + (p.heads > 1 ? slot % p.heads * p.D : 0);
  float aw[E], as[E], an[E];  // dw, dscale, dw_next
#pragma unroll
  for (int e = 0; e < E; ++e) aw[e] = as[e] = an[e] = 0.f;
  for (long long base = slot - threadIdx.x / tpr; base < p.rows; base += slots) {
    const long long row = base + threadIdx.x / tpr;
    const bool on = row < p.rows;
    const long long r0 = on ? row : 0;
    float f[E], z[E], r[E], g[E], inv = 0.f;
    if (p.x) load_row<XT, V>((const XT *)p.x + r0 * p.x_ld, p.D, t, tpr, r);
    if (p.f) load_row<T, V>((const T *)p.f + r0 * p.f_ld, p.D, t, tpr, f);
    if (p.z) load_row<T, V>((const T *)p.z + r0 * p.z_ld, p.D, t, tpr, z);
    if (p.x) load_row<XT, V>(p.dr ? (const XT *)p.dr + r0 * p.D : nullptr, p.D, t, tpr, g);
    else load_row<T, V>(p.dr ? (const T *)p.dr + r0 * p.D : nullptr, p.D, t, tpr, g);
    float dh[E];
    if (p.dh) load_row<T, V>((const T *)p.dh + r0 * p.D, p.D, t, tpr, dh);
    if (p.f) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) ss = fmaf(f[e], f[e], ss);
      inv = rsqrtf(fmaf(row_sum(ss, tpr, sh[0]), invD, p.eps));
    }
    if (p.dh) {  // r, then its gradient
      float s2 = 0.f, sd = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int i = elem<V>(e, t, tpr);
        if (i >= p.D) continue;
        if (p.f) {
          float u = f[e] * inv * __ldg(w + i);
          if (p.z) u *= gate_fn(p.gate, z[e], sigmoidf(z[e]));
          r[e] = p.x ? fmaf(p.scale ? __ldg(p.scale + i) : p.scale_const, u, r[e]) : u;
        }
        s2 = fmaf(r[e], r[e], s2);
        sd = fmaf(__ldg(p.w_next + i) * dh[e], r[e], sd);
      }
      const float i2 = rsqrtf(fmaf(row_sum(s2, tpr, sh[1]), invD, p.eps));
      const float m = row_sum(sd, tpr, sh[2]) * invD * i2 * i2;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int i = elem<V>(e, t, tpr);
        if (i >= p.D) continue;
        if (on) an[e] = fmaf(dh[e] * i2, r[e], an[e]);
        g[e] = fmaf(i2, fmaf(-r[e], m, __ldg(p.w_next + i) * dh[e]), g[e]);
      }
    }
    if (p.x && on) store_row<XT, V>((XT *)p.dx + row * p.D, p.D, t, tpr, g);
    if (!p.f) continue;
    float sd = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int i = elem<V>(e, t, tpr);
      if (i >= p.D) {
        f[e] = g[e] = 0.f;
        continue;
      }
      const float fi = f[e] * inv, wi = __ldg(w + i);
      float act = 1.f, sz = 0.f;
      if (p.z) {
        sz = sigmoidf(z[e]);
        act = gate_fn(p.gate, z[e], sz);
      }
      if (p.x) {
        if (on) as[e] = fmaf(g[e], fi * wi * act, as[e]);
        g[e] *= p.scale ? __ldg(p.scale + i) : p.scale_const;
      }
      if (p.z) z[e] = g[e] * fi * wi * gate_grad(p.gate, z[e], sz);
      const float dn = g[e] * act;
      if (on) aw[e] = fmaf(dn, fi, aw[e]);
      g[e] = dn * wi;
      sd = fmaf(g[e], fi, sd);
      f[e] = fi;
    }
    const float m = row_sum(sd, tpr, sh[3]) * invD;
    if (on) {
      if (p.z) store_row<T, V>((T *)p.dz + row * p.D, p.D, t, tpr, z);
#pragma unroll
      for (int e = 0; e < E; ++e) f[e] = inv * fmaf(-f[e], m, g[e]);
      store_row<T, V>((T *)p.df + row * p.D, p.D, t, tpr, f);
    }
  }
  float *mine = p.part + (size_t)slot * 3 * p.D;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int i = elem<V>(e, t, tpr);
    if (i >= p.D) continue;
    if (p.f) mine[i] = aw[e];
    if (p.scale) mine[p.D + i] = as[e];
    if (p.dh) mine[2 * p.D + i] = an[e];
  }
}

// dw [heads, D], dscale and dw_next [D] from the row slots' partials, in order.
__global__ void __launch_bounds__(512) norm_grad_kernel(const float *__restrict__ part, int D, int heads, int slots,
                                                        float *dw, float *dscale, float *dw_next) {
  __shared__ float sh[16][32];
  const int which = blockIdx.z, head = blockIdx.y;
  const int i = blockIdx.x * 32 + threadIdx.x;
  float *out = which == 0 ? dw : which == 1 ? dscale : dw_next;
  if (!out || (which && head)) return;
  const int first = which ? 0 : head, stride = which ? 1 : heads;
  float a = 0.f;
  if (i < D)
    for (long long q = first + (long long)threadIdx.y * stride; q < slots; q += 16ll * stride)
      a += part[((size_t)q * 3 + which) * D + i];
  sh[threadIdx.y][threadIdx.x] = a;
  __syncthreads();
  if (threadIdx.y || i >= D) return;
#pragma unroll
  for (int y = 1; y < 16; ++y) a += sh[y][threadIdx.x];
  out[(size_t)head * D + i] = a;
}

struct NormPlan {
  int elems;              // of a row per thread
  int tpr, threads, per;  // threads per row and per CTA, rows per CTA
  int ctas;               // of the backward
};
int gcd(int a, int b) { return b ? gcd(b, a % b) : a; }
cudaError_t norm_plan(const rdn_norm_args &a, NormPlan *pl) {
  int nsm = 0;
  const cudaError_t e = sm_count(&nsm);
  pl->elems = a.D <= 8 * 1024 ? 8 : 16;
  pl->tpr = 8;
  while (pl->tpr * pl->elems < a.D) pl->tpr *= 2;
  pl->threads = pl->tpr > kRowThreads ? pl->tpr : kRowThreads;
  pl->per = pl->threads / pl->tpr;
  // a few CTAs per SM, as many slots as a multiple of the heads
  long long ctas = (long long)(e == cudaSuccess ? nsm : 152) * (pl->threads <= 256 ? 2 : 1);
  const int step = a.heads / gcd(a.heads, pl->per);
  const long long need = ((a.rows + pl->per - 1) / pl->per + step - 1) / step * step;
  ctas = (ctas + step - 1) / step * step;
  pl->ctas = (int)(ctas < need ? ctas : need);
  return e;
}

NormP norm_params(const rdn_norm_args &a, const NormPlan &pl) {
  NormP p{};
  p.rows = a.rows; p.D = a.D; p.heads = a.heads; p.tpr = pl.tpr; p.gate = a.gate;
  p.eps = a.eps; p.scale_const = a.scale_const;
  p.f_ld = a.f_ld; p.z_ld = a.z_ld; p.x_ld = a.x_ld;
  p.f = a.f; p.z = a.f ? a.z : nullptr; p.x = a.x; p.dr = a.dr;
  p.dh = a.w_next ? a.dh : nullptr;
  p.w = a.w; p.scale = a.f && a.x ? a.scale : nullptr; p.w_next = a.w_next;
  p.r_out = a.r_out; p.h = a.w_next ? a.h : nullptr;
  p.df = a.df; p.dz = a.dz; p.dx = a.dx;
  p.part = static_cast<float *>(a.workspace);
  return p;
}

bool norm_vec(const rdn_norm_args &a, bool bwd) {
  if (a.D % 8) return false;  // (rows on 16 bytes in either type)
  const size_t es = a.dtype == RDN_BF16 ? 2 : 4, xs = a.x_dtype == RDN_BF16 ? 2 : 4;
  auto on = [](const void *p, size_t bytes) { return !p || (((uintptr_t)p | bytes) & 15) == 0; };
  if (!on(a.f, a.f_ld * es) || !on(a.z, a.z_ld * es) || !on(a.x, a.x_ld * xs)) return false;
  if (!bwd) return on(a.r_out, 0) && on(a.h, 0);
  return on(a.dr, 0) && on(a.dh, 0) && on(a.df, 0) && on(a.dz, 0) && on(a.dx, 0);
}

template <typename T, typename XT, int V, int E, int THREADS>
cudaError_t norm_t(const rdn_norm_args &a, const NormPlan &pl, bool bwd, cudaStream_t s) {
  const NormP p = norm_params(a, pl);
  if (!bwd) {
    const unsigned grid = (unsigned)((a.rows + pl.per - 1) / pl.per);
    RDN_LAUNCH("norm_fwd", s, (norm_fwd_kernel<T, XT, V, E, THREADS><<<grid, pl.threads, 0, s>>>(p)));
    return cudaGetLastError();
  }
  RDN_LAUNCH("norm_bwd", s, (norm_bwd_kernel<T, XT, V, E, THREADS><<<pl.ctas, pl.threads, 0, s>>>(p)));
  const dim3 grid((a.D + 31) / 32, a.heads, 3);
  RDN_LAUNCH("norm_grad", s,
             (norm_grad_kernel<<<grid, dim3(32, 16), 0, s>>>(p.part, a.D, a.heads, pl.ctas * pl.per,
                                                             a.f ? a.dw : nullptr, p.scale ? a.dscale : nullptr,
                                                             p.dh ? a.dw_next : nullptr)));
  return cudaGetLastError();
}
template <typename T, typename XT, int V>
cudaError_t norm_v(const rdn_norm_args &a, bool bwd, cudaStream_t s) {
  NormPlan pl;
  const cudaError_t e = norm_plan(a, &pl);
  if (e != cudaSuccess) return e;
  if (pl.elems == 16) return norm_t<T, XT, V, 16, 1024>(a, pl, bwd, s);
  return pl.threads == kRowThreads ? norm_t<T, XT, V, 8, kRowThreads>(a, pl, bwd, s)
                                   : norm_t<T, XT, V, 8, 1024>(a, pl, bwd, s);
}
template <typename T, typename XT>
cudaError_t norm_x(const rdn_norm_args &a, bool bwd, cudaStream_t s) {
  return norm_vec(a, bwd) ? norm_v<T, XT, 8>(a, bwd, s) : norm_v<T, XT, 1>(a, bwd, s);
}

}  // namespace

size_t norm_bwd_bytes(const rdn_norm_args &a) {
  NormPlan pl;
  (void)norm_plan(a, &pl);  // (without a device: the plan of 152 SMs)
  return round256(sizeof(float) * 3 * (size_t)pl.ctas * pl.per * a.D);
}

cudaError_t launch_norm(const rdn_norm_args &a, bool bwd, cudaStream_t s) {
  const bool xf = a.x_dtype == RDN_F32;
  if (a.dtype == RDN_BF16)
    return xf ? norm_x<__nv_bfloat16, float>(a, bwd, s) : norm_x<__nv_bfloat16, __nv_bfloat16>(a, bwd, s);
  return xf ? norm_x<float, float>(a, bwd, s) : norm_x<float, __nv_bfloat16>(a, bwd, s);
}

}  // namespace rdn
