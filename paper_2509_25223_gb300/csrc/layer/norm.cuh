// norm.cuh -- the norms after and before a block with its gate and its scaled
// residual, per row of D elements (rms(t) = sqrt(mean(t^2) + eps)):
//     u = f / rms(f) w act(z),   r = x + scale u,   h = r / rms(r) w_next
// and the backward, with i1 = 1 / rms(f), i2 = 1 / rms(r), v = f i1 act(z),
// c = scale w, everything recomputed from f, z and x:
//     r = x + c v,   gr = dr + i2 (w_next dh - r i2^2 mean(w_next dh r));   dx = gr
//     dw_next += dh r i2,   q += gr v:  dw = scale q, dscale = w q (both are constant
//         over the rows, so one sum over the rows serves both)
//     dz = gr c f i1 act'(z),   gw = gr c act(z)
//     df = i1 (gw - f i1^2 mean(gw f))
//
// Memory-bound: every operand is read once and every result written once, in
// one pass.  A row belongs to 8, 16 or whole warps of threads of E = 8 elements (one
// 16-byte access of a 2-byte operand): its sums go through shuffles and, above a
// warp, shared memory; rows too long for a CTA are shared by the CTAs of a
// cluster, which write their warps' sums into each other's shared memory.  The
// CTAs stay for many rows: the parameters of a thread's columns and, in the
// backward, the sums of their gradients stay in its registers, and the next row's
// loads are in flight while one is worked on.
// (A warp per row of 2048 with 64 elements a lane needs no barrier but reads
// the parameters again for every row, as much L1 traffic as the operands:
// forward of 32768 x 2048 rows 186 us instead of 124.)  Each row slot's partial
// gradients go to the workspace; a second kernel joins them in order.
//
// bf16, 32768 rows of 2048 with gate, residual and next norm: forward 124 us (671 MB,
// 5.4 TB/s, 80 % of a copy's rate), backward 219 (1.07 GB, 4.9 TB/s, 72 %); 524288
// gated rows of 128: 77 (403 MB, 5.2 TB/s) and 108 (671 MB, 6.2 TB/s).  HBM bounds
// them but for the backward of the wide rows, where three sums over the row follow
// one another: their shuffles and barriers leave 16 warps per SM at half of the
// issue slots.
#pragma once
#include <type_traits>

#include "rows.cuh"
#include "tc_common.cuh"

namespace rdn {
namespace norm {

struct NormP {
  long long rows;
  int D, heads, tpr;  // tpr: threads per row and CTA (8, 16 or a multiple of 32)
  int split, cols;    // CTAs (of a cluster) that share a row, columns of each
  int mode;           // MODE of the call
  float eps, scale_const;
  long long f_ld, z_ld, x_ld;
  const void *f, *z, *x, *dr, *dh;
  const float *w, *scale, *w_next;
  void *r_out, *h, *df, *dz, *dx;
  float *part;  // backward: [row slots][2][D]: q, dw_next
};

// What a call has: the gate (0 none, 1 SiLU, 2 sigmoid), and these bits.  Fixed at
// compile time, or read from NormP::mode (kAny; kSplit: rows shared by the CTAs of
// a cluster).
constexpr int kF = 4, kX = 8, kH = 16, kAny = -1, kSplit = -2;
// Most threads of a CTA: 512, of 128 registers, or 384, of 168: for single elements,
// whose addresses take registers, in the backward for 4-byte operands where a row
// has so few, and for shared rows.  (With 128 registers those spill: backward of 5979
// rows of 2055 bf16 305 us instead of 136, of fp32 244 instead of 66; but rows of 4096 with
// an fp32 residual, shared by two CTAs instead, 157 us, in one of 512 threads 79.)
// At 512 threads the backward with residual and next norm spills 28 bytes in bf16; rows
// above 3072 columns with 4-byte operands, which take those threads too, up to 276.
// Rows of 4104 to 8192 have a CTA of up to 1024 in the forward (46 us for 1500 of 8192,
// shared by three CTAs 93) and are shared in the backward (147, in one CTA 169).
constexpr int kThreads = 512, kFewThreads = 384, kMostThreads = 1024, kSplitMost = 6;
constexpr bool few_threads(bool vec, bool bwd, bool any_f32, int tpr) {
  return !vec || (bwd && any_f32 && tpr <= kFewThreads);
}
// Rows whose loads a thread has in flight: two where its registers hold them.
template <int V, int E, int MODE, bool BWD>
constexpr int kAhead = V == 8 && E == 8 && MODE >= 0 && !(BWD && (MODE & (kX | kH))) ? 2 : 1;
template <int MODE>
struct Has {
  int m;
  __device__ __forceinline__ explicit Has(const NormP &p) : m(MODE < 0 ? p.mode : MODE) {}
  __device__ __forceinline__ int gate() const { return (MODE < 0 ? m : MODE) & 3; }
  __device__ __forceinline__ bool f() const { return (MODE < 0 ? m : MODE) & kF; }
  __device__ __forceinline__ bool x() const { return (MODE < 0 ? m : MODE) & kX; }
  __device__ __forceinline__ bool h() const { return (MODE < 0 ? m : MODE) & kH; }
};

// A thread's E elements of a row, as loaded: groups of V consecutive elements,
// the groups dealt round over the row's threads (V = 8: 16-byte accesses, two of
// them for 4-byte elements; V = 1: single elements).  `at` is the thread's first
// element of the row, `left` the elements from there to its end (0: a row past the
// last, or an operand that is not given: zeros).
template <typename T, int V, int E>
struct Part {
  static constexpr int A = V == 1 ? 1 : kVec<T>;  // elements per access
  using K = Pack<T, A>;
  typename K::Raw raw[E / A];
  __device__ __forceinline__ static int offset(int a, int tpr) { return a * A / V * tpr * V + a * A % V; }
  __device__ __forceinline__ void load(const T *at, int left, int tpr) {
#pragma unroll
    for (int a = 0; a < E / A; ++a) raw[a] = offset(a, tpr) < left ? K::ld(at + offset(a, tpr)) : K::zero();
  }
  // elements 2 k and 2 k + 1
  __device__ __forceinline__ f2 pair(int k) const {
    if constexpr (A == 1) {
      return pack2(to_f32<T>(raw[2 * k]), to_f32<T>(raw[2 * k + 1]));
    } else {
      float v[A];
      K::get(raw[2 * k / A], v);
      return pack2(v[2 * k % A], v[2 * k % A + 1]);
    }
  }
};
template <typename T, int V, int E>
__device__ __forceinline__ void store_part(T *at, int left, int tpr, const f2 (&p)[E / 2]) {
  using Pt = Part<T, V, E>;
  using K = typename Pt::K;
#pragma unroll
  for (int a = 0; a < E / Pt::A; ++a) {
    if (Pt::offset(a, tpr) >= left) continue;
    float v[Pt::A];
#pragma unroll
    for (int k = 0; k < Pt::A; ++k) {
      float lo, hi;
      unpack2(p[(a * Pt::A + k) / 2], lo, hi);
      v[k] = (a * Pt::A + k) & 1 ? hi : lo;
    }
    K::st(at + Pt::offset(a, tpr), K::put(v));
  }
}
// a parameter row's elements from column col on (zero past the row's end, or the CTA's)
template <int V, int E>
__device__ __forceinline__ void load_param(const float *w, int col, int left, int tpr, f2 (&v)[E / 2]) {
  Part<float, V, E> p;
  p.load(w + col, left, tpr);
#pragma unroll
  for (int k = 0; k < E / 2; ++k) v[k] = p.pair(k);
}
// A word of the shared memory of CTA `rank` of the cluster, at the place of `mine` here.
__device__ __forceinline__ void put_cluster(float *mine, int rank, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(tc::map_rank(mine, (uint32_t)rank)), "f"(v) : "memory");
}

// Sums over the tpr threads of a row, in every one of them.  Calls take the two
// halves of sh in turn (n: their number): the barrier of the call between
// separates the reads of one from the next write to the same half.  sh is zero
// past the CTA's warps (SPLIT: past those of the cluster's CTAs, each of which has
// every warp's sum written to it; the barrier is the cluster's).
template <bool SPLIT>
using Sums = float[2][2][SPLIT ? kFewThreads / 32 * kSplitMost : 32];
template <bool SPLIT, int NV>
__device__ __forceinline__ void row_sums(float (&v)[NV], const NormP &p, Sums<SPLIT> &sh, int &n) {
  const int tpr = p.tpr;
  if (!SPLIT && tpr < 32) {
    for (int o = tpr / 2; o; o >>= 1)
#pragma unroll
      for (int i = 0; i < NV; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    return;
  }
#pragma unroll
  for (int o = 16; o; o >>= 1)
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
  if constexpr (SPLIT) {
    const int warps = tpr >> 5, lane = threadIdx.x & 31, half = n++ & 1;
    const int at = (int)(blockIdx.x % p.split) * warps + (threadIdx.x >> 5);
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (lane < p.split) put_cluster(&sh[half][i][at], lane, v[i]);
    tc::cluster_sync();
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      v[i] = 0.f;
#pragma unroll 2
      for (int k = 0; k < warps * p.split; k += 4) {
        const float4 a = *reinterpret_cast<const float4 *>(&sh[half][i][k]);
        v[i] += (a.x + a.y) + (a.z + a.w);
      }
    }
    return;
  }
  if (tpr == 32) return;
  auto &mine = sh[n++ & 1];
  const int warp = threadIdx.x >> 5, per = tpr >> 5, first = warp / per * per;
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int i = 0; i < NV; ++i) mine[i][warp] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    if (per <= 3) {
      v[i] = mine[i][first] + mine[i][first + 1];
      if (per == 3) v[i] += mine[i][first + 2];
    } else if (per == 8) {
      const float4 a = *reinterpret_cast<const float4 *>(&mine[i][first]);
      const float4 b = *reinterpret_cast<const float4 *>(&mine[i][first + 4]);
      v[i] = ((a.x + a.y) + (a.z + a.w)) + ((b.x + b.y) + (b.z + b.w));
    } else {
      v[i] = 0.f;  // (5 warps and more: one row per CTA)
      for (int k = 0; k < per; k += 4) {
        const float4 a = *reinterpret_cast<const float4 *>(&mine[i][first + k]);
        v[i] += (a.x + a.y) + (a.z + a.w);
      }
    }
  }
}

// act(z) from z and its sigmoid; its derivative
__device__ __forceinline__ f2 gate2(int gate, f2 z, f2 s) { return gate == 2 ? s : mul2(z, s); }
__device__ __forceinline__ f2 gate_grad2(int gate, f2 z, f2 s) {
  const f2 one = pack2(1.f, 1.f), c = fma2(s, pack2(-1.f, -1.f), one);  // 1 - s
  return mul2(s, gate == 2 ? c : fma2(z, c, one));
}
__device__ __forceinline__ f2 both(float v) { return pack2(v, v); }

// c = scale w of a thread's columns (w alone without x)
template <int V, int E>
__device__ __forceinline__ void load_c(const NormP &p, bool x, long long slot, int col, int left, f2 (&c)[E / 2]) {
  load_param<V, E>(p.w + (p.heads > 1 ? slot % p.heads * p.D : 0), col, left, p.tpr, c);
  if (!x) return;
  f2 s[E / 2];
#pragma unroll
  for (int k = 0; k < E / 2; ++k) s[k] = both(p.scale_const);
  if (p.scale) load_param<V, E>(p.scale, col, left, p.tpr, s);
#pragma unroll
  for (int k = 0; k < E / 2; ++k) c[k] = mul2(c[k], s[k]);
}

template <typename T, typename XT, int V, int E, int THREADS, int MODE>
__global__ void __launch_bounds__(THREADS, 1) fwd_kernel(const NormP p) {
  constexpr int N = E / 2, R = kAhead<V, E, MODE, false>;
  constexpr bool SPLIT = MODE == kSplit;
  __shared__ __align__(16) Sums<SPLIT> sh;
  for (int i = threadIdx.x; i < (int)(sizeof sh / 4); i += blockDim.x) (&sh[0][0][0])[i] = 0.f;
  const Has<MODE> has(p);
  const int tpr = p.tpr, t = threadIdx.x % tpr, per = blockDim.x / tpr;
  const int split = SPLIT ? p.split : 1, from = SPLIT ? (int)(blockIdx.x % split) * p.cols : 0;
  const int col = from + t * V, left = (SPLIT ? min(p.D, from + p.cols) : p.D) - col;
  const long long slot = (long long)(blockIdx.x / split) * per + threadIdx.x / tpr;
  const long long slots = (long long)(gridDim.x / split) * per;  // (a multiple of heads)
  const float invD = 1.f / (float)p.D;
  f2 c[N], wn[N];
  if (has.f()) load_c<V, E>(p, has.x(), slot, col, left, c);
  if (has.h()) load_param<V, E>(p.w_next, col, left, tpr, wn);
  Part<T, V, E> f[R], z[R];
  Part<XT, V, E> x[R];
  // offsets of this thread's elements in the next row (o: of operands with rows of D)
  long long of = slot * p.f_ld + col, oz = slot * p.z_ld + col, ox = slot * p.x_ld + col, o = slot * p.D + col;
  auto load = [&](int u, long long row) {  // (rows past the end as zeros)
    const int n = row < p.rows ? left : 0;
    if (has.f()) f[u].load((const T *)p.f + of, n, tpr);
    if (has.gate()) z[u].load((const T *)p.z + oz, n, tpr);
    if (has.x()) x[u].load((const XT *)p.x + ox, n, tpr);
    of += slots * p.f_ld;
    oz += slots * p.z_ld;
    ox += slots * p.x_ld;
  };
  int calls = 0;
#pragma unroll
  for (int u = 0; u < R; ++u) load(u, slot + u * slots);
  if (SPLIT) tc::cluster_sync();  // sh
  else __syncthreads();
  for (long long base = slot - threadIdx.x / tpr; base < p.rows; base += R * slots) {
#pragma unroll
  for (int u = 0; u < R; ++u) {
    const long long row = base + u * slots + threadIdx.x / tpr;
    const int out = row < p.rows ? left : 0;
    f2 r[N], v[N], zv[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      if (has.f()) v[k] = f[u].pair(k);
      if (has.gate()) zv[k] = z[u].pair(k);
      if (has.x()) r[k] = x[u].pair(k);
    }
    load(u, row + R * slots);
    if (has.f()) {
      f2 ss = pack2(0.f, 0.f);
#pragma unroll
      for (int k = 0; k < N; ++k) ss = fma2(v[k], v[k], ss);
      float sum[1] = {sum2(ss)};
      row_sums<SPLIT>(sum, p, sh, calls);
      const f2 inv = both(rsqrtf(fmaf(sum[0], invD, p.eps)));
#pragma unroll
      for (int k = 0; k < N; ++k) {
        v[k] = mul2(v[k], inv);
        if (has.gate()) v[k] = mul2(v[k], gate2(has.gate(), zv[k], sigmoid2(zv[k])));
        r[k] = has.x() ? fma2(c[k], v[k], r[k]) : mul2(c[k], v[k]);
      }
      if (p.r_out) {
        if (has.x()) store_part<XT, V, E>((XT *)p.r_out + o, out, tpr, r);
        else store_part<T, V, E>((T *)p.r_out + o, out, tpr, r);
      }
    }
    if (has.h()) {
      f2 ss = pack2(0.f, 0.f);
#pragma unroll
      for (int k = 0; k < N; ++k) ss = fma2(r[k], r[k], ss);  // (zero past D)
      float sum[1] = {sum2(ss)};
      row_sums<SPLIT>(sum, p, sh, calls);
      const f2 inv = both(rsqrtf(fmaf(sum[0], invD, p.eps)));
#pragma unroll
      for (int k = 0; k < N; ++k) r[k] = mul2(mul2(r[k], inv), wn[k]);
      store_part<T, V, E>((T *)p.h + o, out, tpr, r);
    }
    o += slots * p.D;
  }
  }
}

template <typename T, typename XT, int V, int E, int THREADS, int MODE>
__global__ void __launch_bounds__(THREADS, 1) bwd_kernel(const NormP p) {
  constexpr int N = E / 2, R = kAhead<V, E, MODE, true>;
  constexpr bool SPLIT = MODE == kSplit;
  __shared__ __align__(16) Sums<SPLIT> sh;
  for (int i = threadIdx.x; i < (int)(sizeof sh / 4); i += blockDim.x) (&sh[0][0][0])[i] = 0.f;
  const Has<MODE> has(p);
  const int tpr = p.tpr, t = threadIdx.x % tpr, per = blockDim.x / tpr;
  const int split = SPLIT ? p.split : 1, from = SPLIT ? (int)(blockIdx.x % split) * p.cols : 0;
  const int col = from + t * V, left = (SPLIT ? min(p.D, from + p.cols) : p.D) - col;
  const long long slot = (long long)(blockIdx.x / split) * per + threadIdx.x / tpr;
  const long long slots = (long long)(gridDim.x / split) * per;  // (a multiple of heads)
  const float invD = 1.f / (float)p.D;
  const f2 zero2 = pack2(0.f, 0.f);
  f2 c[N], q[N], an[N];
  if (has.f()) load_c<V, E>(p, has.x(), slot, col, left, c);
#pragma unroll
  for (int k = 0; k < N; ++k) q[k] = an[k] = zero2;
  Part<T, V, E> f[R], z[R], dh[R], drt[R];
  Part<XT, V, E> x[R], drx[R];
  // offsets of this thread's elements in the next row (o: of operands with rows of D)
  long long of = slot * p.f_ld + col, oz = slot * p.z_ld + col, ox = slot * p.x_ld + col, o = slot * p.D + col;
  auto load = [&](int u, long long row) {  // (rows past the end as zeros)
    const int n = row < p.rows ? left : 0, nd = p.dr ? n : 0;
    if (has.f()) f[u].load((const T *)p.f + of, n, tpr);
    if (has.gate()) z[u].load((const T *)p.z + oz, n, tpr);
    if (has.x()) {
      x[u].load((const XT *)p.x + ox, n, tpr);
      drx[u].load((const XT *)p.dr + o, nd, tpr);
    } else {
      drt[u].load((const T *)p.dr + o, nd, tpr);
    }
    if (has.h()) dh[u].load((const T *)p.dh + o, n, tpr);
    of += slots * p.f_ld;
    oz += slots * p.z_ld;
    ox += slots * p.x_ld;
    o += slots * p.D;
  };
  int calls = 0;
#pragma unroll
  for (int u = 0; u < R; ++u) load(u, slot + u * slots);
  if (SPLIT) tc::cluster_sync();  // sh
  else __syncthreads();
  for (long long base = slot - threadIdx.x / tpr; base < p.rows; base += R * slots) {
#pragma unroll
  for (int u = 0; u < R; ++u) {
    const long long row = base + u * slots + threadIdx.x / tpr;
    const int out = row < p.rows ? left : 0;
    // (rows past the end are worked on as zeros; with the call's eps, which may be 0, their
    // roots could be infinite and the sums over the rows take 0 times infinity from them)
    const float eps = out > 0 ? p.eps : 1.f;
    const long long now = o - R * slots * p.D;  // this row's place (the loads are R rows ahead)
    f2 fi[N], zv[N], act[N], r[N], g[N], d[N];  // f i1; z, then its gradient; act; r; its gradient; dh
#pragma unroll
    for (int k = 0; k < N; ++k) {
      if (has.f()) fi[k] = f[u].pair(k);
      if (has.gate()) zv[k] = z[u].pair(k);
      if (has.x()) r[k] = x[u].pair(k);
      g[k] = has.x() ? drx[u].pair(k) : drt[u].pair(k);
      if (has.h()) d[k] = dh[u].pair(k);
    }
    load(u, row + R * slots);
    float inv = 0.f;
    if (has.f()) {
      f2 ss = zero2;
#pragma unroll
      for (int k = 0; k < N; ++k) ss = fma2(fi[k], fi[k], ss);
      float sum[1] = {sum2(ss)};
      row_sums<SPLIT>(sum, p, sh, calls);
      inv = rsqrtf(fmaf(sum[0], invD, eps));
#pragma unroll
      for (int k = 0; k < N; ++k) {
        fi[k] = mul2(fi[k], both(inv));
        if (has.gate()) {
          const f2 s = sigmoid2(zv[k]);
          act[k] = gate2(has.gate(), zv[k], s);
          zv[k] = gate_grad2(has.gate(), zv[k], s);
        }
      }
    }
    if (has.h()) {  // r, then its gradient
      // (w_next comes from L1 for every row: with it, too, in registers the kernel spills)
      f2 s2 = zero2, sd = zero2, wn[N];
      load_param<V, E>(p.w_next, col, left, tpr, wn);
#pragma unroll
      for (int k = 0; k < N; ++k) {
        if (has.f()) {
          const f2 v = has.gate() ? mul2(fi[k], act[k]) : fi[k];
          r[k] = has.x() ? fma2(c[k], v, r[k]) : mul2(c[k], v);
        }
        s2 = fma2(r[k], r[k], s2);
        sd = fma2(mul2(wn[k], d[k]), r[k], sd);
      }
      float sum[2] = {sum2(s2), sum2(sd)};
      row_sums<SPLIT>(sum, p, sh, calls);
      const float i2 = rsqrtf(fmaf(sum[0], invD, eps)), m = -sum[1] * invD * i2 * i2;
#pragma unroll
      for (int k = 0; k < N; ++k) {
        an[k] = fma2(mul2(d[k], both(i2)), r[k], an[k]);
        g[k] = fma2(both(i2), fma2(r[k], both(m), mul2(wn[k], d[k])), g[k]);
      }
    }
    if (has.x()) store_part<XT, V, E>((XT *)p.dx + now, out, tpr, g);
    if (has.f()) {
      f2 sd = zero2;
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const f2 gc = mul2(g[k], c[k]);
        if (has.gate()) {
          q[k] = fma2(g[k], mul2(fi[k], act[k]), q[k]);
          zv[k] = mul2(mul2(gc, fi[k]), zv[k]);
          g[k] = mul2(gc, act[k]);
        } else {
          q[k] = fma2(g[k], fi[k], q[k]);
          g[k] = gc;
        }
        sd = fma2(g[k], fi[k], sd);
      }
      if (has.gate()) store_part<T, V, E>((T *)p.dz + now, out, tpr, zv);
      float sum[1] = {sum2(sd)};
      row_sums<SPLIT>(sum, p, sh, calls);
      const float m = -sum[0] * invD;
#pragma unroll
      for (int k = 0; k < N; ++k) g[k] = mul2(both(inv), fma2(fi[k], both(m), g[k]));
      store_part<T, V, E>((T *)p.df + now, out, tpr, g);
    }
  }
  }
  float *mine = p.part + (size_t)slot * 2 * p.D;
  if (has.f()) store_part<float, V, E>(mine + col, left, tpr, q);
  if (has.h()) store_part<float, V, E>(mine + p.D + col, left, tpr, an);
}

struct Launch {
  int ctas, threads;
  bool vec;
};

template <int MODE>
cudaError_t start(void (*kernel)(NormP), const NormP &p, const Launch &l, bool bwd, cudaStream_t s) {
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute cluster{};
  cfg.gridDim = dim3(l.ctas);
  cfg.blockDim = dim3(l.threads);
  cfg.stream = s;
  if (MODE == kSplit) {
    cluster.id = cudaLaunchAttributeClusterDimension;
    cluster.val.clusterDim.x = p.split;
    cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
    cfg.attrs = &cluster;
    cfg.numAttrs = 1;
  }
  if (bwd)
    RDN_LAUNCH("norm_bwd", s, (void)cudaLaunchKernelEx(&cfg, kernel, p));
  else
    RDN_LAUNCH("norm_fwd", s, (void)cudaLaunchKernelEx(&cfg, kernel, p));
  return cudaGetLastError();
}
// A row in one CTA: a kernel for each mode (branches on it cost about a quarter).
template <typename T, typename XT, int V, int MODE>
cudaError_t run(const NormP &p, const Launch &l, bool bwd, cudaStream_t s) {
  constexpr int kMost = V == 1 ? kFewThreads : kThreads;
  constexpr bool f32 = sizeof(T) == 4 || ((MODE & kX) && sizeof(XT) == 4);
  if (!bwd) return start<MODE>(fwd_kernel<T, XT, V, 8, kMost, MODE>, p, l, bwd, s);
  if (few_threads(V > 1, true, f32, p.tpr)) return start<MODE>(bwd_kernel<T, XT, V, 8, f32 ? kFewThreads : kMost, MODE>, p, l, bwd, s);
  return start<MODE>(bwd_kernel<T, XT, V, 8, kMost, MODE>, p, l, bwd, s);
}
template <typename T, typename XT, int V, int BITS>
cudaError_t run_gate(const NormP &p, const Launch &l, bool bwd, cudaStream_t s) {
  switch (p.mode & 3) {
    case 0: return run<T, XT, V, BITS>(p, l, bwd, s);
    case 1: return run<T, XT, V, BITS | 1>(p, l, bwd, s);
    default: return run<T, XT, V, BITS | 2>(p, l, bwd, s);
  }
}
template <typename T, typename XT, int V>
cudaError_t run_mode(const NormP &p, const Launch &l, bool bwd, cudaStream_t s) {
  switch (p.mode & ~3) {
    case kF | kX: return run_gate<T, XT, V, kF | kX>(p, l, bwd, s);
    case kF | kX | kH: return run_gate<T, XT, V, kF | kX | kH>(p, l, bwd, s);
    case kX | kH: return run<T, XT, V, kX | kH>(p, l, bwd, s);
    default: break;
  }
  if constexpr (std::is_same<T, XT>::value)  // (without x its type is f's)
    return p.mode & kH ? run_gate<T, XT, V, kF | kH>(p, l, bwd, s) : run_gate<T, XT, V, kF>(p, l, bwd, s);
  return cudaErrorInvalidValue;
}
template <typename T, typename XT, int V>
cudaError_t run_split(const NormP &p, const Launch &l, bool bwd, cudaStream_t s) {
  return start<kSplit>(bwd ? bwd_kernel<T, XT, V, 8, kFewThreads, kSplit> : fwd_kernel<T, XT, V, 8, kFewThreads, kSplit>,
                       p, l, bwd, s);
}
template <typename T, typename XT>
cudaError_t run_x(const NormP &p, const Launch &l, bool bwd, cudaStream_t s) {
  if (p.split > 1) return l.vec ? run_split<T, XT, 8>(p, l, bwd, s) : run_split<T, XT, 1>(p, l, bwd, s);
  if (l.threads > kThreads) return start<kAny>(fwd_kernel<T, XT, 8, 8, kMostThreads, kAny>, p, l, bwd, s);
  return l.vec ? run_mode<T, XT, 8>(p, l, bwd, s) : run_mode<T, XT, 1>(p, l, bwd, s);
}

// norm_bf16.cu, norm_f32.cu: f, z and h in that type
cudaError_t run_bf16(const NormP &p, const Launch &l, bool x_f32, bool bwd, cudaStream_t s);
cudaError_t run_f32(const NormP &p, const Launch &l, bool x_f32, bool bwd, cudaStream_t s);

}  // namespace norm
}  // namespace rdn
