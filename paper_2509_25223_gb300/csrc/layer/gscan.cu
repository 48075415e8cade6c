// gscan.cu -- the gated linear recurrence (include/rdn.h, rdn_gscan_*): one state per
// channel,
//     h_t = a_t h_{t-1} + m_t s_t x_t,   a = exp(la), la = -c softplus(lam) sigmoid(r),
//     m = sqrt(1 - a^2), s = sigmoid(i).
// A span of tokens maps the state before it to the state after it as h -> A h + H, and
// two spans compose to (A2 A1, A2 H1 + H2).  So a token row is cut three times: a warp
// takes kTok consecutive tokens of 32 V channels (its lanes), a CTA the kTile tokens of
// its warps, and a cluster of up to 8 CTAs as many tiles, one round after another.  Each
// warp works out its span from a zero state with everything in registers; the spans'
// (A, H) go through shared memory, the tiles' to every CTA of the cluster, and the states
// follow as h_t = A_t h_in + H_t.  The data are read once and the results written once.
// The backward is the same over the reversed tokens, with
//     g_t = dy_t + q_{t+1},  q_t = a_t g_t       (q: the gradient of the state before t)
// and the states again from those that the forward kept before every tile:
//     dx = g m s,  di = g m x s (1 - s),  w_t = g (a h_{t-1} la - a^2 s x la / m),
//     dr = (1 - sigmoid(r)) w,  dlam = sigmoid(lam) / softplus(lam) sum_t w_t
// (la / m stays finite where la -> 0: m ~ sqrt(-2 la)).
#include "rows.cuh"
#include "tc_common.cuh"

namespace rdn {

template <>
struct Pack<float, 2> {
  using Raw = float2;
  __device__ static Raw zero() { return make_float2(0.f, 0.f); }
  __device__ static Raw ld(const float *p) { return *reinterpret_cast<const float2 *>(p); }
  __device__ static void get(const Raw &a, float (&v)[2]) { v[0] = a.x; v[1] = a.y; }
  __device__ static Raw put(const float (&v)[2]) { return make_float2(v[0], v[1]); }
  __device__ static void st(float *p, const Raw &a) { *reinterpret_cast<float2 *>(p) = a; }
};
template <>
struct Pack<__nv_bfloat16, 2> {
  using Raw = uint32_t;
  __device__ static Raw zero() { return 0u; }
  __device__ static Raw ld(const __nv_bfloat16 *p) { return *reinterpret_cast<const uint32_t *>(p); }
  __device__ static void get(const Raw &a, float (&v)[2]) {
    v[0] = __uint_as_float(a << 16);
    v[1] = __uint_as_float(a & 0xffff0000u);
  }
  __device__ static Raw put(const float (&v)[2]) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(v[0], v[1]);
    return *reinterpret_cast<const uint32_t *>(&b);
  }
  __device__ static void st(__nv_bfloat16 *p, const Raw &a) { *reinterpret_cast<uint32_t *>(p) = a; }
};

namespace gscan {

constexpr int kTok = 8, kWarps = 8, kTile = kTok * kWarps, kThreads = 32 * kWarps;
constexpr int kCluster = 8;  // the most CTAs of a cluster
static_assert(kTile == RDN_GSCAN_CHUNK, "a tile starts at every kept state");

struct GP {
  int B, T, D, nc, strips, num_seqs, num_slots;
  float c;
  long long x_ld, r_ld, i_ld, y_ld, dy_ld, dx_ld, dr_ld, di_ld;
  const void *x, *r, *i, *dy;
  const float *lam, *h0, *dhT;
  void *y, *dx, *dr, *di;
  float *hT, *chunks, *dh0, *part;
  const int *cu, *slots;
  float *h;
};

__device__ __forceinline__ float softplusf(float v) { return v > 20.f ? v : log1pf(expf(v)); }

// The gates of one element.  k = -c softplus(lam).
struct Gate {
  float sr, si, nr, ni;  // sigmoid(r), sigmoid(i), 1 - sigmoid(r), 1 - sigmoid(i)
  float la, a, m;
};
// Both sigmoids share one reciprocal (the special function unit is the narrowest part of the
// forward): 1 / (1 + e^-r) = (1 + e^-i) / ((1 + e^-r)(1 + e^-i)).  The arguments are cut at -40
// so that the product stays finite (a NaN passes).  u = 1 - a by the series of expm1 where a is
// near 1, so that 1 - a^2 = u (2 - u) keeps its digits.
__device__ __forceinline__ Gate gate(float r, float i, float k) {
  Gate g;
  r = r < -40.f ? -40.f : r;
  i = i < -40.f ? -40.f : i;
  const float er = ex2(-kLog2e * r), ei = ex2(-kLog2e * i);
  const float pr = 1.f + er, pi = 1.f + ei, R = rcp_approx(pr * pi);
  g.sr = R * pi;
  g.si = R * pr;
  g.nr = er * g.sr;
  g.ni = ei * g.si;
  float z = k * g.sr;
  z = z < -88.f ? -88.f : z;
  g.la = z;
  // -expm1(z) = -z (1 + z/2 (1 + z/3 (...))): the term left out is below 0.6^8 / 9! = 5e-8 of the sum
  float u = 1.f / 40320.f;
  u = fmaf(u, z, 1.f / 5040.f);
  u = fmaf(u, z, 1.f / 720.f);
  u = fmaf(u, z, 1.f / 120.f);
  u = fmaf(u, z, 1.f / 24.f);
  u = fmaf(u, z, 1.f / 6.f);
  u = fmaf(u, z, 0.5f);
  u = fmaf(u, z, 1.f);
  u = -z * u;
  g.a = 1.f - u;
  if (z < -0.6f) {
    g.a = ex2(kLog2e * z);
    u = 1.f - g.a;
  }
  g.m = __fsqrt_rn(u * (2.f - u));
  return g;
}

// What the two passes over a row share: this thread's place.
template <typename T, int V>
struct Place {
  int lane, warp, rank, b, ch;
  bool live;  // whether the lane's channels exist
  __device__ explicit Place(const GP &p) {
    lane = threadIdx.x & 31;
    warp = threadIdx.x >> 5;
    rank = blockIdx.x % p.nc;
    const int unit = blockIdx.x / p.nc;
    b = unit / p.strips;
    ch = ((unit % p.strips) * 32 + lane) * V;
    live = ch < p.D;
  }
};

// Sequence that starts / ends at each token of the tile (-1: none).
__device__ __forceinline__ void mark_tile(const GP &p, int t0, int2 *mark) {
  const int k = threadIdx.x;
  if (k < kTile) {
    int2 f = make_int2(-1, -1);
    if (t0 + k < p.T) {
      const SeqSpan q = find_seq(p.cu, p.num_seqs, p.T, 0, t0 + k);
      if (q.begin == t0 + k) f.x = q.s;
      if (q.end == t0 + k + 1) f.y = q.s;
    }
    mark[k] = f;
  }
}

__device__ __forceinline__ void st_cluster(uint32_t addr, float2 v) {
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(addr), "f"(v.x), "f"(v.y) : "memory");
}

// (A, H) of two spans in turn.  A = -1 stands for a span in which a packed sequence starts:
// what comes before it does not enter, not even as 0 times an infinity or NaN.
template <bool kPacked>
__device__ __forceinline__ float over(float2 s, float h) {
  const float r = fmaf(s.x, h, s.y);
  return kPacked && s.x < 0.f ? s.y : r;
}
template <bool kPacked>
__device__ __forceinline__ float2 then(float2 s1, float2 s2) {
  const float A = kPacked && (s1.x < 0.f || s2.x < 0.f) ? -1.f : s1.x * s2.x;
  return make_float2(A, over<kPacked>(s2, s1.y));
}

// Sends the composition of the CTA's warps' spans (in the order 0.. or, kBack, 7..) to the
// slot of this CTA in every CTA of the cluster, and waits until all have.
template <int V, bool kBack, bool kPacked>
__device__ __forceinline__ void exchange(const float2 (*spans)[32 * V], float2 (*tiles)[32 * V], int rank, int nc) {
  if (nc > 1) {
    const int c = threadIdx.x % (32 * V);
    float2 all = spans[kBack ? kWarps - 1 : 0][c];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) all = then<kPacked>(all, spans[kBack ? kWarps - 1 - w : w][c]);
    for (int q = threadIdx.x / (32 * V); q < nc; q += kThreads / (32 * V))
      st_cluster(tc::map_rank(&tiles[rank][c], q), all);
    tc::cluster_sync();
  }
}

// The state that comes into this warp's span, and the one that leaves the cluster's round.
template <int V, bool kBack, bool kPacked>
__device__ __forceinline__ void fold(const float2 (*spans)[32 * V], const float2 (*tiles)[32 * V], int c, int rank,
                                     int nc, int warp, float &carry, float &in) {
  float h = carry;
  in = h;
  if (nc > 1) {
    for (int q = 0; q < nc; ++q) {
      const int k = kBack ? nc - 1 - q : q;
      if (k == rank) in = h;
      h = over<kPacked>(tiles[k][c], h);
    }
  }
  float run = in;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const int k = kBack ? kWarps - 1 - w : w;
    if (k == warp) in = run;
    run = over<kPacked>(spans[k][c], run);
  }
  carry = nc > 1 ? h : run;
}

template <typename T, int V, bool kPacked>
__global__ void __launch_bounds__(kThreads) fwd_kernel(const GP p) {
  using P = Pack<T, V>;
  __shared__ float2 spans[2][kWarps][32 * V], tiles[2][kCluster][32 * V];
  __shared__ int2 mark[2][kTile];
  const Place<T, V> at(p);
  const T *x = static_cast<const T *>(p.x), *r = static_cast<const T *>(p.r), *gi = static_cast<const T *>(p.i);
  T *y = static_cast<T *>(p.y);
  const long long row0 = (long long)at.b * p.T;
  const int ntiles = (p.T + kTile - 1) / kTile;

  float k[V], carry[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    k[v] = at.live ? -p.c * softplusf(p.lam[at.ch + v]) : 0.f;
    carry[v] = !kPacked && at.live && p.h0 ? p.h0[(size_t)at.b * p.D + at.ch + v] : 0.f;
  }
  if (p.hT && at.live) {  // sequences without tokens
    if (!kPacked) {
      if (p.T == 0 && at.rank == 0 && at.warp == 0)
#pragma unroll
        for (int v = 0; v < V; ++v) p.hT[(size_t)at.b * p.D + at.ch + v] = carry[v];
    } else {
      for (int s = at.rank * kWarps + at.warp; s < p.num_seqs; s += p.nc * kWarps)
        if (cu_at(p.cu, p.num_seqs, p.T, s + 1) <= cu_at(p.cu, p.num_seqs, p.T, s))
#pragma unroll
          for (int v = 0; v < V; ++v) {
            const size_t o = (size_t)s * p.D + at.ch + v;
            p.hT[o] = p.h0 ? p.h0[o] : 0.f;
          }
    }
  }

  if (p.nc > 1) tc::cluster_sync();  // every CTA runs before another writes its shared memory
  int par = 0;
  for (int base = 0; base < p.T; base += p.nc * kTile, par ^= 1) {
    const int tile0 = base + at.rank * kTile, t0 = tile0 + at.warp * kTok;
    typename P::Raw xr[kTok], rr[kTok], ir[kTok];
#pragma unroll
    for (int j = 0; j < kTok; ++j) {
      const bool ok = at.live && t0 + j < p.T;
      const long long row = row0 + t0 + j;
      xr[j] = ok ? P::ld(x + row * p.x_ld + at.ch) : P::zero();
      rr[j] = ok ? P::ld(r + row * p.r_ld + at.ch) : P::zero();
      ir[j] = ok ? P::ld(gi + row * p.i_ld + at.ch) : P::zero();
    }
    if (kPacked) {
      mark_tile(p, tile0, mark[par]);
      __syncthreads();
    }
    float A[kTok][V], H[kTok][V], Ac[V], Hc[V];
#pragma unroll
    for (int v = 0; v < V; ++v) { Ac[v] = 1.f; Hc[v] = 0.f; }
#pragma unroll
    for (int j = 0; j < kTok; ++j) {
      float xv[V], rv[V], iv[V];
      P::get(xr[j], xv);
      P::get(rr[j], rv);
      P::get(ir[j], iv);
      const int start = kPacked ? mark[par][at.warp * kTok + j].x : -1;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (t0 + j < p.T) {
          const Gate g = gate(rv[v], iv[v], k[v]);
          float a = g.a, b = g.m * g.si * xv[v];
          if (kPacked && start >= 0) {
            if (p.h0 && at.live) b = fmaf(a, p.h0[(size_t)start * p.D + at.ch + v], b);
            Ac[v] = -1.f;
            Hc[v] = b;
          } else {
            if (!kPacked || Ac[v] >= 0.f) Ac[v] *= a;
            Hc[v] = fmaf(a, Hc[v], b);
          }
        }
        A[j][v] = Ac[v];
        H[j][v] = Hc[v];
      }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) spans[par][at.warp][at.lane * V + v] = make_float2(Ac[v], Hc[v]);
    __syncthreads();
    exchange<V, false, kPacked>(spans[par], tiles[par], at.rank, p.nc);
    float in[V];
#pragma unroll
    for (int v = 0; v < V; ++v)
      fold<V, false, kPacked>(spans[par], tiles[par], at.lane * V + v, at.rank, p.nc, at.warp, carry[v], in[v]);
    if (at.live) {
      if (p.chunks && at.warp == 0 && tile0 < p.T)
#pragma unroll
        for (int v = 0; v < V; ++v)
          p.chunks[((size_t)at.b * ntiles + tile0 / kTile) * p.D + at.ch + v] = in[v];
#pragma unroll
      for (int j = 0; j < kTok; ++j) {
        if (t0 + j >= p.T) break;
        float h[V];
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = over<kPacked>(make_float2(A[j][v], H[j][v]), in[v]);
        if (y) P::st(y + (row0 + t0 + j) * p.y_ld + at.ch, P::put(h));
        const int end = kPacked ? mark[par][at.warp * kTok + j].y : t0 + j == p.T - 1 ? at.b : -1;
        if (p.hT && end >= 0)
#pragma unroll
          for (int v = 0; v < V; ++v) p.hT[(size_t)end * p.D + at.ch + v] = h[v];
      }
    }
    __syncwarp();
  }
}

template <typename T, int V, bool kPacked>
__global__ void __launch_bounds__(kThreads, 2) bwd_kernel(const GP p) {
  using P = Pack<T, V>;
  __shared__ float2 fspans[2][kWarps][32 * V], spans[2][kWarps][32 * V], tiles[2][kCluster][32 * V];
  __shared__ int2 mark[2][kTile];
  const Place<T, V> at(p);
  const T *x = static_cast<const T *>(p.x), *r = static_cast<const T *>(p.r), *gi = static_cast<const T *>(p.i);
  const T *dy = static_cast<const T *>(p.dy);
  T *dx = static_cast<T *>(p.dx), *dr = static_cast<T *>(p.dr), *di = static_cast<T *>(p.di);
  const long long row0 = (long long)at.b * p.T;
  const int ntiles = (p.T + kTile - 1) / kTile;

  float k[V], carry[V], sum[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    k[v] = at.live ? -p.c * softplusf(p.lam[at.ch + v]) : 0.f;
    carry[v] = !kPacked && at.live && p.dhT ? p.dhT[(size_t)at.b * p.D + at.ch + v] : 0.f;
    sum[v] = 0.f;
  }
  if (p.dh0 && at.live) {  // sequences without tokens
    if (!kPacked) {
      if (p.T == 0 && at.rank == 0 && at.warp == 0)
#pragma unroll
        for (int v = 0; v < V; ++v) p.dh0[(size_t)at.b * p.D + at.ch + v] = carry[v];
    } else {
      for (int s = at.rank * kWarps + at.warp; s < p.num_seqs; s += p.nc * kWarps)
        if (cu_at(p.cu, p.num_seqs, p.T, s + 1) <= cu_at(p.cu, p.num_seqs, p.T, s))
#pragma unroll
          for (int v = 0; v < V; ++v) {
            const size_t o = (size_t)s * p.D + at.ch + v;
            p.dh0[o] = p.dhT ? p.dhT[o] : 0.f;
          }
    }
  }

  if (p.nc > 1) tc::cluster_sync();  // every CTA runs before another writes its shared memory
  int par = 0;
  const int round = p.nc * kTile;
  for (int base = (p.T - 1) / round * round; base >= 0 && p.T > 0; base -= round, par ^= 1) {
    const int tile0 = base + at.rank * kTile, t0 = tile0 + at.warp * kTok;
    typename P::Raw xr[kTok], rr[kTok], ir[kTok], gr[kTok];
#pragma unroll
    for (int j = 0; j < kTok; ++j) {
      const bool ok = at.live && t0 + j < p.T;
      const long long row = row0 + t0 + j;
      xr[j] = ok ? P::ld(x + row * p.x_ld + at.ch) : P::zero();
      rr[j] = ok ? P::ld(r + row * p.r_ld + at.ch) : P::zero();
      ir[j] = ok ? P::ld(gi + row * p.i_ld + at.ch) : P::zero();
      gr[j] = ok ? P::ld(dy + row * p.dy_ld + at.ch) : P::zero();
    }
    float h[V];  // the state before the tile
#pragma unroll
    for (int v = 0; v < V; ++v)
      h[v] = at.live && tile0 < p.T ? p.chunks[((size_t)at.b * ntiles + tile0 / kTile) * p.D + at.ch + v] : 0.f;
    if (kPacked) {
      mark_tile(p, tile0, mark[par]);
      __syncthreads();
    }
    // this warp's span from a zero state, both ways
    float a[kTok][V], Af[V], Hf[V], Ab[V], Hb[V];
#pragma unroll
    for (int v = 0; v < V; ++v) { Af[v] = 1.f; Hf[v] = 0.f; Ab[v] = 1.f; Hb[v] = 0.f; }
#pragma unroll
    for (int j = 0; j < kTok; ++j) {
      float xv[V], rv[V], iv[V];
      P::get(xr[j], xv);
      P::get(rr[j], rv);
      P::get(ir[j], iv);
      const int start = kPacked ? mark[par][at.warp * kTok + j].x : -1;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        a[j][v] = 1.f;
        if (t0 + j < p.T) {
          const Gate g = gate(rv[v], iv[v], k[v]);
          a[j][v] = g.a;
          float b = g.m * g.si * xv[v];
          if (kPacked && start >= 0) {
            if (p.h0 && at.live) b = fmaf(g.a, p.h0[(size_t)start * p.D + at.ch + v], b);
            Af[v] = -1.f;
            Hf[v] = b;
          } else {
            if (!kPacked || Af[v] >= 0.f) Af[v] *= g.a;
            Hf[v] = fmaf(g.a, Hf[v], b);
          }
        }
      }
    }
#pragma unroll
    for (int j = kTok - 1; j >= 0; --j) {
      float gv[V];
      P::get(gr[j], gv);
      const int end = kPacked ? mark[par][at.warp * kTok + j].y : -1;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (kPacked && end >= 0) {
          Ab[v] = -1.f;
          Hb[v] = p.dhT && at.live ? p.dhT[(size_t)end * p.D + at.ch + v] : 0.f;
        }
        if (!kPacked || Ab[v] >= 0.f) Ab[v] *= a[j][v];
        Hb[v] = a[j][v] * (gv[v] + Hb[v]);
      }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      fspans[par][at.warp][at.lane * V + v] = make_float2(Af[v], Hf[v]);
      spans[par][at.warp][at.lane * V + v] = make_float2(Ab[v], Hb[v]);
    }
    __syncthreads();
    exchange<V, true, kPacked>(spans[par], tiles[par], at.rank, p.nc);
    float q[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int c = at.lane * V + v;
      fold<V, true, kPacked>(spans[par], tiles[par], c, at.rank, p.nc, at.warp, carry[v], q[v]);
      for (int w = 0; w < at.warp; ++w) h[v] = over<kPacked>(fspans[par][w][c], h[v]);
    }
    if (at.live) {
      float before[kTok][V];  // the state before each token
#pragma unroll
      for (int j = 0; j < kTok; ++j) {
        float xv[V], rv[V], iv[V];
        P::get(xr[j], xv);
        P::get(rr[j], rv);
        P::get(ir[j], iv);
        const int start = kPacked ? mark[par][at.warp * kTok + j].x : -1;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          if (kPacked && start >= 0) h[v] = p.h0 ? p.h0[(size_t)start * p.D + at.ch + v] : 0.f;
          before[j][v] = h[v];
          const Gate g = gate(rv[v], iv[v], k[v]);
          h[v] = fmaf(g.a, h[v], g.m * g.si * xv[v]);
        }
      }
#pragma unroll
      for (int j = kTok - 1; j >= 0; --j) {
        if (t0 + j >= p.T) continue;
        float xv[V], rv[V], iv[V], gv[V], ox[V], orr[V], oi[V];
        P::get(xr[j], xv);
        P::get(rr[j], rv);
        P::get(ir[j], iv);
        P::get(gr[j], gv);
        const int2 f = kPacked ? mark[par][at.warp * kTok + j] : make_int2(t0 + j == 0 ? at.b : -1, -1);
#pragma unroll
        for (int v = 0; v < V; ++v) {
          if (kPacked && f.y >= 0) q[v] = p.dhT ? p.dhT[(size_t)f.y * p.D + at.ch + v] : 0.f;
          const float g = gv[v] + q[v];
          const Gate e = gate(rv[v], iv[v], k[v]);
          const float gs = g * e.si, gm = gs * e.m;
          ox[v] = gm;
          oi[v] = gm * xv[v] * e.ni;
          const float lam = e.m > 0.f ? __fdividef(e.la, e.m) : 0.f;
          const float w = e.a * (g * before[j][v] * e.la - e.a * (gs * xv[v]) * lam);
          orr[v] = e.nr * w;
          sum[v] += w;
          q[v] = e.a * g;
          if (p.dh0 && f.x >= 0) p.dh0[(size_t)f.x * p.D + at.ch + v] = q[v];
        }
        const long long row = row0 + t0 + j;
        P::st(dx + row * p.dx_ld + at.ch, P::put(ox));
        P::st(dr + row * p.dr_ld + at.ch, P::put(orr));
        P::st(di + row * p.di_ld + at.ch, P::put(oi));
      }
    }
    __syncwarp();
  }
  // sum of w over this CTA's tokens, the warps in order
  __syncthreads();
#pragma unroll
  for (int v = 0; v < V; ++v) fspans[0][at.warp][at.lane * V + v] = make_float2(sum[v], 0.f);
  __syncthreads();
  if (at.warp == 0 && at.live)
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float s = 0.f;
      for (int w = 0; w < kWarps; ++w) s += fspans[0][w][at.lane * V + v].x;
      p.part[((size_t)at.b * p.nc + at.rank) * p.D + at.ch + v] = s;
    }
}

// dlam = sigmoid(lam) / softplus(lam) times the sum of the CTAs' sums, in order: 16 interleaved
// sums, joined in order.
__global__ void __launch_bounds__(512) dlam_kernel(const GP p, long long parts, float *dlam) {
  __shared__ float sh[16][32];
  const int ch = blockIdx.x * 32 + threadIdx.x;
  float a = 0.f;
  if (ch < p.D)
    for (long long q = threadIdx.y; q < parts; q += 16) a += p.part[(size_t)q * p.D + ch];
  sh[threadIdx.y][threadIdx.x] = a;
  __syncthreads();
  if (threadIdx.y || ch >= p.D) return;
#pragma unroll
  for (int y = 1; y < 16; ++y) a += sh[y][threadIdx.x];
  const float lam = p.lam[ch], sp = softplusf(lam);
  // (both are e^lam to the last digit where lam is far below zero)
  const float ratio = lam < -20.f ? 1.f : __fdividef(1.f, (1.f + expf(-lam)) * sp);
  dlam[ch] = a * ratio;
}

template <typename T, int V>
__global__ void __launch_bounds__(kThreads) step_kernel(const GP p) {
  using P = Pack<T, V>;
  const int ch = (blockIdx.x * kThreads + threadIdx.x) * V, n = blockIdx.y;
  if (ch >= p.D) return;
  for (int row = n; row < p.B; row += gridDim.y) {
    const int slot = p.slots ? p.slots[row] : row;
    float y[V];
    if (slot < 0 || slot >= p.num_slots) {
#pragma unroll
      for (int v = 0; v < V; ++v) y[v] = 0.f;
    } else {
      float xv[V], rv[V], iv[V];
      P::get(P::ld(static_cast<const T *>(p.x) + row * p.x_ld + ch), xv);
      P::get(P::ld(static_cast<const T *>(p.r) + row * p.r_ld + ch), rv);
      P::get(P::ld(static_cast<const T *>(p.i) + row * p.i_ld + ch), iv);
      float *h = p.h + (size_t)slot * p.D + ch;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const Gate g = gate(rv[v], iv[v], -p.c * softplusf(p.lam[ch + v]));
        y[v] = fmaf(g.a, h[v], g.m * g.si * xv[v]);
        h[v] = y[v];
      }
    }
    P::st(static_cast<T *>(p.y) + row * p.y_ld + ch, P::put(y));
  }
}

// CTAs of a cluster: the tiles of a row, at most 8.
int cluster_of(int T) {
  int nc = 1;
  while (nc < kCluster && (long long)nc * kTile < T) nc *= 2;
  return nc;
}

GP params(const rdn_gscan_args &a, int V) {
  GP p{};
  p.B = a.B; p.T = a.T; p.D = a.D; p.c = a.c;
  p.nc = cluster_of(a.T);
  p.strips = (a.D + 32 * V - 1) / (32 * V);
  p.num_seqs = a.num_seqs; p.cu = a.cu_seqlens;
  p.x_ld = a.x_ld; p.r_ld = a.r_ld; p.i_ld = a.i_ld; p.y_ld = a.y_ld;
  p.dy_ld = a.dy_ld; p.dx_ld = a.dx_ld; p.dr_ld = a.dr_ld; p.di_ld = a.di_ld;
  p.x = a.x; p.r = a.r; p.i = a.i; p.dy = a.dy;
  p.lam = a.lam; p.h0 = a.h0; p.dhT = a.dhT;
  p.y = a.y; p.dx = a.dx; p.dr = a.dr; p.di = a.di;
  p.hT = a.hT; p.chunks = a.h_chunks; p.dh0 = a.dh0;
  return p;
}

// Pairs of channels: an even D, and every row on two elements.
bool pairs_ok(int D, size_t e, std::initializer_list<const void *> ptrs, std::initializer_list<long long> lds) {
  if (D & 1) return false;
  for (const void *q : ptrs)
    if ((uintptr_t)q & (2 * e - 1)) return false;
  for (long long l : lds)
    if (l & 1) return false;
  return true;
}

template <typename T, int V>
cudaError_t run(const GP &p, bool bwd, const char *name, cudaStream_t s) {
  auto kern = bwd ? (p.cu ? bwd_kernel<T, V, true> : bwd_kernel<T, V, false>)
                  : (p.cu ? fwd_kernel<T, V, true> : fwd_kernel<T, V, false>);
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)((long long)p.B * p.strips * p.nc));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = p.nc;
  at.val.clusterDim.y = at.val.clusterDim.z = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  cudaError_t e;
  RDN_LAUNCH(name, s, (e = cudaLaunchKernelEx(&cfg, kern, p)));
  return e;
}
cudaError_t run(const GP &p, bool bwd, int dtype, int V, const char *name, cudaStream_t s) {
  if (dtype == RDN_BF16)
    return V == 2 ? run<__nv_bfloat16, 2>(p, bwd, name, s) : run<__nv_bfloat16, 1>(p, bwd, name, s);
  return V == 2 ? run<float, 2>(p, bwd, name, s) : run<float, 1>(p, bwd, name, s);
}

size_t part_bytes(const rdn_gscan_args &a) {
  return round256(sizeof(float) * (size_t)a.B * cluster_of(a.T) * a.D);
}

}  // namespace gscan

long long gscan_slots(const rdn_gscan_args &a) {
  return (long long)a.B * ((a.T + gscan::kTile - 1) / gscan::kTile);
}
// CTAs of a call at one channel a lane, the most it may take.
long long gscan_ctas(const rdn_gscan_args &a) {
  return (long long)a.B * ((a.D + 31) / 32) * gscan::cluster_of(a.T);
}
size_t gscan_bwd_bytes(const rdn_gscan_args &a) {
  const size_t states = a.h_chunks ? 0 : round256(sizeof(float) * (size_t)gscan_slots(a) * a.D);
  return gscan::part_bytes(a) + states;
}

cudaError_t launch_gscan_fwd(const rdn_gscan_args &a, cudaStream_t s) {
  const size_t e = a.dtype == RDN_BF16 ? 2 : 4;
  const int V = gscan::pairs_ok(a.D, e, {a.x, a.r, a.i, a.y}, {a.x_ld, a.r_ld, a.i_ld, a.y_ld}) ? 2 : 1;
  return gscan::run(gscan::params(a, V), false, a.dtype, V, "gscan_fwd", s);
}

cudaError_t launch_gscan_bwd(const rdn_gscan_args &a, cudaStream_t s) {
  const size_t el = a.dtype == RDN_BF16 ? 2 : 4;
  rdn_gscan_args c = a;
  if (!c.h_chunks) {
    c.h_chunks = reinterpret_cast<float *>(static_cast<char *>(a.workspace) + gscan::part_bytes(a));
    rdn_gscan_args f = c;
    f.y = nullptr;
    f.hT = nullptr;
    if (a.T > 0) {
      const cudaError_t e = launch_gscan_fwd(f, s);
      if (e != cudaSuccess) return e;
    }
  }
  const int V = gscan::pairs_ok(a.D, el, {a.x, a.r, a.i, a.dy, a.dx, a.dr, a.di},
                                {a.x_ld, a.r_ld, a.i_ld, a.dy_ld, a.dx_ld, a.dr_ld, a.di_ld}) ? 2 : 1;
  gscan::GP p = gscan::params(c, V);
  p.part = static_cast<float *>(a.workspace);
  cudaError_t e = gscan::run(p, true, a.dtype, V, "gscan_bwd", s);
  if (e != cudaSuccess) return e;
  RDN_LAUNCH("gscan_dlam", s,
             (gscan::dlam_kernel<<<(a.D + 31) / 32, dim3(32, 16), 0, s>>>(p, (long long)p.B * p.nc, a.dlam)));
  return cudaGetLastError();
}

cudaError_t launch_gscan_step(const rdn_gscan_step_args &a, cudaStream_t s) {
  const size_t e = a.dtype == RDN_BF16 ? 2 : 4;
  const int V = gscan::pairs_ok(a.D, e, {a.x, a.r, a.i, a.y}, {a.x_ld, a.r_ld, a.i_ld, a.y_ld}) ? 2 : 1;
  gscan::GP p{};
  p.B = a.N; p.D = a.D; p.c = a.c; p.num_slots = a.num_slots;
  p.x_ld = a.x_ld; p.r_ld = a.r_ld; p.i_ld = a.i_ld; p.y_ld = a.y_ld;
  p.x = a.x; p.r = a.r; p.i = a.i; p.lam = a.lam; p.h = a.h; p.slots = a.slots; p.y = a.y;
  const dim3 grid((a.D + gscan::kThreads * V - 1) / (gscan::kThreads * V), a.N < 65535 ? a.N : 65535);
  auto kern = a.dtype == RDN_BF16
                  ? (V == 2 ? gscan::step_kernel<__nv_bfloat16, 2> : gscan::step_kernel<__nv_bfloat16, 1>)
                  : (V == 2 ? gscan::step_kernel<float, 2> : gscan::step_kernel<float, 1>);
  RDN_LAUNCH("gscan_step", s, (kern<<<grid, gscan::kThreads, 0, s>>>(p)));
  return cudaGetLastError();
}

}  // namespace rdn
