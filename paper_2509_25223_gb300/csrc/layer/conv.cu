// conv.cu -- the short causal convolution in front of a recurrence: depthwise,
// W = 2..4 taps per channel, optional SiLU,
//     p_t = bias + sum_{k<W} w[W-1-k] x_{t-k},        y_t = act(p_t)
// and its backward
//     dp_t = dy_t act'(p_t),   dx_t = sum_k w[W-1-k] dp_{t+k},
//     dw[W-1-k] = sum_t dp_t x_{t-k},   dbias = sum_t dp_t
// (p recomputed from x), and its step of one token.
//
// Memory-bound: x in and y out, or x and dy in and dx out.  A thread owns a few
// consecutive channels (one vector access) over a run of tokens and slides the
// W-1 older inputs -- in the backward, which walks down, the W-1 later dp --
// through registers, so x is read once but for the W-1 rows above a run.  The
// loads of a group of tokens are issued together, a group ahead, the first one
// before the taps are there.
// Groups within one sequence take a path without per-token checks, worked on as
// pairs of channels; a sequence's start or end within a group is the rare path,
// which takes the taps from state0.
// At 8 x 4096 tokens of 2048 bf16 channels with SiLU the forward takes 50 us (268 MB,
// 5.4 TB/s: 79 % of a copy's rate) at 12 instructions per element, and the backward
// 103 us (403 MB, 3.9 TB/s) at 26, of which 10 are multiply-adds of a pair's half: it
// is bound by the FMA pipe (half of its slots busy, about two thirds being the most
// for operands in three different registers) and the latency of a token's chain
// at the 12 warps per SM that the registers leave.
#include <initializer_list>
#include <utility>

#include "rows.cuh"

namespace rdn {
namespace {

constexpr int kConvThreads = 128;
constexpr int kFwdGroup = 8;  // tokens whose loads a thread issues together
constexpr int kBwdGroup = 4;
constexpr int kRunStep = 8, kRunMost = 64;  // tokens of a thread's run

struct ConvP {
  int B, T, C, ns, run;  // run: tokens per thread
  int runs;              // runs per batch row
  int silu;
  long long x_ld, y_ld, dy_ld, dx_ld;
  const void *x, *state0, *dy, *dstateT;
  void *y, *stateT, *dx, *dstate0;
  const float *w, *bias;
  const int *cu;
  float *part;  // backward: [row groups of the grid][C][W + 1]
};

// The taps w[W-1-k] of V channels (tap[k]) and their biases, through shared
// memory: a thread's V W taps are consecutive, and read one by one straight
// from global memory every one of them would take a line per lane.  Called by
// the whole CTA; sh: blockDim.x * (V W + 1) floats (a row and one: the lanes
// then read different banks).
template <int W, int V>
__device__ __forceinline__ void load_taps(const ConvP &p, int c0, float *sh, f2 (&tap)[W][(V + 1) / 2],
                                          f2 (&bias)[(V + 1) / 2]) {
  constexpr int R = V * W;
  const int tid = threadIdx.y * blockDim.x + threadIdx.x;
  const int base = (c0 - (int)threadIdx.x * V) * W, n = min((int)blockDim.x * R, p.C * W - base);
  for (int i = tid; i < n; i += kConvThreads) sh[i / R * (R + 1) + i % R] = __ldg(p.w + base + i);
  __syncthreads();
  float t[W][V], b[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
#pragma unroll
    for (int k = 0; k < W; ++k) t[k][e] = sh[threadIdx.x * (R + 1) + e * W + W - 1 - k];
    b[e] = p.bias && c0 + e < p.C ? __ldg(p.bias + c0 + e) : 0.f;
  }
#pragma unroll
  for (int k = 0; k < W; ++k) to_pairs<V>(t[k], tap[k]);
  to_pairs<V>(b, bias);
}
template <typename T, int V>
__device__ __forceinline__ void get_pairs(const typename Pack<T, V>::Raw &raw, f2 (&p)[(V + 1) / 2]) {
  float v[V];
  Pack<T, V>::get(raw, v);
  to_pairs<V>(v, p);
}
template <typename T, int V>
__device__ __forceinline__ typename Pack<T, V>::Raw put_pairs(const f2 (&p)[(V + 1) / 2]) {
  float v[V];
  from_pairs<V>(p, v);
  return Pack<T, V>::put(v);
}

// Sequences without tokens pass their state (or its gradient) through.
template <typename T, int W, int V>
__device__ __forceinline__ void pass_empty(const ConvP &p, long long unit, long long units, int c0,
                                           const void *from, void *to) {
  using K = Pack<T, V>;
  if (!to || (!p.cu && p.T > 0)) return;
  for (long long s = unit; s < p.ns; s += units) {
    if (p.cu && cu_at(p.cu, p.ns, p.T, (int)s) < cu_at(p.cu, p.ns, p.T, (int)s + 1)) continue;
#pragma unroll
    for (int i = 0; i < W - 1; ++i) {
      const size_t at = ((size_t)s * (W - 1) + i) * p.C + c0;
      K::st((T *)to + at, from ? K::ld((const T *)from + at) : K::zero());
    }
  }
}

// x before a sequence's start: row i of its state0, or zero
template <typename T, int W, int V>
__device__ __forceinline__ void from_state(const ConvP &p, int s, int i, int c0, f2 (&v)[(V + 1) / 2]) {
  using K = Pack<T, V>;
  get_pairs<T, V>(p.state0 ? K::ld((const T *)p.state0 + ((size_t)s * (W - 1) + i) * p.C + c0) : K::zero(), v);
}

template <typename T, int W, int V>
__global__ void __launch_bounds__(kConvThreads) conv_fwd_kernel(ConvP p) {
  using K = Pack<T, V>;
  constexpr int U = kFwdGroup, P = (V + 1) / 2;
  const int c0 = (blockIdx.y * blockDim.x + threadIdx.x) * V;
  const long long unit = (long long)blockIdx.x * blockDim.y + threadIdx.y;
  const long long units = (long long)p.B * p.runs;
  __shared__ float sh[32 * (V * W + 1)];
  const bool live = c0 < p.C && unit < units;
  const int b = live ? (int)(unit / p.runs) : 0, t0 = live ? (int)(unit % p.runs) * p.run : p.T;
  const long long rb = (long long)b * p.T;  // (rows below are counted from there)
  const int r0 = t0, r1 = t0 + min(p.run, p.T - t0);
  const T *X = (const T *)p.x + c0 + rb * p.x_ld, *xr = X + r0 * p.x_ld;
  T *yr = (T *)p.y + c0 + (rb + r0) * p.y_ld;
  typename K::Raw raw[U], next[U];
  auto load = [&](int g) {  // the group from row g on, xr its first
    if (g + U <= r1) {
#pragma unroll
      for (int u = 0; u < U; ++u) next[u] = K::ld(xr + u * p.x_ld);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) next[u] = g + u < r1 ? K::ld(xr + u * p.x_ld) : K::zero();
    }
    xr += U * p.x_ld;
  };
  load(r0);  // (in flight while the taps come)
  typename K::Raw before[W - 1];
  int qs = 0, qb = 0, qe = 0;  // the sequence, its first row and the one after its last
  if (t0 < p.T) {
    const SeqSpan q = find_seq(p.cu, p.ns, p.T, b, t0);
    qs = q.s;
    qb = (int)(q.begin - rb);
    qe = (int)(q.end - rb);
#pragma unroll
    for (int k = 0; k < W - 1; ++k) before[k] = r0 - 1 - k >= qb ? K::ld(X + (r0 - 1 - k) * p.x_ld) : K::zero();
  }
  f2 tap[W][P], bias[P];
  load_taps<W, V>(p, c0, sh, tap, bias);
  if (live) pass_empty<T, W, V>(p, unit, units, c0, p.state0, p.stateT);
  if (t0 >= p.T) return;
  f2 win[W - 1][P];  // win[k] = x_{t-1-k}
#pragma unroll
  for (int k = 0; k < W - 1; ++k) {
    const int r = r0 - 1 - k;
    if (r >= qb) get_pairs<T, V>(before[k], win[k]);
    else from_state<T, W, V>(p, qs, W - 1 + r - qb, c0, win[k]);
  }
  auto token = [&](const typename K::Raw &raw, T *y) {
    f2 x[P], o[P];
    get_pairs<T, V>(raw, x);
#pragma unroll
    for (int e = 0; e < P; ++e) {
      f2 a = fma2(tap[0][e], x[e], bias[e]);
#pragma unroll
      for (int k = 1; k < W; ++k) a = fma2(tap[k][e], win[k - 1][e], a);
      o[e] = p.silu ? silu2(a) : a;
#pragma unroll
      for (int k = W - 2; k > 0; --k) win[k][e] = win[k - 1][e];
      win[0][e] = x[e];
    }
    K::st(y, put_pairs<T, V>(o));
  };
  auto last_state = [&]() {
#pragma unroll
    for (int k = 0; k < W - 1; ++k)
      K::st((T *)p.stateT + ((size_t)qs * (W - 1) + W - 2 - k) * p.C + c0, put_pairs<T, V>(win[k]));
  };
  for (int g = r0; g < r1; g += U, yr += U * p.y_ld) {
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = next[u];
    load(g + U);
    if (g + U <= r1 && g + U <= qe) {  // whole, within its sequence
#pragma unroll
      for (int u = 0; u < U; ++u) token(raw[u], yr + u * p.y_ld);
      if (g + U == qe && p.stateT) last_state();
      continue;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = g + u;
      if (r >= r1) break;
      if (r >= qe) {  // the next sequence that has tokens (packed rows only)
        while (qs < p.ns - 1 && r >= qe) {
          ++qs;
          qb = qe;
          qe = cu_at(p.cu, p.ns, p.T, qs + 1);
        }
#pragma unroll
        for (int k = 0; k < W - 1; ++k) from_state<T, W, V>(p, qs, W - 2 - k, c0, win[k]);
      }
      token(raw[u], yr + u * p.y_ld);
      if (r == qe - 1 && p.stateT) last_state();
    }
  }
}

template <typename T, int W, int V>
__global__ void __launch_bounds__(kConvThreads) conv_bwd_kernel(ConvP p) {
  using K = Pack<T, V>;
  constexpr int U = kBwdGroup, P = (V + 1) / 2;
  extern __shared__ float sh[];  // [blockDim.y][blockDim.x][V][W + 1]; first the taps
  const int c0 = (blockIdx.y * blockDim.x + threadIdx.x) * V;
  const long long unit = (long long)blockIdx.x * blockDim.y + threadIdx.y;
  const long long units = (long long)p.B * p.runs;
  const bool live = c0 < p.C && unit < units;
  const int b = live ? (int)(unit / p.runs) : 0, t0 = live ? (int)(unit % p.runs) * p.run : p.T;
  const long long rb = (long long)b * p.T;  // (rows below are counted from there)
  const int r0 = t0, r1 = t0 + min(p.run, p.T - t0);
  const int top = min(r1 + W - 2, p.T - 1);  // dx of the last row takes dp of the W-1 rows after it
  const T *X = (const T *)p.x + c0 + rb * p.x_ld, *DY = (const T *)p.dy + c0 + rb * p.dy_ld;
  T *DX = (T *)p.dx + c0 + rb * p.dx_ld;
  // groups [g, g + U) from the top down; xr[i] = x row g - (W-1) + i
  typename K::Raw xr[U + W - 1], xn[U], dyr[U], dyn[U];
  int g = r0 + (top - r0) / U * U;
  const T *xp = X + (g - (W - 1)) * p.x_ld, *dyp = DY + g * p.dy_ld;
  T *dxp = DX + g * p.dx_ld;
  auto load = [&](int at) {  // the rows a group needs beside those of the one above: xp and dyp its first
    if (at >= W - 1 && at + U - 1 <= top && at >= r0) {
#pragma unroll
      for (int i = 0; i < U; ++i) {
        xn[i] = K::ld(xp + i * p.x_ld);
        dyn[i] = K::ld(dyp + i * p.dy_ld);
      }
    } else {
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int r = at - (W - 1) + i;
        xn[i] = r >= 0 && r <= top && at >= r0 ? K::ld(xp + i * p.x_ld) : K::zero();
        dyn[i] = at >= r0 && at + i <= top ? K::ld(dyp + i * p.dy_ld) : K::zero();
      }
    }
    xp -= U * p.x_ld;
    dyp -= U * p.dy_ld;
  };
#pragma unroll
  for (int i = 0; i < W - 1; ++i) {
    const int r = g + U - (W - 1) + i;
    xr[i] = t0 < p.T && r >= 0 && r <= top ? K::ld(X + r * p.x_ld) : K::zero();
  }
  if (t0 < p.T) load(g);  // (in flight while the taps come)
  f2 tap[W][P], bias[P];
  load_taps<W, V>(p, c0, sh, tap, bias);
  f2 dw[W + 1][P];  // dw[k] of tap[k]; dw[W]: the bias
#pragma unroll
  for (int k = 0; k <= W; ++k)
#pragma unroll
    for (int e = 0; e < P; ++e) dw[k][e] = pack2(0.f, 0.f);
  if (live) pass_empty<T, W, V>(p, unit, units, c0, p.dstateT, p.dstate0);
  if (t0 < p.T) {
    const SeqSpan q = find_seq(p.cu, p.ns, p.T, b, top);
    int qs = q.s, qb = (int)(q.begin - rb), qe = (int)(q.end - rb);
    f2 dpw[W - 1][P];  // dpw[k] = dp_{t+1+k} of the same sequence
#pragma unroll
    for (int k = 0; k < W - 1; ++k)
#pragma unroll
      for (int e = 0; e < P; ++e) dpw[k][e] = pack2(0.f, 0.f);
    // dp of one row from its taps, its dx if the row is the run's own
    auto row_dp = [&](const f2 (&x)[W][P], const typename K::Raw &dyr, f2 (&dp)[P]) {
      get_pairs<T, V>(dyr, dp);
      if (p.silu) {
#pragma unroll
        for (int e = 0; e < P; ++e) {
          f2 a = bias[e];
#pragma unroll
          for (int k = 0; k < W; ++k) a = fma2(tap[k][e], x[k][e], a);
          dp[e] = mul2(dp[e], silu_grad2(a));
        }
      }
    };
    auto row_dx = [&](const f2 (&x)[W][P], const f2 (&dp)[P], f2 (&dx)[P]) {
#pragma unroll
      for (int e = 0; e < P; ++e) {
        f2 a = mul2(tap[0][e], dp[e]);
#pragma unroll
        for (int k = 1; k < W; ++k) a = fma2(tap[k][e], dpw[k - 1][e], a);
        dx[e] = a;
#pragma unroll
        for (int k = 0; k < W; ++k) dw[k][e] = fma2(dp[e], x[k][e], dw[k][e]);
        dw[W][e] = add2(dw[W][e], dp[e]);
      }
    };
    auto shift = [&](const f2 (&dp)[P]) {
#pragma unroll
      for (int e = 0; e < P; ++e) {
#pragma unroll
        for (int k = W - 2; k > 0; --k) dpw[k][e] = dpw[k - 1][e];
        dpw[0][e] = dp[e];
      }
    };
    for (; g >= r0; g -= U, dxp -= U * p.dx_ld) {
#pragma unroll
      for (int i = W - 2; i >= 0; --i) xr[U + i] = xr[i];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        xr[i] = xn[i];
        dyr[i] = dyn[i];
      }
      load(g - U);
      if (g + U <= r1 && g - (W - 1) >= qb && g + U <= qe - (p.dstateT ? W - 1 : 0)) {
        f2 x[U + W - 1][P];  // whole, the run's own, inside its sequence
#pragma unroll
        for (int i = 0; i < U + W - 1; ++i) get_pairs<T, V>(xr[i], x[i]);
#pragma unroll
        for (int u = U - 1; u >= 0; --u) {
          f2 taps[W][P], dp[P], dx[P];
#pragma unroll
          for (int k = 0; k < W; ++k)
#pragma unroll
            for (int e = 0; e < P; ++e) taps[k][e] = x[u + W - 1 - k][e];
          row_dp(taps, dyr[u], dp);
          row_dx(taps, dp, dx);
          K::st(dxp + u * p.dx_ld, put_pairs<T, V>(dx));
          shift(dp);
        }
        continue;
      }
#pragma unroll
      for (int u = U - 1; u >= 0; --u) {
        const int r = g + u;
        if (r > top) continue;
        if (r < qb) {  // the sequence before, past empty ones
          while (qs > 0 && r < qb) {
            --qs;
            qe = qb;
            qb = cu_at(p.cu, p.ns, p.T, qs);
          }
#pragma unroll
          for (int k = 0; k < W - 1; ++k)
#pragma unroll
            for (int e = 0; e < P; ++e) dpw[k][e] = pack2(0.f, 0.f);
        }
        f2 x[W][P], dp[P];
#pragma unroll
        for (int k = 0; k < W; ++k) get_pairs<T, V>(xr[u + W - 1 - k], x[k]);
        if (r - (W - 1) < qb) {
#pragma unroll
          for (int k = 1; k < W; ++k)
            if (r - k < qb) from_state<T, W, V>(p, qs, W - 1 + r - k - qb, c0, x[k]);
        }
        row_dp(x, dyr[u], dp);
        if (r < r1) {
          f2 dx[P];
          row_dx(x, dp, dx);
          if (p.dstateT && qe - r <= W - 1) {
            f2 d[P];
            get_pairs<T, V>(K::ld((const T *)p.dstateT + ((size_t)qs * (W - 1) + W - 1 - (qe - r)) * p.C + c0), d);
#pragma unroll
            for (int e = 0; e < P; ++e) dx[e] = add2(dx[e], d[e]);
          }
          K::st(dxp + u * p.dx_ld, put_pairs<T, V>(dx));
        }
        shift(dp);
        if (r == qb && r < r1 && p.dstate0) {
          const int len = qe - qb;
#pragma unroll
          for (int v = 1; v < W; ++v) {  // the input v rows before the start: state row W-1-v
            f2 d[P];
#pragma unroll
            for (int e = 0; e < P; ++e) {
              d[e] = mul2(tap[v][e], dpw[0][e]);
#pragma unroll
              for (int k = v + 1; k < W; ++k) d[e] = fma2(tap[k][e], dpw[k - v][e], d[e]);
            }
            const int i = W - 1 - v;
            if (p.dstateT && i >= len) {  // a sequence shorter than the state hands part of it on
              f2 t[P];
              get_pairs<T, V>(K::ld((const T *)p.dstateT + ((size_t)qs * (W - 1) + i - len) * p.C + c0), t);
#pragma unroll
              for (int e = 0; e < P; ++e) d[e] = add2(d[e], t[e]);
            }
            K::st((T *)p.dstate0 + ((size_t)qs * (W - 1) + i) * p.C + c0, put_pairs<T, V>(d));
          }
        }
      }
    }
  }
  __syncthreads();  // (sh held the taps)
  // the CTA's sums over its runs, in order
  const int row = blockDim.x * V * (W + 1);
  float *mine = sh + threadIdx.y * row + threadIdx.x * V * (W + 1);
#pragma unroll
  for (int k = 0; k <= W; ++k) {
    float v[V];
    from_pairs<V>(dw[k], v);
#pragma unroll
    for (int e = 0; e < V; ++e) mine[e * (W + 1) + (k < W ? W - 1 - k : W)] = v[e];
  }
  __syncthreads();
  const int cbase = blockIdx.y * blockDim.x * V;
  const int tid = threadIdx.y * blockDim.x + threadIdx.x;
  for (int i = tid; i < row; i += blockDim.x * blockDim.y) {
    if (cbase + i / (W + 1) >= p.C) continue;
    float a = 0.f;
    for (int y = 0; y < (int)blockDim.y; ++y) a += sh[y * row + i];
    p.part[((size_t)blockIdx.x * p.C + cbase) * (W + 1) + i] = a;
  }
}

// dw [C][W] and dbias [C] from the partials [parts][C][W + 1], in order
template <int W>
__global__ void __launch_bounds__(512) conv_grad_kernel(const float *__restrict__ part, int C, int parts,
                                                        float *__restrict__ dw, float *__restrict__ dbias) {
  __shared__ float sh[16][32];
  const long long n = (long long)C * (W + 1), i = (long long)blockIdx.x * 32 + threadIdx.x;
  float a = 0.f;
  if (i < n)
    for (int q = threadIdx.y; q < parts; q += 16) a += part[(size_t)q * n + i];
  sh[threadIdx.y][threadIdx.x] = a;
  __syncthreads();
  if (threadIdx.y || i >= n) return;
#pragma unroll
  for (int y = 1; y < 16; ++y) a += sh[y][threadIdx.x];
  const int c = (int)(i / (W + 1)), k = (int)(i % (W + 1));
  if (k < W) dw[(size_t)c * W + k] = a;
  else if (dbias) dbias[c] = a;
}

struct ConvStepP {
  int N, C, num_slots, silu;
  long long x_ld, y_ld;
  const void *x;
  const float *w, *bias;
  void *state, *y;
  const int *slots;
  bool w_vec;  // w on 16 bytes (W = 4: a channel's taps in one access)
};

// One token: a request's W inputs and the taps of V channels per thread, all loads
// but the state's, which waits for the slot, at once.  Bound by the launch and that
// chain of loads: one request of 6144 channels takes 2.2 us in a captured graph, 3.5 with
// the taps loaded one by one.
template <typename T, int W, int V>
__global__ void __launch_bounds__(kConvThreads) conv_step_kernel(ConvStepP p) {
  using K = Pack<T, V>;
  const int c0 = (blockIdx.y * blockDim.x + threadIdx.x) * V;
  const int n = blockIdx.x * blockDim.y + threadIdx.y;
  if (c0 >= p.C || n >= p.N) return;
  const int slot = p.slots ? __ldg(p.slots + n) : n;
  float w[V][W], y[V];  // (loads that do not wait for the slot)
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const float *row = p.w + (size_t)(c0 + e) * W;
    y[e] = p.bias ? __ldg(p.bias + c0 + e) : 0.f;
    if (W == 4 && p.w_vec) {
      const float4 a = __ldg(reinterpret_cast<const float4 *>(row));
      w[e][0] = a.x;
      w[e][1] = a.y;
      w[e][W > 2 ? 2 : 0] = a.z;
      w[e][W > 3 ? 3 : 0] = a.w;
    } else {
#pragma unroll
      for (int j = 0; j < W; ++j) w[e][j] = __ldg(row + j);
    }
  }
  T *Y = (T *)p.y + (size_t)n * p.y_ld + c0;
  if (slot < 0 || slot >= p.num_slots) {
    K::st(Y, K::zero());
    return;
  }
  T *S = (T *)p.state + (size_t)slot * (W - 1) * p.C + c0;
  typename K::Raw raw[W];  // x_{t-W+1} .. x_t
#pragma unroll
  for (int i = 0; i < W - 1; ++i) raw[i] = K::ld(S + (size_t)i * p.C);
  raw[W - 1] = K::ld((const T *)p.x + (size_t)n * p.x_ld + c0);
#pragma unroll
  for (int j = 0; j < W; ++j) {
    float x[V];
    K::get(raw[j], x);
#pragma unroll
    for (int e = 0; e < V; ++e) y[e] = fmaf(w[e][j], x[e], y[e]);
  }
#pragma unroll
  for (int i = 0; i < W - 1; ++i) K::st(S + (size_t)i * p.C, raw[i + 1]);
  if (p.silu) {
#pragma unroll
    for (int e = 0; e < V; ++e) y[e] = siluf(y[e]);
  }
  K::st(Y, K::put(y));
}

// Whether every row of the tensors that are given starts on a multiple of
// `bytes` (pointers and strides in elements of `size` bytes).
bool rows_on(size_t bytes, size_t size, std::initializer_list<std::pair<const void *, long long>> rows) {
  for (const auto &r : rows)
    if (r.first && (((uintptr_t)r.first | ((size_t)r.second * size)) & (bytes - 1))) return false;
  return true;
}

struct ConvPlan {
  int run, runs;      // tokens per thread, runs per batch row
  unsigned bx, by;    // CTA: channel vectors, runs
  unsigned gx, gy;    // grid: CTAs over the runs, over the channels
};
// Threads want long runs (each reads W-1 rows above its own again, its taps, and
// in the backward W-1 rows of dy), the GPU wants threads: runs of 64 tokens where
// there are 512 threads per SM left, else as many as leave those, 8 at least.
// (8 x 4096 tokens of 2048 channels: forward 88 us in runs of 8, 69 of 16, 59 of
// 64, 70 of 256; backward 198, 139, 103, 123; with four channels a thread in the
// forward too, 50 of 64 and 54 of 128.)
ConvPlan conv_plan(const rdn_conv_args &a, int V) {
  ConvPlan pl;
  const long long nvec = (a.C + V - 1) / V, tokens = (long long)a.B * a.T;
  long long run = tokens * nvec / (152ll * 512) / kRunStep * kRunStep;
  pl.run = (int)(run < kRunStep ? kRunStep : run > kRunMost ? kRunMost : run);
  pl.runs = a.T > 0 ? (a.T + pl.run - 1) / pl.run : 1;
  pl.bx = 32;
  while (pl.bx > 1 && pl.bx / 2 >= nvec) pl.bx /= 2;
  pl.by = kConvThreads / pl.bx;
  pl.gx = (unsigned)(((long long)a.B * pl.runs + pl.by - 1) / pl.by);
  pl.gy = (unsigned)((nvec + pl.bx - 1) / pl.bx);
  return pl;
}

// Four channels per thread (in the backward the registers hold up to 4 W + 1
// values per channel; in the forward 8 bf16 channels leave room for the loads of 4
// tokens instead of 8: 56 us instead of 50 at 8 x 4096 x 2048); single ones where
// the rows do not lie on that access.
bool conv_vec(const rdn_conv_args &a, bool bwd) {
  const size_t size = a.dtype == RDN_BF16 ? 2 : 4;
  const int V = 4;
  const size_t bytes = V * size;
  if (a.C % V) return false;
  return bwd ? rows_on(bytes, size, {{a.x, a.x_ld}, {a.dy, a.dy_ld}, {a.dx, a.dx_ld}, {a.state0, 0},
                                     {a.dstateT, 0}, {a.dstate0, 0}})
             : rows_on(bytes, size, {{a.x, a.x_ld}, {a.y, a.y_ld}, {a.state0, 0}, {a.stateT, 0}});
}

ConvP conv_params(const rdn_conv_args &a, const ConvPlan &pl) {
  ConvP p{};
  p.B = a.B; p.T = a.T; p.C = a.C;
  p.ns = a.cu_seqlens ? a.num_seqs : a.B;
  p.run = pl.run; p.runs = pl.runs; p.silu = a.silu;
  p.x_ld = a.x_ld; p.y_ld = a.y_ld; p.dy_ld = a.dy_ld; p.dx_ld = a.dx_ld;
  p.x = a.x; p.state0 = a.state0; p.dy = a.dy; p.dstateT = a.dstateT;
  p.y = a.y; p.stateT = a.stateT; p.dx = a.dx; p.dstate0 = a.dstate0;
  p.w = a.w; p.bias = a.bias; p.cu = a.cu_seqlens;
  p.part = static_cast<float *>(a.workspace);
  return p;
}

template <typename T, int W, int V>
cudaError_t fwd_t(const rdn_conv_args &a, cudaStream_t s) {
  const ConvPlan pl = conv_plan(a, V);
  const ConvP p = conv_params(a, pl);
  RDN_LAUNCH("conv_fwd", s,
             (conv_fwd_kernel<T, W, V><<<dim3(pl.gx, pl.gy), dim3(pl.bx, pl.by), 0, s>>>(p)));
  return cudaGetLastError();
}
template <typename T, int W, int V>
cudaError_t bwd_t(const rdn_conv_args &a, cudaStream_t s) {
  const ConvPlan pl = conv_plan(a, V);
  const ConvP p = conv_params(a, pl);
  const size_t smem = sizeof(float) * kConvThreads * (V * (W + 1) + 1);
  RDN_LAUNCH("conv_bwd", s,
             (conv_bwd_kernel<T, W, V><<<dim3(pl.gx, pl.gy), dim3(pl.bx, pl.by), smem, s>>>(p)));
  const unsigned grid = (unsigned)(((long long)a.C * (W + 1) + 31) / 32);
  RDN_LAUNCH("conv_grad", s,
             (conv_grad_kernel<W><<<grid, dim3(32, 16), 0, s>>>(p.part, a.C, (int)pl.gx, a.dw, a.dbias)));
  return cudaGetLastError();
}
template <typename T, int W>
cudaError_t conv_w(const rdn_conv_args &a, bool bwd, cudaStream_t s) {
  const bool vec = conv_vec(a, bwd);
  if (bwd) return vec ? bwd_t<T, W, 4>(a, s) : bwd_t<T, W, 1>(a, s);
  return vec ? fwd_t<T, W, 4>(a, s) : fwd_t<T, W, 1>(a, s);
}
template <typename T>
cudaError_t conv_d(const rdn_conv_args &a, bool bwd, cudaStream_t s) {
  return a.W == 2 ? conv_w<T, 2>(a, bwd, s) : a.W == 3 ? conv_w<T, 3>(a, bwd, s) : conv_w<T, 4>(a, bwd, s);
}

template <typename T, int W, int V>
cudaError_t step_t(const ConvStepP &p, cudaStream_t s) {
  const int nvec = (p.C + V - 1) / V;
  unsigned bx = kConvThreads;
  while (bx > 32 && bx / 2 >= (unsigned)nvec) bx /= 2;
  const unsigned by = kConvThreads / bx;
  RDN_LAUNCH("conv_step", s,
             (conv_step_kernel<T, W, V><<<dim3((p.N + by - 1) / by, (nvec + bx - 1) / bx), dim3(bx, by), 0, s>>>(p)));
  return cudaGetLastError();
}
template <typename T, int V>
cudaError_t step_w(const ConvStepP &p, int W, cudaStream_t s) {
  return W == 2 ? step_t<T, 2, V>(p, s) : W == 3 ? step_t<T, 3, V>(p, s) : step_t<T, 4, V>(p, s);
}

}  // namespace

size_t conv_bwd_bytes(const rdn_conv_args &a) {
  // (the larger of the two accesses' plans: the query sees no pointers)
  const ConvPlan v = conv_plan(a, 4), e = conv_plan(a, 1);
  const size_t parts = v.gx > e.gx ? v.gx : e.gx;
  return round256(sizeof(float) * parts * a.C * (a.W + 1));
}

cudaError_t launch_conv(const rdn_conv_args &a, bool bwd, cudaStream_t s) {
  return a.dtype == RDN_BF16 ? conv_d<__nv_bfloat16>(a, bwd, s) : conv_d<float>(a, bwd, s);
}

cudaError_t launch_conv_step(const rdn_conv_step_args &a, cudaStream_t s) {
  ConvStepP p{a.N, a.C, a.num_slots, a.silu, a.x_ld, a.y_ld, a.x, a.w, a.bias, a.state, a.y, a.slots,
              ((uintptr_t)a.w & 15) == 0};
  const size_t size = a.dtype == RDN_BF16 ? 2 : 4;
  const bool vec = a.C % (16 / size) == 0 && rows_on(16, size, {{a.x, a.x_ld}, {a.y, a.y_ld}, {a.state, 0}});
  if (a.dtype == RDN_BF16)
    return vec ? step_w<__nv_bfloat16, 8>(p, a.W, s) : step_w<__nv_bfloat16, 1>(p, a.W, s);
  return vec ? step_w<float, 4>(p, a.W, s) : step_w<float, 1>(p, a.W, s);
}

}  // namespace rdn
