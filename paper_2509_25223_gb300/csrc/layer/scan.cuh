// scan.cuh -- what the selective scan's kernels share: the work's layout over
// the GPU, the decay's exponential and the parameters.
//
// The scan is a recurrence per (channel d, state n),
//     h_t = a_t h_{t-1} + dl_t x_t B_t[n],   a_t = exp(dl_t A[d,n]),
// one exponential and about four multiply-adds per (token, channel, state): 16
// states cost about as many FMA-pipe and exponential cycles as their channel's
// 8 to 14 bytes per token cost in HBM, so the kernels keep every state in
// registers from one end of a run of tokens to the other and touch HBM once.
//
// A warp's lanes are L state lanes (4 states each, L = 2 .. 16) times 32 / L
// channel lanes (4 channels each): 16 (channel, state) pairs per lane, worked
// on as packed pairs of channels.  What limits the loop beside the FMA pipe and
// the exponentials is what shared memory hands out (128 bytes per clock and SM,
// to the lanes, equal addresses or not): per token a lane takes 4 states of B
// and C and 4 channels' (dl, dl x), 12 to 16 words for 16 pairs.  A lane per
// channel takes 34 for as many, 2 channels by 4 states 24 (measured 1.5 times
// as long).  A sum over the states takes 3 exchanges for 4 channels.
//
// A sequence is cut into units of `seg` tokens where there are too few
// channels and sequences to fill the GPU: a first pass finds each unit's end
// state from a zero start and the sum of its dl; since A is constant in time
// the decay over a unit is exp(A sum dl), so a unit's start state is a short
// chain over the units before it (the backward likewise, from the end).
#pragma once
#include "rows.cuh"

namespace rdn {

constexpr int kScanThreads = 64, kScanWarps = 2;  // small CTAs: their number divides over the SMs finely
constexpr int kScanTile = RDN_SCAN_CHUNK;  // tokens staged at a time, and between kept states

// A's factor in the decay's exponent, A log2 e.  An infinite one (A of -inf: a state without
// memory) counts as the largest finite number, so that a step of zero, as the tokens past a
// sequence's end have, makes a decay of one as it does for every other A, not 0 times infinity;
// NaN stays.
__device__ __forceinline__ float log2_rate(float A) {
  const float r = A * kLog2e, most = 3.402823466e38f;
  return r > most ? most : r < -most ? -most : r;
}

// exp2 of the decay's exponent.  ex2.approx comes out low by about 2e-8 on
// average for small arguments; with decays near 1 the factors of a thousand
// tokens multiply, and the mean error adds up where rounding would average
// out.  kExpShift (added in the multiply that forms the argument, at no cost)
// takes the mean below 5e-9 for exponents in [-0.5, 0]; expf has 1e-8 to
// 1.5e-8 there.
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kExpShift = 2.5e-8f;
__device__ __forceinline__ float decay(float dl, float A2) { return ex2(fmaf(dl, A2, kExpShift)); }

// decay() of a pair
__device__ __forceinline__ f2 decay2(f2 dl, f2 A2, f2 shift) {
  float lo, hi;
  unpack2(fma2(dl, A2, shift), lo, hi);
  return pack2(ex2(lo), ex2(hi));
}

// softplus(v) = max(v, 0) + log1p(u), u = exp(-|v|); log1p(u) = 2 atanh(t), t = u / (2 + u) <= 1/3,
// with atanh(t) / t as a polynomial in t^2 fitted to 8e-9 on [0, 1/9].  About 14 instructions
// (the library's log1p takes three times as many, and log2 of 1 + u would lose a small u).  The
// exponent |v| log2 e is rounded to 32 bits, so below zero the relative error grows with |v|: at
// most 7.3e-8 |v| + 7e-7.  (With the other operations exact, 4 units in the last place on [-1, 1],
// 16 on [-20, -10], 62 at -80, where the result is 1e-35; above 1 one unit.)
__device__ __forceinline__ float softplusf(float v) {
  const float u = ex2(fabsf(v) * -kLog2e);
  const float t = u * rcp_approx(2.f + u), q = t * t;
  float a = fmaf(0.28178335f, q, 0.27960603f);
  a = fmaf(a, q, 0.40024910f);
  a = fmaf(a, q, 0.66666315f);
  a = fmaf(a, q, 2.f);
  return fmaf(t, a, fmaxf(v, 0.f));
}
// of a pair
__device__ __forceinline__ f2 softplus2(f2 v) {
  float x, y;
  unpack2(v, x, y);
  const float u0 = ex2(fabsf(x) * -kLog2e), u1 = ex2(fabsf(y) * -kLog2e);
  const f2 u = pack2(u0, u1);
  float w0, w1;
  unpack2(add2(u, pack2(2.f, 2.f)), w0, w1);
  const f2 t = mul2(u, pack2(rcp_approx(w0), rcp_approx(w1))), q = mul2(t, t);
  f2 a = fma2(pack2(0.28178335f, 0.28178335f), q, pack2(0.27960603f, 0.27960603f));
  a = fma2(a, q, pack2(0.40024910f, 0.40024910f));
  a = fma2(a, q, pack2(0.66666315f, 0.66666315f));
  a = fma2(a, q, pack2(2.f, 2.f));
  return fma2(t, a, pack2(fmaxf(x, 0.f), fmaxf(y, 0.f)));
}

struct ScanP {
  int B, T, D, S, G, ns;
  int softplus;
  int seg;          // tokens per unit (a multiple of kScanTile)
  int units, units_row;  // units of the call (packed: a bound); without cu: per sequence
  int tiles_g;      // channel tiles per group
  bool bc_vec;      // rows of B and C on 16 bytes
  long long x_ld, dt_ld, z_ld, b_ld, c_ld, out_ld, dout_ld, dx_ld, ddt_ld, dz_ld;
  const void *x, *dt, *z, *Bm, *Cm, *dout;
  const float *A, *Dskip, *dt_bias, *h0, *dhT;
  void *out, *dx, *ddt, *dz;
  float *hT, *chunks, *dh0;
  const int *cu;
  long long slots;              // blocks in chunks (a bound kept even for a broken table)
  float *carry, *sumd;          // [units][D][4 L], [units][D]: the first pass's results
  float *part_bc;               // [channel tiles][B * T][8 L]: dB and dC of a tile's channels
  float *part_A;                // [units][D][S]
  float *part_D;                // [units][2][D]: dD and ddt_bias
};

// A unit of work: tokens [begin + j * seg, ..) of a sequence.
struct Unit {
  bool ok;
  int s, j, n;              // sequence, unit within it, its units
  long long begin, end;     // the sequence's rows
  long long chunk0;         // its first slot of the kept states
};
// Unit u of the call, found by a whole warp (packed: a scan over the table).
__device__ __forceinline__ Unit find_unit(const ScanP &p, int u) {
  Unit w;
  if (!p.cu) {
    w.ok = true;
    w.s = u / p.units_row;
    w.j = u % p.units_row;
    w.n = p.units_row;
    w.begin = (long long)w.s * p.T;
    w.end = w.begin + p.T;
    w.chunk0 = (long long)w.s * ((p.T + kScanTile - 1) / kScanTile);
    return w;
  }
  const int lane = threadIdx.x & 31;
  int before = 0;  // units of the sequences before this group of 32
  long long chunks = 0;
  for (int base = 0; base < p.ns; base += 32) {
    const int s = base + lane;
    int from = 0, len = 0, nu = 0;
    if (s < p.ns) {
      from = cu_at(p.cu, p.ns, p.T, s);
      len = max(cu_at(p.cu, p.ns, p.T, s + 1) - from, 0);
      nu = max((len + p.seg - 1) / p.seg, 1);
    }
    int nc = (len + kScanTile - 1) / kScanTile;
    int iu = nu, ic = nc;  // inclusive sums over the lanes
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int a = __shfl_up_sync(0xffffffffu, iu, o), b = __shfl_up_sync(0xffffffffu, ic, o);
      if (lane >= o) {
        iu += a;
        ic += b;
      }
    }
    const unsigned hit = __ballot_sync(0xffffffffu, u >= before + iu - nu && u < before + iu);
    if (hit) {
      const int src = __ffs(hit) - 1;
      w.ok = true;
      w.s = base + src;
      w.n = __shfl_sync(0xffffffffu, nu, src);
      w.j = u - before - (__shfl_sync(0xffffffffu, iu, src) - w.n);
      w.n = min(w.n, p.units - (u - w.j));  // (a broken table may ask for more units than there are)
      w.begin = __shfl_sync(0xffffffffu, from, src);
      w.end = w.begin + __shfl_sync(0xffffffffu, len, src);
      w.chunk0 = chunks + __shfl_sync(0xffffffffu, ic - nc, src);
      return w;
    }
    before += __shfl_sync(0xffffffffu, iu, 31);
    chunks += __shfl_sync(0xffffffffu, ic, 31);
  }
  w.ok = false;
  return w;
}

// The shape of a CTA's work for L state lanes.
template <typename T, int L, bool VEC>
struct ScanShape {
  static constexpr int CL = 32 / L;                // channel lanes
  static constexpr int CW = 4 * CL;                // channels of a warp
  static constexpr int CT = kScanWarps * CW;       // and of a CTA
  static constexpr int SP = 4 * L;                 // states, padded
  static constexpr int V = VEC ? kVec<T> : 1;      // channels per global access
  static constexpr int COLS = CT / V;              // accesses per token
  static constexpr int NV = (kScanTile * COLS + kScanThreads - 1) / kScanThreads;  // per thread
  using K = Pack<T, V>;
  using Raw = typename K::Raw;
  // access i of this thread: its token and its first channel in the tile
  __device__ static int tok(int i) { return (i * kScanThreads + (int)threadIdx.x) / COLS; }
  __device__ static int chan(int i) { return (i * kScanThreads + (int)threadIdx.x) % COLS * V; }
};

// A slot of shared memory filled from global memory (zero if src is NULL),
// 16-byte ones without a register in between (fetched() waits for them).
template <typename Raw>
__device__ __forceinline__ void fetch(Raw *slot, const void *src) {
  if constexpr (sizeof(Raw) == 16) {
    if (src) {
      const uint32_t to = (uint32_t)__cvta_generic_to_shared(slot);
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(src) : "memory");
      return;
    }
  }
  Raw v{};
  if (src) v = *static_cast<const Raw *>(src);
  *slot = v;
}
__device__ __forceinline__ void prefetch(const void *p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }
__device__ __forceinline__ void fetched() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// One operand's tile into the threads' own slots: tokens [0, ntok) from `base`
// (channel column included), channels [0, nch).
template <typename Sh, typename T>
__device__ __forceinline__ void fetch_rows(typename Sh::Raw (*slot)[kScanThreads], const T *base, long long ld, int ntok,
                                           int nch) {
#pragma unroll
  for (int i = 0; i < Sh::NV; ++i) {
    const int t = Sh::tok(i), c = Sh::chan(i);
    fetch(&slot[i][threadIdx.x], base && t < ntok && c < nch ? base + t * ld + c : nullptr);
  }
}
// B or C of a tile, in the inputs' type (zero past S and ntok)
template <int SP, typename T>
__device__ __forceinline__ void fetch_states(T (*dst)[SP], const T *base, long long ld, int ntok, int S, bool vec) {
  constexpr int V = kVec<T>;
  if (vec) {
    for (int id = threadIdx.x; id < kScanTile * SP / V; id += kScanThreads) {
      const int t = id / (SP / V), n = id % (SP / V) * V;
      fetch(reinterpret_cast<uint4 *>(&dst[t][n]), t < ntok && n < S ? base + t * ld + n : nullptr);
    }
  } else {
    for (int id = threadIdx.x; id < kScanTile * SP; id += kScanThreads) {
      const int t = id / SP, n = id % SP;
      dst[t][n] = t < ntok && n < S ? base[t * ld + n] : from_f32<T>(0.f);
    }
  }
}

// 4 consecutive states of B or C from shared memory, each in both halves of a
// pair; in the order n ^ perm (perm < 4, the lane's own).
__device__ __forceinline__ void states4(const __nv_bfloat16 *row, int perm, f2 (&v)[4]) {
  const uint2 w = *reinterpret_cast<const uint2 *>(row);
  const uint32_t lo = perm & 2 ? w.y : w.x, hi = perm & 2 ? w.x : w.y;
  const uint32_t even = perm & 1 ? 0x3244u : 0x1044u, odd = perm & 1 ? 0x1044u : 0x3244u;  // bytes (x y 0 0)
  const uint32_t a[4] = {__byte_perm(lo, 0u, even), __byte_perm(lo, 0u, odd), __byte_perm(hi, 0u, even),
                         __byte_perm(hi, 0u, odd)};
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = pack2(__uint_as_float(a[i]), __uint_as_float(a[i]));
}
// out[i] = v[i ^ perm]
__device__ __forceinline__ void permute(const float (&v)[4], int perm, float (&out)[4]) {
  const bool b0 = perm & 1, b1 = perm & 2;
  float a[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) a[i] = b0 ? v[i ^ 1] : v[i];
#pragma unroll
  for (int i = 0; i < 4; ++i) out[i] = b1 ? a[i ^ 2] : a[i];
}
__device__ __forceinline__ void states4(const float *row, int perm, f2 (&v)[4]) {
  const float4 w = *reinterpret_cast<const float4 *>(row);
  const float a[4] = {w.x, w.y, w.z, w.w};
  float b[4];
  permute(a, perm, b);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = pack2(b[i], b[i]);
}

// Where the 16-byte entry of channel pair c lies in a row of them: the threads
// of a phase, which write the same entry of consecutive groups of 4 or 2 pairs,
// then write 8 different ones of the 8 that a 128-byte line of banks holds.
__device__ __forceinline__ int spread16(int c) { return c ^ ((c >> 3) & 3); }

// A lane's part (pairs v[0], v[1] of channels) of the sums over the states,
// summed over the L state lanes into row[channel].  v[0] holds the pair
// 2 cl + (sl & 1) of the warp, v[1] the other: the lanes that exchange hold
// them in opposite orders, so the first exchange needs no selects.
template <int L>
__device__ __forceinline__ void sum_states(const f2 (&v)[2], float *row, int first, int sl) {
  constexpr unsigned all = 0xffffffffu;
  float a, b, c, d;
  unpack2(v[0], a, b);
  unpack2(v[1], c, d);
  a += __shfl_xor_sync(all, c, 1);
  b += __shfl_xor_sync(all, d, 1);
  const int pair = first + 2 * (sl & 1);  // (first: channel of the lane's first pair in the tile)
  if (L == 2) {
    *reinterpret_cast<float2 *>(row + pair) = make_float2(a, b);
    return;
  }
  const bool hi = sl & 2;
  float r = (hi ? b : a) + __shfl_xor_sync(all, hi ? a : b, 2);
  if (L >= 8) r += __shfl_xor_sync(all, r, 4);
  if (L >= 16) r += __shfl_xor_sync(all, r, 8);
  if (sl < 4) row[pair + (hi ? 1 : 0)] = r;
}

// 4 consecutive states n0 .. n0 + 3 of a row of S (zero past S), and their store
__device__ __forceinline__ void load_states(const float *row, int S, int n0, float (&v)[4]) {
  if (S % 4 == 0) {
    const float4 a = n0 < S ? *reinterpret_cast<const float4 *>(row + n0) : make_float4(0.f, 0.f, 0.f, 0.f);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = n0 + i < S ? row[n0 + i] : 0.f;
  }
}
__device__ __forceinline__ void store_states(float *row, int S, int n0, const float (&v)[4]) {
  if (S % 4 == 0) {
    if (n0 < S) *reinterpret_cast<float4 *>(row + n0) = make_float4(v[0], v[1], v[2], v[3]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n0 + i < S) row[n0 + i] = v[i];
  }
}

// The states v of a lane's 4 channels (from channel d0 on, `left` of them in the
// tile; those of the lane's first pair first) over the units from, from + step, ..
// before `to`: v <- exp(A sum dl) v + the unit's result.  All channels' loads of
// a few units are in flight together: one channel after the other the chain of a
// late unit took longer than its tokens.
template <int SP>
__device__ __forceinline__ void chain(const ScanP &p, int from, int to, int step, int d0, int left, int sl,
                                      const float (&a)[4][4], float (&v)[4][4]) {
#pragma unroll 2
  for (int u = from; u != to; u += step) {
    float sd[4];
    float4 x[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int k = 2 * ((c >> 1) ^ (sl & 1)) + (c & 1);
      const size_t at = (size_t)u * p.D + d0 + k;
      sd[c] = k < left ? p.sumd[at] : 0.f;
      x[c] = k < left ? *reinterpret_cast<const float4 *>(p.carry + at * SP + sl * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      v[c][0] = fmaf(decay(sd[c], a[c][0]), v[c][0], x[c].x);
      v[c][1] = fmaf(decay(sd[c], a[c][1]), v[c][1], x[c].y);
      v[c][2] = fmaf(decay(sd[c], a[c][2]), v[c][2], x[c].z);
      v[c][3] = fmaf(decay(sd[c], a[c][3]), v[c][3], x[c].w);
    }
  }
}

// V consecutive floats of shared memory (16 bytes at a time where V is a multiple of 4)
template <int V>
__device__ __forceinline__ void load_vec(const float *p, float (&v)[V]) {
  if constexpr (V % 4 == 0) {
#pragma unroll
    for (int e = 0; e < V; e += 4) {
      const float4 a = *reinterpret_cast<const float4 *>(p + e);
      v[e] = a.x; v[e + 1] = a.y; v[e + 2] = a.z; v[e + 3] = a.w;
    }
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = p[e];
  }
}
template <int V>
__device__ __forceinline__ void store_vec(float *p, const float (&v)[V]) {
  if constexpr (V % 4 == 0) {
#pragma unroll
    for (int e = 0; e < V; e += 4) *reinterpret_cast<float4 *>(p + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) p[e] = v[e];
  }
}

// the same as pairs (V = 1: with a zero)
template <int V>
__device__ __forceinline__ void get_pairs(const float *p, f2 (&v)[(V + 1) / 2]) {
  float a[V];
  load_vec<V>(p, a);
  to_pairs<V>(a, v);
}
template <int V>
__device__ __forceinline__ void put_pairs(float *p, const f2 (&v)[(V + 1) / 2]) {
  float a[V];
  from_pairs<V>(v, a);
  store_vec<V>(p, a);
}

// o *= silu(z) of V channels
template <int V>
__device__ __forceinline__ void silu_gate(const float (&z)[V], float (&o)[V]) {
  if constexpr (V % 2 == 0) {
#pragma unroll
    for (int e = 0; e < V; e += 2) unpack2(mul2(pack2(o[e], o[e + 1]), silu2(pack2(z[e], z[e + 1]))), o[e], o[e + 1]);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) o[e] *= siluf(z[e]);
  }
}

// a parameter of V channels from d on (zero where there is none; V > 1: on 16 bytes)
template <int V>
__device__ __forceinline__ void param(const float *p, int d, bool on, float (&v)[V]) {
#pragma unroll
  for (int e = 0; e < V; ++e) v[e] = 0.f;
  if (p && on) load_vec<V>(p + d, v);
}

// V channels' step sizes from dt: bias, softplus; none for a token past the
// end (dl = 0: a decay of exactly 1, nothing added).
template <int V>
__device__ __forceinline__ void step_sizes(const ScanP &p, const float (&bias)[V], bool live, float (&dl)[V]) {
#pragma unroll
  for (int e = 0; e < V; ++e) dl[e] += bias[e];
  if (p.softplus) {
    if constexpr (V % 2 == 0) {
#pragma unroll
      for (int e = 0; e < V; e += 2) unpack2(softplus2(pack2(dl[e], dl[e + 1])), dl[e], dl[e + 1]);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) dl[e] = softplusf(dl[e]);
    }
  }
  if (!live) {
#pragma unroll
    for (int e = 0; e < V; ++e) dl[e] = 0.f;
  }
}
template <int V>
__device__ __forceinline__ void step_sizes(const ScanP &p, const float *bias, bool live, float (&dl)[V]) {
  float b[V];
  load_vec<V>(bias, b);
  step_sizes<V>(p, b, live, dl);
}
// Two values of each of V channels from channel c on into a token's row of
// entries (a, a', b, b') of channel pairs.
template <int V>
__device__ __forceinline__ void store_two(float4 *row, int c, const float (&a)[V], const float (&b)[V]) {
  if constexpr (V % 2 == 0) {
#pragma unroll
    for (int e = 0; e < V; e += 2) row[spread16((c + e) / 2)] = make_float4(a[e], a[e + 1], b[e], b[e + 1]);
  } else {
    float *at = reinterpret_cast<float *>(row + spread16(c / 2)) + (c & 1);
    at[0] = a[0];
    at[2] = b[0];
  }
}
// (dl, dl x) of V channels
template <int V>
__device__ __forceinline__ void store_steps(float4 *row, int c, const float (&dl)[V], const float (&x)[V]) {
  float dx[V];
#pragma unroll
  for (int e = 0; e < V; ++e) dx[e] = dl[e] * x[e];
  store_two<V>(row, c, dl, dx);
}
// States n0 .. n0 + 3 of the channel pair `pair` of the tile into block `block`
// of to[..][D][S].
__device__ __forceinline__ void store_pairs(float *to, long long block, bool on, const ScanP &p, int c0, int pair,
                                            int nch, int n0, const f2 (&h)[4]) {
  float v[2][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) unpack2(h[i], v[0][i], v[1][i]);
#pragma unroll
  for (int e = 0; e < 2; ++e)
    if (on && pair + e < nch) store_states(to + ((size_t)block * p.D + c0 + pair + e) * p.S, p.S, n0, v[e]);
}

// Dynamic shared memory beyond 48 KB has to be asked for.
template <typename F>
inline cudaError_t allow_smem(F kernel, int bytes) {
  return bytes <= 48 * 1024 ? cudaSuccess
                            : cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

struct ScanPlan {
  int L, CT, tiles_g, tiles;
  int seg, units, units_row;
  bool split;  // some sequence may have more than one unit
};
long long scan_slots(const rdn_scan_args &a);
// The forward without out (and hT): the kept states alone, into p.chunks.
cudaError_t scan_states(const rdn_scan_args &a, ScanP p, const ScanPlan &pl, cudaStream_t s);
ScanPlan scan_plan(const rdn_scan_args &a, bool bwd);
ScanP scan_params(const rdn_scan_args &a, const ScanPlan &pl);
bool scan_vec(const rdn_scan_args &a, bool bwd);

}  // namespace rdn
