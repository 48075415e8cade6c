// scan.cu -- the selective state space scan, forward, and its step of one token:
//     h_t = exp(dl_t A) h_{t-1} + dl_t x_t B_t,  y_t = C_t . h_t + Dskip x_t,
//     out_t = y_t SiLU(z_t),  dl_t = softplus(dt_t + dt_bias)
// (layout and units: scan.cuh).
//
// A CTA owns 256 / L channels of one unit.  Per tile of 16 tokens its threads
// turn the loaded dt and x into (dl, dl x) in shared memory, where B and C are in
// their own type, then run the 16 steps from registers and shared memory alone; the
// sums over the states come back through shared memory to the threads that
// hold x and z of the same elements, which finish and store them.  The next
// tile's global loads are in flight during the steps.
//
// At 4096 channels of 16 states, bf16, with softplus and gate: 16384 tokens 525 us
// (first pass 209, main pass 317: 3.4e12 (token, channel, state) per second, of
// 538 MB), 777 tokens 45 us (19 and 29), 4 x 2048 tokens with the kept states 112
// and 176 us.  4 multiply-adds and an exponential per state are 116 us of either
// pipe at 16384 tokens; the main pass issues 8 instructions per state, of which
// about 3 are work per (token, channel) spread over 16 states (softplus, gate,
// conversions, stores), and keeps issue slots 62 %, shared memory 54 %, FMA 51 % and
// exponentials 43 % busy.  Registers and shared memory (27 KB a CTA) both hold 8 CTAs per
// SM; whether more warps would help is open.  Launch bounds of 9 and 10 CTAs, which leave
// fewer registers but, by the shared memory, no more warps, took 564 and 572 us where 8
// took 552 (with the sums over the states after every token).
#include <math.h>

#include "scan.cuh"

namespace rdn {
namespace {

constexpr int kGroup = 4;  // tokens whose sums over the states follow together (16384 tokens: 2 549 us, 4 527, 8 524)

template <typename T, int L, bool VEC>
struct FwdSmem {
  using Sh = ScanShape<T, L, VEC>;
  float4 dx[kScanTile][Sh::CT / 2];                       // (dl, dl', dl x, dl' x') of a pair, at spread16
  float y[kScanTile][Sh::CT];
  typename Sh::Raw raw[2][3][Sh::NV][kScanThreads];       // each thread's x, dt, z: this tile's and the next's
  T B[2][kScanTile][Sh::SP], C[2][kScanTile][Sh::SP];
  float bias[Sh::CT], D[Sh::CT];
};

// FIRST: the first pass over the units (end state from a zero start, sum of dl).
template <typename T, int L, bool VEC, bool FIRST>
__global__ void __launch_bounds__(kScanThreads, 8) scan_fwd_kernel(ScanP p) {
  using Sh = ScanShape<T, L, VEC>;
  using K = typename Sh::K;
  constexpr int V = Sh::V;
  extern __shared__ __align__(16) unsigned char smem_raw[];
  FwdSmem<T, L, VEC> &sm = *reinterpret_cast<FwdSmem<T, L, VEC> *>(smem_raw);
  const Unit w = find_unit(p, blockIdx.x);
  if (!w.ok || (FIRST && w.j == w.n - 1)) return;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int sl = lane % L, cl = lane / L, n0 = sl * 4;
  const int g = blockIdx.y / p.tiles_g, Dg = p.D / p.G;
  const int c0 = g * Dg + blockIdx.y % p.tiles_g * Sh::CT;  // the tile's first channel
  const int nch = min(Sh::CT, (g + 1) * Dg - c0);
  const int first = warp * Sh::CW + cl * 4;                 // this lane's first channel in the tile
  int at[2];                                                // entries of its pairs
#pragma unroll
  for (int j = 0; j < 2; ++j) at[j] = spread16(first / 2 + (j ^ (sl & 1)));
  for (int c = tid; c < Sh::CT; c += kScanThreads) {
    sm.bias[c] = p.dt_bias && c < nch ? p.dt_bias[c0 + c] : 0.f;
    sm.D[c] = p.Dskip && c < nch ? p.Dskip[c0 + c] : 0.f;
  }
  // channel pair j, state n0 + i
  f2 A2[2][4], h[2][4], sumd[2];
  const f2 shift = pack2(kExpShift, kExpShift);
  float a[4][4], v[4][4];  // of this lane's 4 channels, pair by pair
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const int ch = first + 2 * ((c >> 1) ^ (sl & 1)) + (c & 1);
    const bool on = ch < nch;
    const size_t d = c0 + ch;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[c][i] = v[c][i] = 0.f;
    if (on) load_states(p.A + d * p.S, p.S, n0, a[c]);
    if (on && !FIRST && p.h0) load_states(p.h0 + ((size_t)w.s * p.D + d) * p.S, p.S, n0, v[c]);
#pragma unroll
    for (int i = 0; i < 4; ++i) a[c][i] = log2_rate(a[c][i]);
  }
  if (!FIRST) chain<Sh::SP>(p, blockIdx.x - w.j, blockIdx.x, 1, c0 + first, nch - first, sl, a, v);
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    sumd[j] = pack2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      A2[j][i] = pack2(a[2 * j][i], a[2 * j + 1][i]);
      h[j][i] = pack2(v[2 * j][i], v[2 * j + 1][i]);
    }
  }
  const long long r0 = w.begin + (long long)w.j * p.seg;
  const long long r1 = min(r0 + p.seg, w.end);
  const bool out = !FIRST && p.out;
  const T *X = (const T *)p.x + c0, *DT = (const T *)p.dt + c0, *Z = p.z ? (const T *)p.z + c0 : nullptr;
  const T *Bm = (const T *)p.Bm + (size_t)g * p.S, *Cm = (const T *)p.Cm + (size_t)g * p.S;
  auto load = [&](long long r, int b) {
    const int ntok = (int)max(0ll, min((long long)kScanTile, r1 - r));
    fetch_rows<Sh>(sm.raw[b][0], X + r * p.x_ld, p.x_ld, ntok, nch);
    fetch_rows<Sh>(sm.raw[b][1], DT + r * p.dt_ld, p.dt_ld, ntok, nch);
    fetch_states(sm.B[b], Bm + r * p.b_ld, p.b_ld, ntok, p.S, p.bc_vec);
    if (out) {
      if (Z) fetch_rows<Sh>(sm.raw[b][2], Z + r * p.z_ld, p.z_ld, ntok, nch);
      fetch_states(sm.C[b], Cm + r * p.c_ld, p.c_ld, ntok, p.S, p.bc_vec);
    }
  };
  if (r0 < r1) load(r0, 0);
  __syncthreads();  // bias, D
  int b = 0;
  for (long long r = r0; r < r1; r += kScanTile, b ^= 1) {
    const int ntok = (int)min((long long)kScanTile, r1 - r);
    fetched();
#pragma unroll
    for (int i = 0; i < Sh::NV; ++i) {
      const int t = Sh::tok(i), c = Sh::chan(i);
      if (t >= kScanTile) break;
      float xv[V], dl[V];
      K::get(sm.raw[b][0][i][tid], xv);
      K::get(sm.raw[b][1][i][tid], dl);
      step_sizes<V>(p, sm.bias + c, t < ntok, dl);
      store_steps<V>(sm.dx[t], c, dl, xv);
    }
    __syncthreads();
    load(r + kScanTile, b ^ 1);
    if (!FIRST && p.chunks) {
      const long long slot = w.chunk0 + (r - w.begin) / kScanTile;
#pragma unroll
      for (int j = 0; j < 2; ++j) store_pairs(p.chunks, slot, slot < p.slots, p, c0, first + 2 * (j ^ (sl & 1)), nch, n0, h[j]);
    }
    // four tokens at a time (those past the end have dl = 0 and change nothing), their
    // sums after the last: a store between them would hold up the next one's loads
    for (int t0 = 0; t0 < ntok; t0 += kGroup) {
      f2 y[kGroup][2];
#pragma unroll
      for (int u = 0; u < kGroup; ++u) {
        const int t = t0 + u;
        f2 bb[4], cc[4];
        states4(&sm.B[b][t][n0], 0, bb);
        if (!FIRST) states4(&sm.C[b][t][n0], 0, cc);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const ulonglong2 d = *reinterpret_cast<const ulonglong2 *>(&sm.dx[t][at[j]]);
          if (FIRST) sumd[j] = add2(sumd[j], d.x);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            h[j][i] = fma2(decay2(d.x, A2[j][i], shift), h[j][i], mul2(d.y, bb[i]));
            if (!FIRST) y[u][j] = i ? fma2(cc[i], h[j][i], y[u][j]) : mul2(cc[i], h[j][i]);
          }
        }
      }
      if (out) {
#pragma unroll
        for (int u = 0; u < kGroup; ++u) sum_states<L>(y[u], sm.y[t0 + u], first, sl);
      }
    }
    __syncthreads();
    if (!out) continue;
    T *O = (T *)p.out + r * p.out_ld + c0;
#pragma unroll
    for (int i = 0; i < Sh::NV; ++i) {
      const int t = Sh::tok(i), c = Sh::chan(i);
      if (t >= ntok || c >= nch) continue;
      float o[V], v[V], Dk[V];
      load_vec<V>(&sm.y[t][c], o);
      if (p.Dskip) {
        K::get(sm.raw[b][0][i][tid], v);
        load_vec<V>(sm.D + c, Dk);
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = fmaf(Dk[e], v[e], o[e]);
      }
      if (p.z) {
        K::get(sm.raw[b][2][i][tid], v);
        silu_gate<V>(v, o);
      }
      K::st(O + t * p.out_ld + c, K::put(o));
    }
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int pair = first + 2 * (j ^ (sl & 1));
    if (FIRST) {
      const size_t u = blockIdx.x;
      float s[2], v[2][4];
      unpack2(sumd[j], s[0], s[1]);
#pragma unroll
      for (int i = 0; i < 4; ++i) unpack2(h[j][i], v[0][i], v[1][i]);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        if (pair + e >= nch) continue;
        const size_t d = c0 + pair + e;
        if (sl == 0) p.sumd[u * p.D + d] = s[e];
        *reinterpret_cast<float4 *>(p.carry + (u * p.D + d) * Sh::SP + n0) =
            make_float4(v[e][0], v[e][1], v[e][2], v[e][3]);
      }
    } else if (p.hT && w.j == w.n - 1) {
      store_pairs(p.hT, w.s, true, p, c0, pair, nch, n0, h[j]);
    }
  }
}

template <typename T, int L, bool VEC>
cudaError_t fwd_l(const ScanP &p, const ScanPlan &pl, cudaStream_t s) {
  const dim3 grid(pl.units, pl.tiles);
  const int smem = (int)sizeof(FwdSmem<T, L, VEC>);
  cudaError_t e;
  if ((e = allow_smem(scan_fwd_kernel<T, L, VEC, true>, smem)) != cudaSuccess) return e;
  if ((e = allow_smem(scan_fwd_kernel<T, L, VEC, false>, smem)) != cudaSuccess) return e;
  if (pl.split)
    RDN_LAUNCH("scan_carry", s, (scan_fwd_kernel<T, L, VEC, true><<<grid, kScanThreads, smem, s>>>(p)));
  RDN_LAUNCH("scan_fwd", s, (scan_fwd_kernel<T, L, VEC, false><<<grid, kScanThreads, smem, s>>>(p)));
  return cudaGetLastError();
}
template <typename T, bool VEC>
cudaError_t fwd_v(const ScanP &p, const ScanPlan &pl, cudaStream_t s) {
  switch (pl.L) {
    case 2: return fwd_l<T, 2, VEC>(p, pl, s);
    case 4: return fwd_l<T, 4, VEC>(p, pl, s);
    case 8: return fwd_l<T, 8, VEC>(p, pl, s);
    default: return fwd_l<T, 16, VEC>(p, pl, s);
  }
}

struct StepP {
  int N, D, S, G, num_slots, softplus;
  int rows;     // requests per CTA
  bool bc_vec;  // 4 states of B and C in one access
  long long x_ld, dt_ld, z_ld, b_ld, c_ld, out_ld;
  const void *x, *dt, *z, *Bm, *Cm;
  const float *A, *Dskip, *dt_bias;
  float *h;
  const int *slots;
  void *out;
};

// One token: L = 1 .. 8 lanes per channel, 8 states each (two quads, so that the
// lanes of a channel read whole sectors); the states stream through once
// (memory-bound: 8 bytes per state).  A CTA does its channels for up to kStepRows
// requests, so that A (as many bytes as one request's states) and the channels'
// parameters are read once for all of them; a request's loads are in flight while
// the one before is worked on.  4096 channels of 16 states: one request 2.4 us in a
// captured graph, 256 requests 29 us (141 MB, 4.9 TB/s; with B and C, too, a request
// ahead the registers leave 5 CTAs per SM: 36 us).
constexpr int kStepThreads = 128, kStepRows = 32;
// 4 states of B or C from global memory (zero past S)
template <typename T>
__device__ __forceinline__ void states_of(const T *row, int S, int n0, bool vec, float (&v)[4]) {
  using K = Pack<T, 4>;
  if (vec) {
    K::get(n0 < S ? K::ld(row + n0) : K::zero(), v);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = n0 + i < S ? to_f32<T>(row[n0 + i]) : 0.f;
  }
}
template <typename T, int L>
__global__ void __launch_bounds__(kStepThreads) scan_step_kernel(StepP p) {
  constexpr int CH = kStepThreads / L;
  __shared__ int s_slot[kStepRows];
  const int sl = threadIdx.x % L, n0[2] = {sl * 4, 4 * L + sl * 4};
  const int d = blockIdx.y * CH + threadIdx.x / L;
  const int first = blockIdx.x * p.rows, count = min(p.rows, p.N - first);
  if (threadIdx.x < count) {
    const int n = first + threadIdx.x, slot = p.slots ? __ldg(p.slots + n) : n;
    s_slot[threadIdx.x] = slot < p.num_slots ? slot : -1;
  }
  const bool on = d < p.D;
  const int g = on ? d / (p.D / p.G) : 0;
  float A2[2][4] = {}, bias = 0.f, Dk = 0.f;
  if (on) {
#pragma unroll
    for (int q = 0; q < 2; ++q) load_states(p.A + (size_t)d * p.S, p.S, n0[q], A2[q]);
    if (p.dt_bias) bias = __ldg(p.dt_bias + d);
    if (p.Dskip) Dk = __ldg(p.Dskip + d);
  }
#pragma unroll
  for (int q = 0; q < 2; ++q)
#pragma unroll
    for (int i = 0; i < 4; ++i) A2[q][i] = log2_rate(A2[q][i]);
  __syncthreads();
  float hn[2][4] = {}, xn = 0.f, dn = 0.f, zn = 0.f;  // of the next request
  auto load = [&](int r) {
    const int slot = r < count ? s_slot[r] : -1;
    if (!on || slot < 0) return;
    const float *row = p.h + ((size_t)slot * p.D + d) * p.S;
    const size_t n = first + r;
#pragma unroll
    for (int q = 0; q < 2; ++q) load_states(row, p.S, n0[q], hn[q]);
    xn = to_f32<T>(((const T *)p.x)[n * p.x_ld + d]);
    dn = to_f32<T>(((const T *)p.dt)[n * p.dt_ld + d]);
    if (p.z) zn = to_f32<T>(((const T *)p.z)[n * p.z_ld + d]);
  };
  load(0);
  for (int r = 0; r < count; ++r) {
    float h[2][4];
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int i = 0; i < 4; ++i) h[q][i] = hn[q][i];
    const float x = xn, v = dn + bias, z = zn;
    load(r + 1);
    const int slot = s_slot[r];
    const size_t n = first + r;
    float y = 0.f;
    if (slot >= 0) {
      const T *Bm = (const T *)p.Bm + n * p.b_ld + (size_t)g * p.S;
      const T *Cm = (const T *)p.Cm + n * p.c_ld + (size_t)g * p.S;
      const float dl = p.softplus ? softplusf(v) : v, dx = dl * x;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        float bb[4], cc[4];
        states_of<T>(Bm, p.S, n0[q], p.bc_vec, bb);
        states_of<T>(Cm, p.S, n0[q], p.bc_vec, cc);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          h[q][i] = fmaf(decay(dl, A2[q][i]), h[q][i], dx * bb[i]);
          y = fmaf(cc[i], h[q][i], y);
        }
        if (on) store_states(p.h + ((size_t)slot * p.D + d) * p.S, p.S, n0[q], h[q]);
      }
    }
#pragma unroll
    for (int o = L / 2; o; o >>= 1) y += __shfl_xor_sync(0xffffffffu, y, o);
    if (!on || sl) continue;
    if (slot >= 0) {
      if (p.Dskip) y = fmaf(Dk, x, y);
      if (p.z) y *= siluf(z);
    }
    ((T *)p.out)[n * p.out_ld + d] = from_f32<T>(slot >= 0 ? y : 0.f);
  }
}

template <typename T, int L>
cudaError_t step_l(StepP p, cudaStream_t s) {
  constexpr int CH = kStepThreads / L;
  const unsigned tiles = (p.D + CH - 1) / CH;
  // the requests shared out over the 8 CTAs that an SM holds (4096 x 16 states: 256
  // requests in 38 us one per CTA, 31 us eight in 1.7 waves, 29 us so)
  const int groups = tiles < 152 * 8 ? 152 * 8 / tiles : 1, rows = (p.N + groups - 1) / groups;
  p.rows = rows < kStepRows ? rows : kStepRows;
  const dim3 grid((p.N + p.rows - 1) / p.rows, tiles);
  RDN_LAUNCH("scan_step", s, (scan_step_kernel<T, L><<<grid, kStepThreads, 0, s>>>(p)));
  return cudaGetLastError();
}
template <typename T>
cudaError_t step_d(const StepP &p, cudaStream_t s) {
  return p.S <= 8 ? step_l<T, 1>(p, s) : p.S <= 16 ? step_l<T, 2>(p, s) : p.S <= 32 ? step_l<T, 4>(p, s) : step_l<T, 8>(p, s);
}

}  // namespace

long long scan_slots(const rdn_scan_args &a) {
  const long long nc = ((long long)a.T + kScanTile - 1) / kScanTile;
  return a.cu_seqlens ? a.num_seqs + nc : a.B * nc;
}

// Time per token of an SM that has r CTAs of a pass to run, of which `resident`
// fit at a time: up to about half of those it is latency, the same for one as
// for several, then issue slots.  In us, measured at 4096 bf16 channels of 16 states
// over cuts of 1 to 28 units (prefill of 16384 tokens, training pass of 4 x 2048), and
// used for every type and number of states.  `resident` is that instance's too: by its
// shared memory the forward and its first pass hold 4 CTAs per SM for bf16 with up to 8
// states, 5 and 3 for fp32 with up to 16 and up to 8; the backward of up to 8 states 4, its
// first pass 7 (fp32 with up to 8 states 5).  There the cut is a guess.
struct PassTime {
  int resident;
  double least, fixed, each;
  double at(long long r) const {
    auto wave = [&](long long k) { return fmax(least, fixed + each * fmin((double)k, resident)); };
    return (r / resident) * wave(resident) + (r % resident ? wave(r % resident + 1) : 0.0);
  }
  // the same per token-CTA where units of many lengths fill each other's gaps
  double packed(double sms) const { return (fixed + each * resident) / (resident * sms); }
};
constexpr PassTime kFwdTime{8, 0.245, 0.090, 0.037}, kFirstTime{8, 0.150, 0.060, 0.027};
constexpr PassTime kBwdTime{6, 0.54, 0.25, 0.146};

// Units: the cut of the sequences that ends first by those times, with each
// unit's start (its parameters, the states of the units before it) as 8 tokens
// more and a quarter of one for each of the n units.  Packed sequences, whose
// lengths are on the device: their tokens at full occupancy, about half a unit
// more for each, and one unit's time at the end.  Units are at least 32 tokens.
ScanPlan scan_plan(const rdn_scan_args &a, bool bwd) {
  constexpr int kSMs = 152;
  const PassTime &main = bwd ? kBwdTime : kFwdTime;
  ScanPlan pl;
  pl.L = a.S <= 8 ? 2 : a.S <= 16 ? 4 : a.S <= 32 ? 8 : 16;
  pl.CT = 256 / pl.L;
  const int Dg = a.D / a.G;
  pl.tiles_g = (Dg + pl.CT - 1) / pl.CT;
  pl.tiles = pl.tiles_g * a.G;
  const long long columns = (a.cu_seqlens ? 1ll : (long long)a.B) * pl.tiles;
  const long long T16 = ((long long)a.T + kScanTile - 1) / kScanTile;  // tiles of tokens
  const long long more = a.cu_seqlens ? a.num_seqs / 2 : 0;
  auto time = [&](long long n, long long len) {
    const double tokens = (double)len * kScanTile, start = 8 + 0.25 * n;
    const double launch = n > 1 ? 2.0 : 0.0;  // of the first pass
    if (a.cu_seqlens) {
      const double share = 1.0 - 1.0 / n, units = n + more;
      return (main.packed(kSMs) + share * kFirstTime.packed(kSMs)) * columns * (a.T + units * start) +
             (main.least + (n > 1 ? kFirstTime.least : 0.0)) * (tokens + start) + launch;
    }
    const long long ctas = columns * n, first = columns * (n - 1);
    return main.at((ctas + kSMs - 1) / kSMs) * (tokens + start) +
           kFirstTime.at((first + kSMs - 1) / kSMs) * (tokens + 8) + launch;
  };
  long long best = T16 > 2 ? T16 : 2;  // tiles per unit
  double cost = time(1, best);
  for (long long n = 2; n <= 64 && T16 >= 2 * n; ++n) {
    const long long len = (T16 + n - 1) / n, m = (T16 + len - 1) / len;
    const double c = time(m, len);
    if (c < cost) { cost = c; best = len; }
  }
  pl.seg = (int)best * kScanTile;
  pl.units_row = a.T > 0 ? (a.T + pl.seg - 1) / pl.seg : 1;
  pl.units = a.cu_seqlens ? a.num_seqs + (a.T + pl.seg - 1) / pl.seg : a.B * pl.units_row;
  pl.split = a.T > pl.seg;
  return pl;
}

ScanP scan_params(const rdn_scan_args &a, const ScanPlan &pl) {
  ScanP p{};
  p.B = a.B; p.T = a.T; p.D = a.D; p.S = a.S; p.G = a.G;
  p.ns = a.cu_seqlens ? a.num_seqs : a.B;
  p.softplus = a.dt_softplus;
  p.seg = pl.seg; p.units = pl.units; p.units_row = pl.units_row; p.tiles_g = pl.tiles_g;
  const size_t esz = a.dtype == RDN_BF16 ? 2 : 4;
  p.bc_vec = a.S % (16 / esz) == 0 &&
             (((uintptr_t)a.Bm | (uintptr_t)a.Cm | (size_t)a.b_ld * esz | (size_t)a.c_ld * esz) & 15) == 0;
  p.x_ld = a.x_ld; p.dt_ld = a.dt_ld; p.z_ld = a.z_ld; p.b_ld = a.b_ld; p.c_ld = a.c_ld;
  p.out_ld = a.out_ld; p.dout_ld = a.dout_ld; p.dx_ld = a.dx_ld; p.ddt_ld = a.ddt_ld; p.dz_ld = a.dz_ld;
  p.x = a.x; p.dt = a.dt; p.z = a.z; p.Bm = a.Bm; p.Cm = a.Cm; p.dout = a.dout;
  p.A = a.A; p.Dskip = a.Dskip; p.dt_bias = a.dt_bias; p.h0 = a.h0; p.dhT = a.dhT;
  p.out = a.out; p.dx = a.dx; p.ddt = a.ddt; p.dz = a.dz;
  p.slots = scan_slots(a);
  p.hT = a.hT; p.chunks = a.h_chunks; p.dh0 = a.dh0; p.cu = a.cu_seqlens;
  return p;
}

// 16-byte accesses: every row of every operand and every channel tile on 16 bytes
bool scan_vec(const rdn_scan_args &a, bool bwd) {
  const size_t size = a.dtype == RDN_BF16 ? 2 : 4;
  if ((a.D / a.G) % (16 / size)) return false;
  auto on = [&](const void *p, long long ld) { return !p || (((uintptr_t)p | (size_t)ld * size) & 15) == 0; };
  if (!on(a.x, a.x_ld) || !on(a.dt, a.dt_ld) || !on(a.z, a.z_ld)) return false;
  if (!bwd) return on(a.out, a.out_ld);
  if (!on(a.dt_bias, 0) || !on(a.Dskip, 0)) return false;  // read once per tile
  return on(a.dout, a.dout_ld) && on(a.dx, a.dx_ld) && on(a.ddt, a.ddt_ld) && on(a.dz, a.dz_ld);
}

size_t scan_fwd_bytes(const rdn_scan_args &a) {
  const ScanPlan pl = scan_plan(a, false);
  if (!pl.split) return 0;
  return round256(sizeof(float) * (size_t)pl.units * a.D * 4 * pl.L) +
         round256(sizeof(float) * (size_t)pl.units * a.D);
}

namespace {
cudaError_t scan_run(const rdn_scan_args &a, const ScanP &p, const ScanPlan &pl, cudaStream_t s) {
  const bool vec = scan_vec(a, false);
  if (a.dtype == RDN_BF16)
    return vec ? fwd_v<__nv_bfloat16, true>(p, pl, s) : fwd_v<__nv_bfloat16, false>(p, pl, s);
  return vec ? fwd_v<float, true>(p, pl, s) : fwd_v<float, false>(p, pl, s);
}
}  // namespace

cudaError_t launch_scan_fwd(const rdn_scan_args &a, cudaStream_t s) {
  const ScanPlan pl = scan_plan(a, false);
  ScanP p = scan_params(a, pl);
  if (pl.split) {
    p.carry = static_cast<float *>(a.workspace);
    p.sumd = p.carry + round256(sizeof(float) * (size_t)pl.units * a.D * 4 * pl.L) / sizeof(float);
  }
  return scan_run(a, p, pl, s);
}

cudaError_t scan_states(const rdn_scan_args &a, ScanP p, const ScanPlan &pl, cudaStream_t s) {
  p.out = nullptr;
  p.hT = nullptr;
  return scan_run(a, p, pl, s);
}

cudaError_t launch_scan_step(const rdn_scan_step_args &a, cudaStream_t s) {
  const size_t esz = a.dtype == RDN_BF16 ? 2 : 4;
  const bool bc_vec = a.S % 4 == 0 && (((uintptr_t)a.Bm | (uintptr_t)a.Cm | (size_t)a.b_ld * esz | (size_t)a.c_ld * esz) & (4 * esz - 1)) == 0;
  const StepP p{a.N, a.D, a.S, a.G, a.num_slots, a.dt_softplus, 1, bc_vec, a.x_ld, a.dt_ld, a.z_ld, a.b_ld,
                a.c_ld, a.out_ld, a.x, a.dt, a.z, a.Bm, a.Cm, a.A, a.Dskip, a.dt_bias, a.h, a.slots, a.out};
  return a.dtype == RDN_BF16 ? step_d<__nv_bfloat16>(p, s) : step_d<float>(p, s);
}

}  // namespace rdn
