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
// channel lanes (2 channels each): 8 (channel, state) pairs per lane.  B and C
// are read once per 2 channels, and a sum over the states takes log2(L)
// exchanges, where a thread per channel would read all of B and C for each of
// its channels (twice the shared-memory reads) and sums over the channels
// (backward: dB, dC) would exchange every state.
//
// A sequence is cut into units of `seg` tokens where there are too few
// channels and sequences to fill the GPU: a first pass finds each unit's end
// state from a zero start and the sum of its dl; since A is constant in time
// the decay over a unit is exp(A sum dl), so a unit's start state is a short
// chain over the units before it (the backward likewise, from the end).
#pragma once
#include "rows.cuh"

namespace rdn {

constexpr int kScanThreads = 128, kScanWarps = 4;
constexpr int kScanTile = RDN_SCAN_CHUNK;  // tokens staged at a time, and between kept states

// exp2 of the decay's exponent.  ex2.approx comes out low by about 2e-8 on
// average for small arguments; with decays near 1 the factors of a thousand
// tokens multiply, and the mean error adds up where rounding would average
// out.  kExpShift (added in the multiply that forms the argument, at no cost)
// takes the mean below 5e-9 for exponents in [-0.5, 0]; expf has 1e-8 to
// 1.5e-8 there.
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kExpShift = 2.5e-8f;
__device__ __forceinline__ float decay(float dl, float A2) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(fmaf(dl, A2, kExpShift)));
  return y;
}

// softplus, and its derivative from its argument
__device__ __forceinline__ float softplusf(float v) { return v > 20.f ? v : log1pf(__expf(v)); }

struct ScanP {
  int B, T, D, S, G, ns;
  int softplus;
  int seg;          // tokens per unit (a multiple of kScanTile)
  int units, units_row;  // units of the call (packed: a bound); without cu: per sequence
  int tiles_g;      // channel tiles per group
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
  static constexpr int CW = 64 / L;                // channels of a warp
  static constexpr int CT = kScanWarps * CW;       // and of a CTA
  static constexpr int SP = 4 * L;                 // states, padded
  static constexpr int V = VEC ? kVec<T> : 1;      // channels per global access
  static constexpr int COLS = CT / V;              // accesses per token
  static constexpr int NV = (kScanTile * COLS + kScanThreads - 1) / kScanThreads;  // per thread
  static constexpr int NB = kScanTile * SP / kScanThreads;  // B (or C) elements per thread
};

// A thread's part of one operand's tile (kScanTile tokens x CT channels), as loaded.
template <typename T, int L, bool VEC>
struct TileRows {
  using Sh = ScanShape<T, L, VEC>;
  using K = Pack<T, Sh::V>;
  typename K::Raw raw[Sh::NV];
  // tokens [0, ntok) at base + t * ld, channels [0, nch) of the tile
  __device__ void load(const T *base, long long ld, int ntok, int nch) {
#pragma unroll
    for (int i = 0; i < Sh::NV; ++i) {
      const int id = i * kScanThreads + threadIdx.x, t = id / Sh::COLS, c = id % Sh::COLS * Sh::V;
      raw[i] = base && t < ntok && c < nch ? K::ld(base + t * ld + c) : K::zero();
    }
  }
  __device__ void get(int i, float (&v)[Sh::V]) const { K::get(raw[i], v); }
};

// A thread's part of B or C: kScanTile tokens x SP states (zero past S).
template <typename T, int L>
struct TileBC {
  static constexpr int SP = 4 * L, NB = kScanTile * SP / kScanThreads;
  T raw[NB];
  __device__ void load(const T *base, long long ld, int ntok, int S) {
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int id = i * kScanThreads + threadIdx.x, t = id / SP, n = id % SP;
      raw[i] = t < ntok && n < S ? base[t * ld + n] : from_f32<T>(0.f);
    }
  }
};

// y[t] over 4 tokens, each a lane's part of two channels' sums over the states
// (v[t][0]: the channel cl * 2 + (sl & 1), v[t][1]: the other one), summed over
// the L state lanes and written to dst[token][channel] (row pitch `pitch`).
// The order of the channels differs between the lanes that exchange, so the
// first exchange needs no selects; the next two split the tokens.
template <int L>
__device__ __forceinline__ void sum_states(float (&v)[4][2], float *dst, int pitch, int ch, int sl) {
  float r[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) r[t] = v[t][0] + __shfl_xor_sync(0xffffffffu, v[t][1], 1);
  if (L == 2) {
#pragma unroll
    for (int t = 0; t < 4; ++t) dst[t * pitch + ch] = r[t];
    return;
  }
  float r2[2];
  const bool b1 = sl & 2;
#pragma unroll
  for (int t = 0; t < 2; ++t)
    r2[t] = (b1 ? r[2 * t + 1] : r[2 * t]) + __shfl_xor_sync(0xffffffffu, b1 ? r[2 * t] : r[2 * t + 1], 2);
  if (L == 4) {
#pragma unroll
    for (int t = 0; t < 2; ++t) dst[(2 * t + (b1 ? 1 : 0)) * pitch + ch] = r2[t];
    return;
  }
  const bool b2 = sl & 4;
  float r1 = (b2 ? r2[1] : r2[0]) + __shfl_xor_sync(0xffffffffu, b2 ? r2[0] : r2[1], 4);
  if (L == 16) r1 += __shfl_xor_sync(0xffffffffu, r1, 8);
  if (L == 8 || !(sl & 8)) dst[((b2 ? 2 : 0) + (b1 ? 1 : 0)) * pitch + ch] = r1;
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

struct ScanPlan {
  int L, CT, tiles_g, tiles;
  int seg, units, units_row;
  bool split;  // some sequence may have more than one unit
};
long long scan_slots(const rdn_scan_args &a);
// The forward without out (and hT): the kept states alone, into p.chunks.
cudaError_t scan_states(const rdn_scan_args &a, ScanP p, const ScanPlan &pl, cudaStream_t s);
ScanPlan scan_plan(const rdn_scan_args &a);
ScanP scan_params(const rdn_scan_args &a, const ScanPlan &pl);
bool scan_vec(const rdn_scan_args &a, bool bwd);

}  // namespace rdn
