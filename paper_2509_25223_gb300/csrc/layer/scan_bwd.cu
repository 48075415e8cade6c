// scan_bwd.cu -- backward of the selective scan (scan.cu).  With
// gy_t = dout_t SiLU(z_t), from the last token down,
//     g_t = C_t gy_t + q_{t+1},   q_t = a_t g_t         (q past the end: dhT)
//     dC_t += gy_t h_t            dB_t += g_t dl_t x_t          (sums over channels)
//     dA += dl_t q_t h_{t-1}      (sum over tokens)
//     ddl_t = sum_n A q_t h_{t-1} + x_t sum_n g_t B_t
//     dx_t = dl_t sum_n g_t B_t + Dskip gy_t,   dz_t = dout_t y_t SiLU'(z_t)
// and dh0 = q of the first token.
//
// The states are recomputed from those kept at every 16 tokens: 4 tokens' states
// at a time stay in registers (4 x 16 pairs per lane) while the reverse steps
// consume them, from states advanced once through the tile and left in shared
// memory at every fourth token, so that three tokens of four are recomputed twice.
// Keeping 8 tokens' states in registers takes 255 of them and a loop body beyond
// the instruction cache: 744 us for 4 x 2048 x 4096 channels of 16 states where
// this takes 660 (0.81e12 (token, channel, state) per second, 1.0 TB/s of HBM
// traffic).  About 15 multiply-adds and 2.75 exponentials for each of those, 25
// instructions in all (a pair's count as half): no pipe is full -- issue slots 52 %,
// FMA 44 %, shared memory 43 %, exponentials 27 % -- and the registers leave 12
// warps per SM to fill them.  At these 6 CTAs per SM most instances spill 4 to 16
// bytes; with the registers of 7 the kernel takes 857 us.  The
// first pass (scan_bwd_carry) takes 135 us there, the joins of dB, dC 24 and of the
// parameters' gradients 14.  The sums over
// channels for dB and dC are exchanged within a warp in an order that needs no
// selects (the lanes that exchange hold their four states in orders that differ by
// the bit they exchange over), joined over the CTA's warps in shared memory, and
// over the channel tiles through the workspace, always in the same order.
#include "scan.cuh"

namespace rdn {
namespace {

constexpr int kHalf = 8;  // tokens between two joins of the warps' sums
constexpr int kSub = 4;   // tokens whose states are in registers together

template <typename T, int L, bool VEC>
struct CarrySmem {
  using Sh = ScanShape<T, L, VEC>;
  float4 dg[kScanTile][Sh::CT / 2];                  // (dl, dl', gy, gy') of a pair, at spread16
  typename Sh::Raw raw[3][Sh::NV][kScanThreads];     // each thread's dt, z, dout of the next tile
  T C[2][kScanTile][Sh::SP];
  float bias[Sh::CT];
};

// The first pass: each unit's q at its first token from q = 0 past its end,
// and the sum of its dl (units but the first of a sequence).
template <typename T, int L, bool VEC>
__global__ void __launch_bounds__(kScanThreads, 7) scan_bwd_carry_kernel(ScanP p) {
  using Sh = ScanShape<T, L, VEC>;
  using K = typename Sh::K;
  constexpr int V = Sh::V;
  extern __shared__ __align__(16) unsigned char smem_raw[];
  CarrySmem<T, L, VEC> &sm = *reinterpret_cast<CarrySmem<T, L, VEC> *>(smem_raw);
  const Unit w = find_unit(p, blockIdx.x);
  if (!w.ok || w.j == 0) return;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int sl = lane % L, cl = lane / L, n0 = sl * 4;
  const int g = blockIdx.y / p.tiles_g, Dg = p.D / p.G;
  const int c0 = g * Dg + blockIdx.y % p.tiles_g * Sh::CT;
  const int nch = min(Sh::CT, (g + 1) * Dg - c0);
  const int first = warp * Sh::CW + cl * 4;
  const int at[2] = {spread16(first / 2), spread16(first / 2 + 1)};
  for (int c = tid; c < Sh::CT; c += kScanThreads) sm.bias[c] = p.dt_bias && c < nch ? p.dt_bias[c0 + c] : 0.f;
  f2 A2[2][4], q[2][4], sumd[2];
  const f2 shift = pack2(kExpShift, kExpShift), zero2 = pack2(0.f, 0.f);
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    float a[2][4];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int i = 0; i < 4; ++i) a[e][i] = 0.f;
      if (first + 2 * j + e < nch) load_states(p.A + (size_t)(c0 + first + 2 * j + e) * p.S, p.S, n0, a[e]);
    }
    sumd[j] = zero2;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      A2[j][i] = pack2(log2_rate(a[0][i]), log2_rate(a[1][i]));
      q[j][i] = zero2;
    }
  }
  const long long r0 = w.begin + (long long)w.j * p.seg;
  const long long r1 = min(r0 + p.seg, w.end);
  const long long last = r0 + (r1 - 1 - r0) / kScanTile * kScanTile;
  const T *Cm = (const T *)p.Cm + (size_t)g * p.S;
  auto load = [&](long long r, int b) {
    const int ntok = r < r0 ? 0 : (int)min((long long)kScanTile, r1 - r);
    fetch_rows<Sh>(sm.raw[0], (const T *)p.dt + c0 + r * p.dt_ld, p.dt_ld, ntok, nch);
    if (p.z) fetch_rows<Sh>(sm.raw[1], (const T *)p.z + c0 + r * p.z_ld, p.z_ld, ntok, nch);
    fetch_rows<Sh>(sm.raw[2], (const T *)p.dout + c0 + r * p.dout_ld, p.dout_ld, ntok, nch);
    fetch_states(sm.C[b], Cm + r * p.c_ld, p.c_ld, ntok, p.S, p.bc_vec);
  };
  load(last, 0);
  __syncthreads();  // bias
  int b = 0;
  for (long long r = last; r >= r0; r -= kScanTile, b ^= 1) {
    const int ntok = (int)min((long long)kScanTile, r1 - r);
    fetched();
#pragma unroll
    for (int i = 0; i < Sh::NV; ++i) {
      const int t = Sh::tok(i), c = Sh::chan(i);
      if (t >= kScanTile) break;
      float dl[V], gv[V], zv[V];
      K::get(sm.raw[0][i][tid], dl);
      K::get(sm.raw[2][i][tid], gv);
      step_sizes<V>(p, sm.bias + c, t < ntok, dl);
      if (p.z) {
        K::get(sm.raw[1][i][tid], zv);
        silu_gate<V>(zv, gv);
      }
      store_two<V>(sm.dg[t], c, dl, gv);
    }
    __syncthreads();
    load(r - kScanTile, b ^ 1);
#pragma unroll 4
    for (int t = ntok - 1; t >= 0; --t) {
      f2 cc[4];
      states4(&sm.C[b][t][n0], 0, cc);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const ulonglong2 d = *reinterpret_cast<const ulonglong2 *>(&sm.dg[t][at[j]]);
        sumd[j] = add2(sumd[j], d.x);
#pragma unroll
        for (int i = 0; i < 4; ++i) q[j][i] = mul2(decay2(d.x, A2[j][i], shift), fma2(cc[i], d.y, q[j][i]));
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const size_t u = blockIdx.x;
    float s[2], v[2][4];
    unpack2(sumd[j], s[0], s[1]);
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2(q[j][i], v[0][i], v[1][i]);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      if (first + 2 * j + e >= nch) continue;
      const size_t d = c0 + first + 2 * j + e;
      if (sl == 0) p.sumd[u * p.D + d] = s[e];
      *reinterpret_cast<float4 *>(p.carry + (u * p.D + d) * Sh::SP + n0) = make_float4(v[e][0], v[e][1], v[e][2], v[e][3]);
    }
  }
}

// The sums over a warp's channel lanes of db[i] and dc[i] (i-th state in this
// lane's order, i ^ (cl & 3)), written to red[0 .. 4 L) (dB) and red[4 L .. 8 L) (dC).
template <int L>
__device__ __forceinline__ void sum_channels(const float (&db)[4], const float (&dc)[4], int sl, int cl,
                                             float *red) {
  constexpr unsigned all = 0xffffffffu;
  // over bit 0: the partner's value i + 1 is this lane's state i
  float b0 = db[0] + __shfl_xor_sync(all, db[1], L), b1 = db[2] + __shfl_xor_sync(all, db[3], L);
  float g0 = dc[0] + __shfl_xor_sync(all, dc[1], L), g1 = dc[2] + __shfl_xor_sync(all, dc[3], L);
  if (L == 16) {  // two channel lanes: states (cl & 1) and 2 + (cl & 1)
    float *r = red + sl * 4 + (cl & 1);
    r[0] = b0;
    r[2] = b1;
    r[4 * L] = g0;
    r[4 * L + 2] = g1;
    return;
  }
  float b = b0 + __shfl_xor_sync(all, b1, 2 * L), c = g0 + __shfl_xor_sync(all, g1, 2 * L);
  float *r = red + sl * 4 + (cl & 3);
  if (L == 8) {
    r[0] = b;
    r[4 * L] = c;
    return;
  }
  const bool hi = cl & 4;
  float v = (hi ? c : b) + __shfl_xor_sync(all, hi ? b : c, 4 * L);
  if (L == 2) v += __shfl_xor_sync(all, v, 8 * L);
  if (L == 4 || !(cl & 8)) r[hi ? 4 * L : 0] = v;
}

template <typename T, int L, bool VEC>
struct BwdSmem {
  using Sh = ScanShape<T, L, VEC>;
  float4 dx[kScanTile][Sh::CT / 2];                  // (dl, dl', dl x, dl' x') of a pair, at spread16
  float2 gy[kScanTile][Sh::CT / 2];
  float sums[3][kHalf][Sh::CT];                      // sum_n g B, sum_n A2 q h, y
  float red[kScanWarps][kHalf][2 * Sh::SP];          // dB, dC of each warp's channels
  static constexpr int AC = Sh::COLS > kScanThreads ? Sh::COLS / kScanThreads : 1;  // columns of a thread
  float acc[2][AC][kScanThreads][Sh::V];             // dD and ddt_bias of a thread's elements
  float4 kept[3][4][kScanThreads];                   // each lane's states before tokens 0, 4 and 8 of the tile
  T B[kScanTile][Sh::SP], C[kScanTile][Sh::SP];
};

// (6 CTAs per SM by registers; of the wide tiles of L = 2 shared memory holds 4)
template <typename T, int L, bool VEC>
__global__ void __launch_bounds__(kScanThreads, L == 2 ? 4 : 6) scan_bwd_kernel(ScanP p) {
  using Sh = ScanShape<T, L, VEC>;
  using K = typename Sh::K;
  constexpr int V = Sh::V;
  extern __shared__ __align__(16) unsigned char smem_raw[];
  using Sm = BwdSmem<T, L, VEC>;
  Sm &sm = *reinterpret_cast<Sm *>(smem_raw);
  const Unit w = find_unit(p, blockIdx.x);
  const size_t u = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int sl = lane % L, cl = lane / L, n0 = sl * 4, perm = cl & (Sh::CL < 4 ? Sh::CL - 1 : 3);
  const int g = blockIdx.y / p.tiles_g, Dg = p.D / p.G;
  const int c0 = g * Dg + blockIdx.y % p.tiles_g * Sh::CT;
  const int nch = min(Sh::CT, (g + 1) * Dg - c0);
  const int first = warp * Sh::CW + cl * 4;
  int pair[2], at[2];  // this lane's channel pairs in the tile (opposite orders in the lanes that exchange)
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    pair[j] = first / 2 + (j ^ (sl & 1));
    at[j] = spread16(pair[j]);
  }
#pragma unroll
  for (int e = 0; e < Sm::AC * V; ++e) sm.acc[0][e / V][tid][e % V] = sm.acc[1][e / V][tid][e % V] = 0.f;
  const f2 shift = pack2(kExpShift, kExpShift), zero2 = pack2(0.f, 0.f);
  f2 A2[2][4], q[2][4], dA[2][4];  // [channel pair][state n0 + (i ^ perm)]
  {
    float a[4][4], v[4][4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int ch = 2 * pair[c >> 1] + (c & 1);
      const bool on = ch < nch;
      const size_t d = c0 + ch;
#pragma unroll
      for (int i = 0; i < 4; ++i) a[c][i] = v[c][i] = 0.f;
      if (on) load_states(p.A + d * p.S, p.S, n0, a[c]);
      if (on && w.ok && p.dhT) load_states(p.dhT + ((size_t)w.s * p.D + d) * p.S, p.S, n0, v[c]);
#pragma unroll
      for (int i = 0; i < 4; ++i) a[c][i] = log2_rate(a[c][i]);
    }
    // q past the unit's end, over the units after it
    if (w.ok) chain<Sh::SP>(p, (int)u - w.j + w.n - 1, (int)u, -1, c0 + first, nch - first, sl, a, v);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float x[2][4], y[2][4];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        permute(a[2 * j + e], perm, x[e]);
        permute(v[2 * j + e], perm, y[e]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        A2[j][i] = pack2(x[0][i], x[1][i]);
        q[j][i] = pack2(y[0][i], y[1][i]);
        dA[j][i] = zero2;
      }
    }
  }
  const long long r0 = w.ok ? w.begin + (long long)w.j * p.seg : 0;
  const long long r1 = w.ok ? min(r0 + p.seg, w.end) : 0;
  const long long last = r1 > r0 ? r0 + (r1 - 1 - r0) / kScanTile * kScanTile : r0 - kScanTile;
  const T *X = (const T *)p.x + c0, *DT = (const T *)p.dt + c0, *DO = (const T *)p.dout + c0;
  const T *Bm = (const T *)p.Bm + (size_t)g * p.S, *Cm = (const T *)p.Cm + (size_t)g * p.S;
  // the rows of the tile at r into L2 now, into shared memory when it is begun
  auto ahead = [&](long long r) {
    const int ntok = r < r0 ? 0 : (int)min((long long)kScanTile, r1 - r);
#pragma unroll
    for (int i = 0; i < Sh::NV; ++i) {
      const int t = Sh::tok(i), c = Sh::chan(i);
      if (t >= ntok || c >= nch) continue;
      prefetch(X + (r + t) * p.x_ld + c);
      prefetch(DT + (r + t) * p.dt_ld + c);
      prefetch(DO + (r + t) * p.dout_ld + c);
      if (p.z) prefetch((const T *)p.z + c0 + (r + t) * p.z_ld + c);
    }
    constexpr int sector = 32 / (int)sizeof(T);
    if (tid % kScanTile < ntok) {
      const T *row = tid / kScanTile % 2 ? Cm + (r + tid % kScanTile) * p.c_ld : Bm + (r + tid % kScanTile) * p.b_ld;
      for (int n = tid / (2 * kScanTile) * sector; n < p.S; n += kScanThreads / (2 * kScanTile) * sector) prefetch(row + n);
    }
  };
  // the kept states before the tile at r: read by this lane alone
  auto load_kept = [&](long long r) {
    const long long slot = w.chunk0 + (r - w.begin) / kScanTile;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int ch = 2 * pair[k >> 1] + (k & 1);
      const bool on = r >= r0 && ch < nch && slot < p.slots;
      const float *row = p.chunks + ((size_t)slot * p.D + c0 + ch) * p.S;
      if (p.S % 4 == 0) {
        fetch(&sm.kept[0][k][tid], on && n0 < p.S ? row + n0 : nullptr);
      } else {
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        if (on) load_states(row, p.S, n0, v);
        sm.kept[0][k][tid] = make_float4(v[0], v[1], v[2], v[3]);
      }
    }
  };
  if (last >= r0) load_kept(last);
  for (long long r = last; r >= r0; r -= kScanTile) {
    const int ntok = (int)min((long long)kScanTile, r1 - r);
    // the tile's operands into shared memory
    fetch_states(sm.B, Bm + r * p.b_ld, p.b_ld, ntok, p.S, p.bc_vec);
    fetch_states(sm.C, Cm + r * p.c_ld, p.c_ld, ntok, p.S, p.bc_vec);
    typename Sh::Raw raw[4][Sh::NV];
#pragma unroll
    for (int i = 0; i < Sh::NV; ++i) {
      const int t = Sh::tok(i), c = Sh::chan(i);
      const bool on = t < ntok && c < nch;
      raw[0][i] = on ? K::ld(X + (r + t) * p.x_ld + c) : K::zero();
      raw[1][i] = on ? K::ld(DT + (r + t) * p.dt_ld + c) : K::zero();
      raw[2][i] = on && p.z ? K::ld((const T *)p.z + c0 + (r + t) * p.z_ld + c) : K::zero();
      raw[3][i] = on ? K::ld(DO + (r + t) * p.dout_ld + c) : K::zero();
    }
#pragma unroll
    for (int i = 0; i < Sh::NV; ++i) {
      const int t = Sh::tok(i), c = Sh::chan(i);
      if (t >= kScanTile) break;
      float xv[V], dl[V], gv[V], zv[V];
      K::get(raw[0][i], xv);
      K::get(raw[1][i], dl);
      K::get(raw[3][i], gv);
      param<V>(p.dt_bias, c0 + c, c < nch, zv);
      step_sizes<V>(p, zv, t < ntok, dl);
      if (p.z) {
        K::get(raw[2][i], zv);
        silu_gate<V>(zv, gv);
      }
      store_steps<V>(sm.dx[t], c, dl, xv);
      store_vec<V>(&sm.gy[t][0].x + c, gv);
    }
    fetched();
    __syncthreads();
    ahead(r - kScanTile);
    auto step = [&](int t, const f2 (&from)[2][4], f2 (&to)[2][4]) {
      f2 bb[4];
      states4(&sm.B[t][n0], perm, bb);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const ulonglong2 d = *reinterpret_cast<const ulonglong2 *>(&sm.dx[t][at[j]]);
#pragma unroll
        for (int i = 0; i < 4; ++i) to[j][i] = fma2(decay2(d.x, A2[j][i], shift), from[j][i], mul2(d.y, bb[i]));
      }
    };
    auto states = [&](int k, f2 (&h)[2][4]) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float v[2][4];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float4 a = sm.kept[k][2 * j + e][tid];
          const float x[4] = {a.x, a.y, a.z, a.w};
          permute(x, perm, v[e]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) h[j][i] = pack2(v[0][i], v[1][i]);
      }
    };
    // the states before the tile's last quarter, those before the others kept on the way
    f2 h0[2][4];
    states(0, h0);
    const int quarter = (ntok - 1) / kSub;
#pragma unroll 1
    for (int k = 0; k < quarter; ++k) {
#pragma unroll 2
      for (int t = 0; t < kSub; ++t) step(k * kSub + t, h0, h0);
      if (k == 2) break;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float x[2][4], v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) unpack2(h0[j][i], x[0][i], x[1][i]);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          permute(x[e], perm, v);
          sm.kept[k + 1][2 * j + e][tid] = make_float4(v[0], v[1], v[2], v[3]);
        }
      }
    }
#pragma unroll 1
    for (int half = ntok > kHalf ? 1 : 0; half >= 0; --half) {
      const int th = half * kHalf, nh = min(ntok - th, kHalf);  // tokens [th, th + nh) of the tile
#pragma unroll 1
      for (int sub = nh > kSub ? 1 : 0; sub >= 0; --sub) {
        const int ts = th + sub * kSub;
        f2 hist[kSub][2][4];
        if (ts < quarter * kSub) states(ts / kSub, h0);
        if (ts == 0) load_kept(r - kScanTile);
#pragma unroll
        for (int t = 0; t < kSub; ++t) step(ts + t, t ? hist[t - 1] : h0, hist[t]);
#pragma unroll
        for (int tl = kSub - 1; tl >= 0; --tl) {
          const int t = ts + tl, tr = t - th;
          f2 bb[4], cc[4], db[4], dc[4], gB[2], Aq[2], y[2];
          states4(&sm.B[t][n0], perm, bb);
          states4(&sm.C[t][n0], perm, cc);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const ulonglong2 d = *reinterpret_cast<const ulonglong2 *>(&sm.dx[t][at[j]]);
            const f2 gy = *reinterpret_cast<const f2 *>(&sm.gy[t][pair[j]]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const f2 h = hist[tl][j][i], hp = tl ? hist[tl > 0 ? tl - 1 : 0][j][i] : h0[j][i];
              const f2 gr = fma2(cc[i], gy, q[j][i]);
              y[j] = i ? fma2(cc[i], h, y[j]) : mul2(cc[i], h);
              gB[j] = i ? fma2(gr, bb[i], gB[j]) : mul2(gr, bb[i]);
              dc[i] = j ? fma2(gy, h, dc[i]) : mul2(gy, h);
              db[i] = j ? fma2(gr, d.y, db[i]) : mul2(gr, d.y);
              q[j][i] = mul2(decay2(d.x, A2[j][i], shift), gr);
              const f2 qh = mul2(q[j][i], hp);
              dA[j][i] = fma2(d.x, qh, dA[j][i]);
              Aq[j] = i ? fma2(A2[j][i], qh, Aq[j]) : mul2(A2[j][i], qh);
            }
          }
          float dbv[4], dcv[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            dbv[i] = sum2(db[i]);
            dcv[i] = sum2(dc[i]);
          }
          sum_channels<L>(dbv, dcv, sl, cl, &sm.red[warp][tr][0]);
          sum_states<L>(gB, sm.sums[0][tr], first, sl);
          sum_states<L>(Aq, sm.sums[1][tr], first, sl);
          if (p.z) sum_states<L>(y, sm.sums[2][tr], first, sl);
        }
      }
      // results of the half's elements; its operands once more, from the caches
      constexpr int NH = (Sh::NV + 1) / 2, P = (V + 1) / 2;
      typename Sh::Raw own[4][NH];
#pragma unroll
      for (int i = 0; i < NH; ++i) {
        const int t = Sh::tok(i), c = Sh::chan(i);
        const bool on = t < nh && c < nch;
        const long long row = r + th + t;
        own[0][i] = on ? K::ld(X + row * p.x_ld + c) : K::zero();
        own[1][i] = on ? K::ld(DT + row * p.dt_ld + c) : K::zero();
        own[2][i] = on && p.z ? K::ld((const T *)p.z + c0 + row * p.z_ld + c) : K::zero();
        own[3][i] = on && p.z ? K::ld(DO + row * p.dout_ld + c) : K::zero();
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < NH; ++i) {
        const int t = Sh::tok(i), c = Sh::chan(i);
        if (t >= nh || c >= nch) continue;
        const long long row = r + th + t;
        float f[V];  // of one operand or result
        f2 xv[P], v[P], gy[P], gB[P], Aq[P], Dk[P], o[P];
        K::get(own[0][i], f);
        to_pairs<V>(f, xv);
        K::get(own[1][i], f);
        to_pairs<V>(f, v);
        get_pairs<V>(&sm.gy[th + t][0].x + c, gy);
        get_pairs<V>(&sm.sums[0][t][c], gB);
        get_pairs<V>(&sm.sums[1][t][c], Aq);
        param<V>(p.Dskip, c0 + c, true, f);
        to_pairs<V>(f, Dk);
#pragma unroll
        for (int e = 0; e < P; ++e) {
          const float4 *d = &sm.dx[th + t][spread16(c / 2 + e)];
          const f2 dl = V > 1 ? *reinterpret_cast<const f2 *>(d) : pack2((&d->x)[c & 1], 0.f);
          o[e] = mul2(dl, gB[e]);
          Aq[e] = fma2(Aq[e], pack2(kLn2, kLn2), mul2(gB[e], xv[e]));
        }
        if (p.Dskip) {
#pragma unroll
          for (int e = 0; e < P; ++e) o[e] = fma2(Dk[e], gy[e], o[e]);
        }
        if (p.softplus) {
          f2 bias[P];
          param<V>(p.dt_bias, c0 + c, true, f);
          to_pairs<V>(f, bias);
#pragma unroll
          for (int e = 0; e < P; ++e) Aq[e] = mul2(Aq[e], sigmoid2(add2(v[e], bias[e])));
        }
        from_pairs<V>(o, f);
        K::st((T *)p.dx + c0 + row * p.dx_ld + c, K::put(f));
        from_pairs<V>(Aq, f);
        K::st((T *)p.ddt + c0 + row * p.ddt_ld + c, K::put(f));
        float *aD = sm.acc[0][i % Sm::AC][tid], *ab = sm.acc[1][i % Sm::AC][tid];
        get_pairs<V>(aD, o);
        get_pairs<V>(ab, v);
#pragma unroll
        for (int e = 0; e < P; ++e) {
          o[e] = fma2(gy[e], xv[e], o[e]);
          v[e] = add2(v[e], Aq[e]);
        }
        put_pairs<V>(aD, o);
        put_pairs<V>(ab, v);
        if (p.z) {
          K::get(own[2][i], f);
          to_pairs<V>(f, v);
          K::get(own[3][i], f);
          to_pairs<V>(f, gy);
          get_pairs<V>(&sm.sums[2][t][c], o);
          if (p.Dskip) {
#pragma unroll
            for (int e = 0; e < P; ++e) o[e] = fma2(Dk[e], xv[e], o[e]);
          }
#pragma unroll
          for (int e = 0; e < P; ++e) o[e] = mul2(mul2(gy[e], o[e]), silu_grad2(v[e]));
          from_pairs<V>(o, f);
          K::st((T *)p.dz + c0 + row * p.dz_ld + c, K::put(f));
        }
      }
      for (int i = tid; i < nh * 2 * Sh::SP; i += kScanThreads) {
        const int t = i / (2 * Sh::SP), n = i % (2 * Sh::SP);
        float a = sm.red[0][t][n];
#pragma unroll
        for (int k = 1; k < kScanWarps; ++k) a += sm.red[k][t][n];
        p.part_bc[((size_t)blockIdx.y * p.B * p.T + r + th + t) * (2 * Sh::SP) + n] = a;
      }
      __syncthreads();
    }
  }
  // parameter gradients of the unit (zero where it has no tokens), dh0
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    float x[2][4], v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2(dA[j][i], x[0][i], x[1][i]);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      permute(x[e], perm, v);  // (its own inverse)
      if (2 * pair[j] + e < nch) store_states(p.part_A + (u * p.D + c0 + 2 * pair[j] + e) * p.S, p.S, n0, v);
    }
    if (!p.dh0 || !w.ok || w.j) continue;
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2(q[j][i], x[0][i], x[1][i]);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      permute(x[e], perm, v);
      if (2 * pair[j] + e < nch) store_states(p.dh0 + ((size_t)w.s * p.D + c0 + 2 * pair[j] + e) * p.S, p.S, n0, v);
    }
  }
  __syncthreads();
  for (int i = tid; i < 2 * Sh::CT; i += kScanThreads) {
    const int which = i / Sh::CT, c = i % Sh::CT, col = c / V;
    if (c >= nch) continue;
    float a = 0.f;  // the threads whose accesses are of column col
    for (int k = col % kScanThreads; k < kScanThreads; k += Sh::COLS)
      a += sm.acc[which][col / kScanThreads][k][c % V];
    p.part_D[(u * 2 + which) * p.D + c0 + c] = a;
  }
}

// dB and dC [B, T, G, S] from the channel tiles' partials, in order.
template <typename T>
__global__ void __launch_bounds__(256) scan_bc_kernel(const float *__restrict__ part, long long M, int G, int S,
                                                      int SP, int tiles_g, T *__restrict__ dB, T *__restrict__ dC) {
  const long long n = M * G * 2 * SP;
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (long long)gridDim.x * blockDim.x) {
    const int k = (int)(i % (2 * SP)), s = k % SP;
    const long long row = i / (2 * SP) % M;
    const int g = (int)(i / (2 * SP) / M);
    if (s >= S) continue;
    float a = 0.f;
#pragma unroll 4
    for (int t = 0; t < tiles_g; ++t) a += part[((size_t)(g * tiles_g + t) * M + row) * (2 * SP) + k];
    (k < SP ? dB : dC)[((size_t)row * G + g) * S + s] = from_f32<T>(a);
  }
}

// dA [D, S] from part_A and dD, ddt_bias [D] from part_D: columns of one sum
// over the units, 16 interleaved sums joined in order.
__global__ void __launch_bounds__(512) scan_grad_kernel(ScanP p, int units, float *dA, float *dD, float *dbias) {
  __shared__ float sh[16][32];
  const long long nA = (long long)p.D * p.S, i = (long long)blockIdx.x * 32 + threadIdx.x;
  const bool isA = i < nA;
  const long long k = isA ? i : i - nA, n = isA ? nA : 2ll * p.D;
  const float *part = isA ? p.part_A : p.part_D;
  float a = 0.f;
  if (k < n)
    for (int u = threadIdx.y; u < units; u += 16) a += part[(size_t)u * n + k];
  sh[threadIdx.y][threadIdx.x] = a;
  __syncthreads();
  if (threadIdx.y || k >= n) return;
#pragma unroll
  for (int y = 1; y < 16; ++y) a += sh[y][threadIdx.x];
  if (isA) dA[k] = a;
  else if (k < p.D) {
    if (dD) dD[k] = a;
  } else if (dbias) {
    dbias[k - p.D] = a;
  }
}

struct BwdWs {
  size_t carry, sumd, bc, A, D, states, total;  // byte offsets
};
BwdWs bwd_ws(const rdn_scan_args &a, const ScanPlan &pl, const ScanPlan &fwd) {
  BwdWs w{};
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t o = at;
    at += round256(n * sizeof(float));
    return o;
  };
  const size_t SP = 4 * pl.L, units = pl.units, M = (size_t)a.B * a.T;
  // (shared with the forward that computes the kept states, where none are given)
  size_t first = pl.split ? pl.units : 0;
  if (!a.h_chunks && fwd.split && (size_t)fwd.units > first) first = fwd.units;
  w.carry = take(first * a.D * SP);
  w.sumd = take(first * a.D);
  w.bc = take((size_t)pl.tiles * M * 2 * SP);
  w.A = take(units * a.D * a.S);
  w.D = take(units * 2 * a.D);
  w.states = take(a.h_chunks ? 0 : (size_t)scan_slots(a) * a.D * a.S);
  w.total = at;
  return w;
}

template <typename T, int L, bool VEC>
cudaError_t bwd_l(const ScanP &p, const ScanPlan &pl, cudaStream_t s) {
  const dim3 grid(pl.units, pl.tiles);
  const int first = (int)sizeof(CarrySmem<T, L, VEC>), smem = (int)sizeof(BwdSmem<T, L, VEC>);
  cudaError_t e;
  if ((e = allow_smem(scan_bwd_carry_kernel<T, L, VEC>, first)) != cudaSuccess) return e;
  if ((e = allow_smem(scan_bwd_kernel<T, L, VEC>, smem)) != cudaSuccess) return e;
  if (pl.split)
    RDN_LAUNCH("scan_bwd_carry", s, (scan_bwd_carry_kernel<T, L, VEC><<<grid, kScanThreads, first, s>>>(p)));
  RDN_LAUNCH("scan_bwd", s, (scan_bwd_kernel<T, L, VEC><<<grid, kScanThreads, smem, s>>>(p)));
  return cudaGetLastError();
}
template <typename T, bool VEC>
cudaError_t bwd_v(const ScanP &p, const ScanPlan &pl, cudaStream_t s) {
  switch (pl.L) {
    case 2: return bwd_l<T, 2, VEC>(p, pl, s);
    case 4: return bwd_l<T, 4, VEC>(p, pl, s);
    case 8: return bwd_l<T, 8, VEC>(p, pl, s);
    default: return bwd_l<T, 16, VEC>(p, pl, s);
  }
}
template <typename T>
cudaError_t bwd_t(const rdn_scan_args &a, const ScanP &p, const ScanPlan &pl, cudaStream_t s) {
  cudaError_t e = scan_vec(a, true) ? bwd_v<T, true>(p, pl, s) : bwd_v<T, false>(p, pl, s);
  if (e != cudaSuccess) return e;
  const long long M = (long long)a.B * a.T;
  const int SP = 4 * pl.L;
  if (M > 0) {
    const long long n = M * a.G * 2 * SP, want = (n + 255) / 256;
    const unsigned grid = (unsigned)(want < 65536 ? want : 65536);
    RDN_LAUNCH("scan_bc", s, (scan_bc_kernel<T><<<grid, 256, 0, s>>>(p.part_bc, M, a.G, a.S, SP, pl.tiles_g,
                                                                     (T *)a.dB, (T *)a.dC)));
  }
  const unsigned grid = (unsigned)(((long long)a.D * (a.S + 2) + 31) / 32 + 1);
  RDN_LAUNCH("scan_grad", s,
             (scan_grad_kernel<<<grid, dim3(32, 16), 0, s>>>(p, pl.units, a.dA, a.dD, a.ddt_bias)));
  return cudaGetLastError();
}

}  // namespace

size_t scan_bwd_bytes(const rdn_scan_args &a) { return bwd_ws(a, scan_plan(a, true), scan_plan(a, false)).total; }

cudaError_t launch_scan_bwd(const rdn_scan_args &a, cudaStream_t s) {
  const ScanPlan pl = scan_plan(a, true), fwd = scan_plan(a, false);
  const BwdWs ws = bwd_ws(a, pl, fwd);
  ScanP p = scan_params(a, pl);
  char *base = static_cast<char *>(a.workspace);
  p.carry = reinterpret_cast<float *>(base + ws.carry);
  p.sumd = reinterpret_cast<float *>(base + ws.sumd);
  p.part_bc = reinterpret_cast<float *>(base + ws.bc);
  p.part_A = reinterpret_cast<float *>(base + ws.A);
  p.part_D = reinterpret_cast<float *>(base + ws.D);
  cudaError_t e;
  if (!a.h_chunks) {  // (the forward's own unit results go where the backward's will)
    p.chunks = reinterpret_cast<float *>(base + ws.states);
    ScanP f = scan_params(a, fwd);
    f.chunks = p.chunks;
    f.carry = p.carry;
    f.sumd = p.sumd;
    if ((e = scan_states(a, f, fwd, s)) != cudaSuccess) return e;
  }
  return a.dtype == RDN_BF16 ? bwd_t<__nv_bfloat16>(a, p, pl, s) : bwd_t<float>(a, p, pl, s);
}

}  // namespace rdn
