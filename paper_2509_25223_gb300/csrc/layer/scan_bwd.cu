// scan_bwd.cu -- backward of the selective scan (scan.cu).  With
// gy_t = dout_t SiLU(z_t), from the last token down,
//     g_t = C_t gy_t + q_{t+1},   q_t = a_t g_t         (q past the end: dhT)
//     dC_t += gy_t h_t            dB_t += g_t dl_t x_t          (sums over channels)
//     dA += dl_t q_t h_{t-1}      (sum over tokens)
//     ddl_t = sum_n A q_t h_{t-1} + x_t sum_n g_t B_t
//     dx_t = dl_t sum_n g_t B_t + Dskip gy_t,   dz_t = dout_t y_t SiLU'(z_t)
// and dh0 = q of the first token.
//
// The states are recomputed from those kept at every 16 tokens: 8 steps at a
// time stay in registers (8 steps x 8 pairs per lane) while the reverse steps
// consume them; the later 8 of a tile need the earlier 8 advanced once more.
// About 15 multiply-adds and 2.5 exponentials per (token, channel, state):
// FMA-bound.  The sums over channels for dB and dC are exchanged within a warp
// in an order that needs no selects (the lanes that exchange hold their four
// states in orders that differ by the bit they exchange over), joined over the
// CTA's warps in shared memory, and over the channel tiles through the
// workspace, always in the same order.
#include "scan.cuh"

namespace rdn {
namespace {

constexpr int kSub = 8;  // tokens whose states are in registers together

// The first pass: each unit's q at its first token from q = 0 past its end,
// and the sum of its dl (units but the first of a sequence).
template <typename T, int L, bool VEC>
__global__ void __launch_bounds__(kScanThreads) scan_bwd_carry_kernel(ScanP p) {
  using Sh = ScanShape<T, L, VEC>;
  using Rows = TileRows<T, L, VEC>;
  __shared__ __align__(16) float2 s_dg[kScanTile][Sh::CT];  // (dl, gy)
  __shared__ __align__(16) float s_C[kScanTile][Sh::SP];
  const Unit w = find_unit(p, blockIdx.x);
  if (!w.ok || w.j == 0) return;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int sl = lane % L, cl = lane / L, n0 = sl * 4;
  const int g = blockIdx.y / p.tiles_g, Dg = p.D / p.G;
  const int c0 = g * Dg + blockIdx.y % p.tiles_g * Sh::CT;
  const int nch = min(Sh::CT, (g + 1) * Dg - c0);
  float A2[2][4], q[2][4], sumd[2] = {0.f, 0.f};
  const int ch0 = warp * Sh::CW + cl * 2;
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      q[j][i] = 0.f;
      A2[j][i] = ch0 + j < nch && n0 + i < p.S ? __ldg(p.A + (size_t)(c0 + ch0 + j) * p.S + n0 + i) * kLog2e : 0.f;
    }
  const long long r0 = w.begin + (long long)w.j * p.seg;
  const long long r1 = min(r0 + p.seg, w.end);
  const T *DT = (const T *)p.dt + c0, *DO = (const T *)p.dout + c0;
  const T *Z = p.z ? (const T *)p.z + c0 : nullptr;
  const T *Cm = (const T *)p.Cm + (size_t)g * p.S;
  Rows dt, z, dout;
  TileBC<T, L> tc;
  auto load = [&](long long r) {
    const int ntok = r < r0 ? 0 : (int)min((long long)kScanTile, r1 - r);
    dt.load(DT + r * p.dt_ld, p.dt_ld, ntok, nch);
    dout.load(DO + r * p.dout_ld, p.dout_ld, ntok, nch);
    z.load(Z ? Z + r * p.z_ld : nullptr, p.z_ld, ntok, nch);
    tc.load(Cm + r * p.c_ld, p.c_ld, ntok, p.S);
  };
  const long long last = r0 + (r1 - 1 - r0) / kScanTile * kScanTile;
  load(last);
  for (long long r = last; r >= r0; r -= kScanTile) {
    const int ntok = (int)min((long long)kScanTile, r1 - r);
#pragma unroll
    for (int i = 0; i < Sh::NV; ++i) {
      const int id = i * kScanThreads + tid, t = id / Sh::COLS, c = id % Sh::COLS * Sh::V;
      if (t >= kScanTile) break;
      float dv[Sh::V], zv[Sh::V], gv[Sh::V];
      dt.get(i, dv);
      z.get(i, zv);
      dout.get(i, gv);
#pragma unroll
      for (int e = 0; e < Sh::V; ++e) {
        float v = dv[e];
        if (p.dt_bias && c + e < nch) v += __ldg(p.dt_bias + c0 + c + e);
        s_dg[t][c + e] = make_float2(p.softplus ? softplusf(v) : v, p.z ? gv[e] * siluf(zv[e]) : gv[e]);
      }
    }
#pragma unroll
    for (int i = 0; i < Sh::NB; ++i) {
      const int id = i * kScanThreads + tid;
      s_C[id / Sh::SP][id % Sh::SP] = to_f32<T>(tc.raw[i]);
    }
    __syncthreads();
    load(r - kScanTile);
#pragma unroll 4
    for (int t = ntok - 1; t >= 0; --t) {
      const float4 c4 = *reinterpret_cast<const float4 *>(&s_C[t][n0]);
      const float cc[4] = {c4.x, c4.y, c4.z, c4.w};
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float2 d = s_dg[t][ch0 + j];
        sumd[j] += d.x;
#pragma unroll
        for (int i = 0; i < 4; ++i) q[j][i] = decay(d.x, A2[j][i]) * fmaf(cc[i], d.y, q[j][i]);
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    if (ch0 + j >= nch) continue;
    const size_t u = blockIdx.x, d = c0 + ch0 + j;
    if (sl == 0) p.sumd[u * p.D + d] = sumd[j];
    *reinterpret_cast<float4 *>(p.carry + (u * p.D + d) * Sh::SP + n0) =
        make_float4(q[j][0], q[j][1], q[j][2], q[j][3]);
  }
}

template <int L>
struct BwdShape {
  static constexpr int CL = 32 / L;                // channel lanes
  static constexpr int PB = CL < 4 ? CL : 4;       // orders of a lane's four states (n ^ (cl % PB))
};

// The sums over a warp's channel lanes of db[i] and dc[i] (i-th state in this
// lane's order), written to red[0 .. 4 L) (dB) and red[4 L .. 8 L) (dC).
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

// out[i] = v[i ^ perm]
__device__ __forceinline__ void permute(const float (&v)[4], int perm, float (&out)[4]) {
  const bool b0 = perm & 1, b1 = perm & 2;
  float a[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) a[i] = b0 ? v[i ^ 1] : v[i];
#pragma unroll
  for (int i = 0; i < 4; ++i) out[i] = b1 ? a[i ^ 2] : a[i];
}

template <typename T, int L, bool VEC>
struct BwdSmem {
  using Sh = ScanShape<T, L, VEC>;
  static constexpr int PB = BwdShape<L>::PB;
  float2 dx[kScanTile][Sh::CT];                    // (dl, dl x)
  float gy[kScanTile][Sh::CT];
  float B[kScanTile][PB][Sh::SP], C[kScanTile][PB][Sh::SP];  // in each of the PB orders
  float sums[3][kScanTile][Sh::CT];                // sum_n g B, sum_n A2 q h, y
  float red[kScanWarps][kScanTile][2 * Sh::SP];    // dB, dC of each warp's channels
  float acc[2][Sh::V][kScanThreads];               // dD and ddt_bias of a thread's elements
};

template <typename T, int L, bool VEC>
__global__ void __launch_bounds__(kScanThreads) scan_bwd_kernel(ScanP p) {
  using Sh = ScanShape<T, L, VEC>;
  using Rows = TileRows<T, L, VEC>;
  using K = typename Rows::K;
  using Sm = BwdSmem<T, L, VEC>;
  extern __shared__ __align__(16) unsigned char smem_raw[];
  Sm &sm = *reinterpret_cast<Sm *>(smem_raw);
  const Unit w = find_unit(p, blockIdx.x);
  const size_t u = blockIdx.x;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int sl = lane % L, cl = lane / L, n0 = sl * 4, perm = cl % Sm::PB;
  const int g = blockIdx.y / p.tiles_g, Dg = p.D / p.G;
  const int c0 = g * Dg + blockIdx.y % p.tiles_g * Sh::CT;
  const int nch = min(Sh::CT, (g + 1) * Dg - c0);
  int ch[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) ch[j] = warp * Sh::CW + cl * 2 + (j ^ (sl & 1));
  float A2[2][4], q[2][4], dA[2][4];
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = n0 + (i ^ perm);
      q[j][i] = dA[j][i] = 0.f;
      A2[j][i] = ch[j] < nch && n < p.S ? __ldg(p.A + (size_t)(c0 + ch[j]) * p.S + n) * kLog2e : 0.f;
    }
#pragma unroll
  for (int e = 0; e < Sh::V; ++e) sm.acc[0][e][tid] = sm.acc[1][e][tid] = 0.f;
  const long long r0 = w.ok ? w.begin + (long long)w.j * p.seg : 0;
  const long long r1 = w.ok ? min(r0 + p.seg, w.end) : 0;
  if (w.ok) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {  // q past the unit's end
      if (ch[j] >= nch) continue;
      const size_t d = c0 + ch[j];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int n = n0 + (i ^ perm);
        if (p.dhT && n < p.S) q[j][i] = p.dhT[((size_t)w.s * p.D + d) * p.S + n];
      }
      for (int k = w.n - 1; k > w.j; --k) {
        const size_t v = u - w.j + k;
        const float sd = p.sumd[v * p.D + d];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          q[j][i] = fmaf(decay(sd, A2[j][i]), q[j][i], p.carry[(v * p.D + d) * Sh::SP + n0 + (i ^ perm)]);
      }
    }
  }
  const T *X = (const T *)p.x + c0, *DT = (const T *)p.dt + c0, *DO = (const T *)p.dout + c0;
  const T *Z = p.z ? (const T *)p.z + c0 : nullptr;
  const T *Bm = (const T *)p.Bm + (size_t)g * p.S, *Cm = (const T *)p.Cm + (size_t)g * p.S;
  Rows x, dt, z, dout;
  TileBC<T, L> tb, tc;
  float hn[2][4];  // the state before the tile, in this lane's order
  auto load = [&](long long r) {
    const int ntok = r < r0 ? 0 : (int)min((long long)kScanTile, r1 - r);
    const long long slot = w.chunk0 + (r - w.begin) / kScanTile;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float v[4] = {0.f, 0.f, 0.f, 0.f};
      if (ntok && ch[j] < nch && slot < p.slots)
        load_states(p.chunks + ((size_t)slot * p.D + c0 + ch[j]) * p.S, p.S, n0, v);
      permute(v, perm, hn[j]);
    }
    x.load(X + r * p.x_ld, p.x_ld, ntok, nch);
    dt.load(DT + r * p.dt_ld, p.dt_ld, ntok, nch);
    dout.load(DO + r * p.dout_ld, p.dout_ld, ntok, nch);
    z.load(Z ? Z + r * p.z_ld : nullptr, p.z_ld, ntok, nch);
    tb.load(Bm + r * p.b_ld, p.b_ld, ntok, p.S);
    tc.load(Cm + r * p.c_ld, p.c_ld, ntok, p.S);
  };
  const long long last = r1 > r0 ? r0 + (r1 - 1 - r0) / kScanTile * kScanTile : r0 - kScanTile;
  if (last >= r0) load(last);
  for (long long r = last; r >= r0; r -= kScanTile) {
    const int ntok = (int)min((long long)kScanTile, r1 - r);
    // the tile's operands into shared memory
#pragma unroll
    for (int i = 0; i < Sh::NV; ++i) {
      const int id = i * kScanThreads + tid, t = id / Sh::COLS, c = id % Sh::COLS * Sh::V;
      if (t >= kScanTile) break;
      float xv[Sh::V], dv[Sh::V], zv[Sh::V], gv[Sh::V];
      x.get(i, xv);
      dt.get(i, dv);
      z.get(i, zv);
      dout.get(i, gv);
#pragma unroll
      for (int e = 0; e < Sh::V; ++e) {
        float v = dv[e];
        if (p.dt_bias && c + e < nch) v += __ldg(p.dt_bias + c0 + c + e);
        const float dl = p.softplus ? softplusf(v) : v;
        sm.dx[t][c + e] = make_float2(dl, dl * xv[e]);
        sm.gy[t][c + e] = p.z ? gv[e] * siluf(zv[e]) : gv[e];
      }
    }
#pragma unroll
    for (int i = 0; i < Sh::NB; ++i) {
      const int id = i * kScanThreads + tid, t = id / Sh::SP, n = id % Sh::SP;
      const float b = to_f32<T>(tb.raw[i]), c = to_f32<T>(tc.raw[i]);
#pragma unroll
      for (int k = 0; k < Sm::PB; ++k) {
        sm.B[t][k][n ^ k] = b;
        sm.C[t][k][n ^ k] = c;
      }
    }
    float hs[2][4];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) hs[j][i] = hn[j][i];
    const Rows xc = x, zc = z, doc = dout, dtc = dt;
    __syncthreads();
    load(r - kScanTile);
#pragma unroll 1
    for (int half = ntok > kSub ? 1 : 0; half >= 0; --half) {
      float h0[2][4], hist[kSub][2][4];
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) h0[j][i] = hs[j][i];
      auto step = [&](int t, const float (&from)[2][4], float (&to)[2][4]) {
        const float4 b4 = *reinterpret_cast<const float4 *>(&sm.B[t][perm][n0]);
        const float bb[4] = {b4.x, b4.y, b4.z, b4.w};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float2 d = sm.dx[t][ch[j]];
#pragma unroll
          for (int i = 0; i < 4; ++i) to[j][i] = fmaf(decay(d.x, A2[j][i]), from[j][i], d.y * bb[i]);
        }
      };
      if (half) {
#pragma unroll
        for (int t = 0; t < kSub; ++t) step(t, h0, h0);
      }
#pragma unroll
      for (int t = 0; t < kSub; ++t) step(half * kSub + t, t ? hist[t - 1] : h0, hist[t]);
#pragma unroll
      for (int t4 = kSub - 4; t4 >= 0; t4 -= 4) {
        float gB[4][2], Aq[4][2], y[4][2];
#pragma unroll
        for (int k = 3; k >= 0; --k) {
          const int tl = t4 + k, t = half * kSub + tl;
#pragma unroll
          for (int j = 0; j < 2; ++j) gB[k][j] = Aq[k][j] = y[k][j] = 0.f;
          if (t >= ntok) continue;
          const float4 b4 = *reinterpret_cast<const float4 *>(&sm.B[t][perm][n0]);
          const float4 c4 = *reinterpret_cast<const float4 *>(&sm.C[t][perm][n0]);
          const float bb[4] = {b4.x, b4.y, b4.z, b4.w}, cc[4] = {c4.x, c4.y, c4.z, c4.w};
          float db[4] = {0.f, 0.f, 0.f, 0.f}, dc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float2 d = sm.dx[t][ch[j]];
            const float gy = sm.gy[t][ch[j]];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float h = hist[tl][j][i], hp = tl ? hist[tl - 1][j][i] : h0[j][i];
              const float gg = fmaf(cc[i], gy, q[j][i]);
              y[k][j] = fmaf(cc[i], h, y[k][j]);
              gB[k][j] = fmaf(gg, bb[i], gB[k][j]);
              dc[i] = fmaf(gy, h, dc[i]);
              db[i] = fmaf(gg, d.y, db[i]);
              q[j][i] = decay(d.x, A2[j][i]) * gg;
              const float qh = q[j][i] * hp;
              dA[j][i] = fmaf(d.x, qh, dA[j][i]);
              Aq[k][j] = fmaf(A2[j][i], qh, Aq[k][j]);
            }
          }
          sum_channels<L>(db, dc, sl, cl, &sm.red[warp][t][0]);
        }
        const int tb4 = half * kSub + t4;
        sum_states<L>(gB, &sm.sums[0][tb4][0], Sh::CT, ch[0], sl);
        sum_states<L>(Aq, &sm.sums[1][tb4][0], Sh::CT, ch[0], sl);
        sum_states<L>(y, &sm.sums[2][tb4][0], Sh::CT, ch[0], sl);
      }
    }
    __syncthreads();
    // results of the tile's elements
#pragma unroll
    for (int i = 0; i < Sh::NV; ++i) {
      const int id = i * kScanThreads + tid, t = id / Sh::COLS, c = id % Sh::COLS * Sh::V;
      if (t >= ntok || c >= nch) continue;
      float xv[Sh::V], dv[Sh::V], zv[Sh::V], gv[Sh::V], dx[Sh::V], ddt[Sh::V], dz[Sh::V];
      xc.get(i, xv);
      dtc.get(i, dv);
      zc.get(i, zv);
      doc.get(i, gv);
#pragma unroll
      for (int e = 0; e < Sh::V; ++e) {
        const float dl = sm.dx[t][c + e].x, gy = sm.gy[t][c + e], gB = sm.sums[0][t][c + e];
        const float Dk = p.Dskip ? __ldg(p.Dskip + c0 + c + e) : 0.f;
        float v = dv[e];
        if (p.dt_bias) v += __ldg(p.dt_bias + c0 + c + e);
        dx[e] = fmaf(dl, gB, Dk * gy);
        const float ddl = fmaf(sm.sums[1][t][c + e], kLn2, gB * xv[e]);
        ddt[e] = p.softplus ? ddl * sigmoidf(v) : ddl;
        if (p.z) dz[e] = gv[e] * fmaf(Dk, xv[e], sm.sums[2][t][c + e]) * silu_grad(zv[e], sigmoidf(zv[e]));
        sm.acc[0][e][tid] = fmaf(gy, xv[e], sm.acc[0][e][tid]);
        sm.acc[1][e][tid] += ddt[e];
      }
      const long long row = r + t;
      K::st((T *)p.dx + c0 + row * p.dx_ld + c, K::put(dx));
      K::st((T *)p.ddt + c0 + row * p.ddt_ld + c, K::put(ddt));
      if (p.z) K::st((T *)p.dz + c0 + row * p.dz_ld + c, K::put(dz));
    }
    for (int i = tid; i < ntok * 2 * Sh::SP; i += kScanThreads) {
      const int t = i / (2 * Sh::SP), n = i % (2 * Sh::SP);
      float a = sm.red[0][t][n];
#pragma unroll
      for (int k = 1; k < kScanWarps; ++k) a += sm.red[k][t][n];
      p.part_bc[((size_t)blockIdx.y * p.B * p.T + r + t) * (2 * Sh::SP) + n] = a;
    }
    __syncthreads();
  }
  // parameter gradients of the unit (zero where it has no tokens), dh0
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    if (ch[j] >= nch) continue;
    const size_t d = c0 + ch[j];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = n0 + (i ^ perm);
      if (n >= p.S) continue;
      p.part_A[(u * p.D + d) * p.S + n] = dA[j][i];
      if (p.dh0 && w.ok && w.j == 0) p.dh0[((size_t)w.s * p.D + d) * p.S + n] = q[j][i];
    }
  }
  __syncthreads();
  for (int i = tid; i < 2 * Sh::CT; i += kScanThreads) {
    const int which = i / Sh::CT, c = i % Sh::CT;
    if (c >= nch) continue;
    float a = 0.f;  // the threads that hold channel c: columns c / V of every row of threads
    for (int k = c / Sh::V; k < kScanThreads; k += Sh::COLS) a += sm.acc[which][c % Sh::V][k];
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
BwdWs bwd_ws(const rdn_scan_args &a, const ScanPlan &pl) {
  BwdWs w{};
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t o = at;
    at += round256(n * sizeof(float));
    return o;
  };
  const size_t SP = 4 * pl.L, units = pl.units, M = (size_t)a.B * a.T;
  w.carry = take(pl.split ? units * a.D * SP : 0);
  w.sumd = take(pl.split ? units * a.D : 0);
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
  if (pl.split)
    RDN_LAUNCH("scan_bwd_carry", s, (scan_bwd_carry_kernel<T, L, VEC><<<grid, kScanThreads, 0, s>>>(p)));
  const int smem = (int)sizeof(BwdSmem<T, L, VEC>);
  cudaError_t e = cudaFuncSetAttribute(scan_bwd_kernel<T, L, VEC>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
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

size_t scan_bwd_bytes(const rdn_scan_args &a) { return bwd_ws(a, scan_plan(a)).total; }

cudaError_t launch_scan_bwd(const rdn_scan_args &a, cudaStream_t s) {
  const ScanPlan pl = scan_plan(a);
  const BwdWs ws = bwd_ws(a, pl);
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
    if ((e = scan_states(a, p, pl, s)) != cudaSuccess) return e;
  }
  return a.dtype == RDN_BF16 ? bwd_t<__nv_bfloat16>(a, p, pl, s) : bwd_t<float>(a, p, pl, s);
}

}  // namespace rdn
