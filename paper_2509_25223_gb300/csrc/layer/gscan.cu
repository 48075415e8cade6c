// gscan.cu -- the gated linear recurrence (include/rdn.h, rdn_gscan_*): one state per
// channel,
//     h_t = a_t h_{t-1} + m_t s_t x_t,   a = exp(la), la = -c softplus(lam) sigmoid(r),
//     m = sqrt(1 - a^2), s = sigmoid(i).
// A span of tokens maps the state before it to the state after it as h -> A h + H, and
// two spans compose to (A2 A1, A2 H1 + H2).  So a token row is cut: half a warp takes kTok
// consecutive tokens of 16 V channels (its lanes), a CTA the kTile tokens of its warps, and,
// where there are too few rows and channels to fill the GPU, a cluster of up to 8 CTAs as many
// tiles, one round after another.  Each half warp works out its span from a zero state; the
// spans' (A, H) go through shared memory, the tiles' to every CTA of the cluster, and the
// states follow as h_t = A_t h_in + H_t.  The data are read once, a round ahead, and the results
// written once.
// The backward is the same over the reversed tokens, with
//     g_t = dy_t + q_{t+1},  q_t = a_t g_t       (q: the gradient of the state before t)
// and the states again from those that the forward kept before every tile:
// with b = m s x, the token's own part of h:
//     dx = g m s,  di = g b (1 - s),  w_t = a g la (h_{t-1} - a b / (1 - a^2)),
//     dr = (1 - sigmoid(r)) w,  dlam = sigmoid(lam) / softplus(lam) sum_t w_t
// (la b / (1 - a^2) stays finite where la -> 0: it is la s x / m, and m ~ sqrt(-2 la)).
#include <float.h>
#include <limits.h>

#include "launch.cuh"
#include "maps.cuh"
#include "rows.cuh"
#include "status.cuh"
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

constexpr int kTok = 8, kWarps = 8, kTile = 2 * kTok * kWarps, kThreads = 32 * kWarps;
constexpr int kLanes = 16;   // lanes of a span
constexpr int kCluster = 8;  // the most CTAs of a cluster
constexpr int kFwdCtas = 3, kBwdCtas = 2;  // resident on an SM (80 and 128 registers a thread, nothing spilled)
constexpr int kKeep = RDN_GSCAN_CHUNK;  // tokens from one kept state to the next
static_assert(kKeep == kTok * kWarps && kTile == 2 * kKeep, "a tile, and its half, start at a kept state");

struct GP {
  int B, T, D, nc, strips, num_seqs, num_slots;
  int inject;  // a test: the copies of each cluster's first CTA seem short, or it sends nothing to the others
  float c;
  long long x_ld, r_ld, i_ld, y_ld, dy_ld, dx_ld, dr_ld, di_ld;
  const void *x, *r, *i, *dy;
  const float *lam, *h0, *dhT;
  void *y, *dx, *dr, *di;
  float *hT, *chunks, *dh0, *part, *dlam;
  const int *cu, *slots;
  float *h;
  int *status;
};

__device__ __forceinline__ float softplusf(float v) { return v > 20.f ? v : log1pf(expf(v)); }

// The arithmetic is on pairs of channels (rows.cuh): one issue slot for two of them.  A lane with
// one channel (V = 1) has a second one of zeros.
__device__ __forceinline__ f2 both(float v) { return pack2(v, v); }
template <typename T, int V>
__device__ __forceinline__ f2 get2(const typename Pack<T, V>::Raw &raw) {
  float v[V];
  Pack<T, V>::get(raw, v);
  return pack2(v[0], V == 2 ? v[V - 1] : 0.f);
}
template <typename T, int V>
__device__ __forceinline__ void put2(T *p, f2 v) {
  float lo, hi;
  unpack2(v, lo, hi);
  float o[V];
  o[0] = lo;
  if (V == 2) o[V - 1] = hi;
  Pack<T, V>::st(p, Pack<T, V>::put(o));
}
template <int V>
__device__ __forceinline__ f2 ldf(const float *p) { return pack2(p[0], V == 2 ? p[V - 1] : 0.f); }
template <int V>
__device__ __forceinline__ void stf(float *p, f2 v) {
  float lo, hi;
  unpack2(v, lo, hi);
  p[0] = lo;
  if (V == 2) p[V - 1] = hi;
}
// The larger of two numbers, or the NaN among them.
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.ftz.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// fn of each of a pair.
template <typename Fn>
__device__ __forceinline__ f2 each(f2 x, Fn fn) {
  float lo, hi;
  unpack2(x, lo, hi);
  return pack2(fn(lo), fn(hi));
}
__device__ __forceinline__ f2 sqrt2(f2 x) {
  return each(x, [](float v) {
    asm("sqrt.approx.ftz.f32 %0, %0;" : "+f"(v));
    return v;
  });
}
// 1 / x, a large number for x = 0
__device__ __forceinline__ f2 rcp2(f2 x) {
  return each(x, [](float v) { return rcp_approx(max_nan(v, 2e-38f)); });
}
__device__ __forceinline__ f2 sub2(f2 a, f2 b) {
  float x, y, z, w;
  unpack2(a, x, y);
  unpack2(b, z, w);
  return pack2(x - z, y - w);
}

// The gates of a pair: s = sigmoid of r and of i, u = 1 - a, t = log2(a).
//   k = -c softplus(lam) log2(e);  log2 of a decay below 2^-125 is taken as -125.
// u keeps its digits where a is near 1, so that 1 - a^2 = u (2 - u) does: with t = n + f, n the
// nearest integer (both exact), 1 - 2^t = (1 - 2^n) - 2^n (2^f - 1), and 2^f - 1 = f P(f) with the
// polynomial P of degree 5 that has the least largest relative error on |f| <= 1/2, fitted by
// reweighted least squares: 1.1e-8, u within 1.2e-7.
struct Gate {
  f2 sr, si, u;
};
// The steps are packed ones (kPairs) in the kernels by TMA: packed instructions take no constants, so that each
// constant is a pair of registers, and those kernels have them (16384 tokens of 4096 channels 148 -> 138 us).
// The others do not: with two plain instructions that hold the constant they stay under their register limits.
__device__ __forceinline__ float sigmoid_of(float x) { return rcp_approx(1.f + ex2(-kLog2e * x)); }
__device__ __forceinline__ f2 log2_decay(f2 k, f2 sr) {
  return each(mul2(k, sr), [](float v) { return max_nan(v, -125.f); });
}
constexpr float kRound = 12582912.f;  // 1.5 * 2^23
constexpr float kP0 = 0.6931471824645996f, kP1 = 0.24022649228572845f, kP2 = 5.550357326865196e-2f,
                kP3 = 9.618237614631653e-3f, kP4 = 1.3390735257416964e-3f, kP5 = 1.5403510769829154e-4f;
__device__ __forceinline__ float decayed(float t) {  // 1 - 2^t, -125 <= t <= 0
  const float nr = t + kRound, f = t - (nr - kRound);
  float q = fmaf(kP5, f, kP4);
  q = fmaf(q, f, kP3);
  q = fmaf(q, f, kP2);
  q = fmaf(q, f, kP1);
  q = fmaf(q, f, kP0);
  const float s = __uint_as_float((__float_as_uint(nr) << 23) + 0x3f800000u);  // 2^n
  return fmaf(-s, q * f, 1.f - s);
}
template <bool kPairs>
__device__ __forceinline__ f2 one_minus(f2 x) {
  if (kPairs) return fma2(x, both(-1.f), both(1.f));
  return each(x, [](float v) { return 1.f - v; });
}
// 1 - a^2
template <bool kPairs>
__device__ __forceinline__ f2 rest(f2 u) {
  if (kPairs) return mul2(u, fma2(u, both(-1.f), both(2.f)));
  return mul2(u, each(u, [](float v) { return 2.f - v; }));
}
template <bool kPairs>
__device__ __forceinline__ Gate gate(f2 r, f2 i, f2 k) {
  Gate g;
  if (!kPairs) {
    g.sr = each(r, sigmoid_of);
    g.si = each(i, sigmoid_of);
    g.u = each(log2_decay(k, g.sr), decayed);
    return g;
  }
  const f2 one = both(1.f);
  g.sr = each(add2(each(mul2(r, both(-kLog2e)), ex2), one), rcp_approx);
  g.si = each(add2(each(mul2(i, both(-kLog2e)), ex2), one), rcp_approx);
  const f2 t = log2_decay(k, g.sr), nr = add2(t, both(kRound));
  const f2 f = fma2(add2(nr, both(-kRound)), both(-1.f), t);
  f2 q = fma2(both(kP5), f, both(kP4));
  q = fma2(q, f, both(kP3));
  q = fma2(q, f, both(kP2));
  q = fma2(q, f, both(kP1));
  q = fma2(q, f, both(kP0));
  const f2 s = each(nr, [](float v) { return __uint_as_float((__float_as_uint(v) << 23) + 0xbf800000u); });  // -2^n
  g.u = fma2(s, mul2(q, f), add2(one, s));
  return g;
}

constexpr float kLn2 = 0.69314718f;
template <int V>
__device__ __forceinline__ f2 rate(const GP &p, int ch) {  // -c softplus(lam) log2(e)
  // (finite factors: a softplus of 0 times the largest c is 0 too)
  const float c = fmaxf(-p.c * kLog2e, -FLT_MAX);
  const f2 k = mul2(pack2(softplusf(p.lam[ch]), V == 2 ? softplusf(p.lam[ch + V - 1]) : 0.f), both(c));
  return each(k, [](float v) { return max_nan(v, -1e30f); });  // (finite: a closed gate's 0 times it is 0)
}

// The map h -> A h + H of a span of tokens, for a pair of channels.  A = -1 stands for a span in
// which a packed sequence starts: what comes before it does not enter, not even as 0 times an
// infinity or NaN.
struct alignas(16) Span {
  f2 A, H;
};
__device__ __forceinline__ bool cuts(f2 A) {
  float lo, hi;
  unpack2(A, lo, hi);
  return lo < 0.f;
}
template <bool kPacked>
__device__ __forceinline__ f2 over(const Span &s, f2 h) {
  const f2 r = fma2(s.A, h, s.H);
  return kPacked && cuts(s.A) ? s.H : r;
}
// s1, then s2
template <bool kPacked>
__device__ __forceinline__ Span then(const Span &s1, const Span &s2) {
  const f2 A = mul2(s1.A, s2.A);
  return {kPacked && (cuts(s1.A) || cuts(s2.A)) ? both(-1.f) : A, over<kPacked>(s2, s1.H)};
}
// s, then the token h -> a h + b
template <bool kPacked>
__device__ __forceinline__ void step(Span &s, f2 a, f2 b) {
  const f2 A = mul2(s.A, a);
  s.A = kPacked && cuts(s.A) ? s.A : A;
  s.H = fma2(a, s.H, b);
}

// This thread's place.
template <int V>
struct Place {
  int lane, half, warp, rank, b, strip, ch;
  bool live;  // whether the lane's channels exist (if not, it reads the strip's first ones)
  __device__ explicit Place(const GP &p) {
    lane = threadIdx.x & (kLanes - 1);
    half = (threadIdx.x >> 4) & 1;
    warp = threadIdx.x >> 5;
    rank = blockIdx.x % p.nc;
    const int unit = blockIdx.x / p.nc;
    b = unit / p.strips;
    strip = (unit % p.strips) * kLanes * V;
    live = strip + lane * V < p.D;
    ch = live ? strip + lane * V : strip;
  }
  // token of the tile that this thread's span starts at
  __device__ int token() const { return (2 * warp + half) * kTok; }
};

// Sequence that starts / ends at each token of the tile (-1: none).
template <int kTokens = kTile>
__device__ __forceinline__ void mark_tile(const GP &p, int t0, int2 *mark) {
  const int k = threadIdx.x;
  if (k < kTokens) {
    int2 f = make_int2(-1, -1);
    if (t0 + k < p.T) {
      const SeqSpan q = find_seq(p.cu, p.num_seqs, p.T, 0, t0 + k);
      if (q.begin == t0 + k) f.x = q.s;
      if (q.end == t0 + k + 1) f.y = q.s;
    }
    mark[k] = f;
  }
}

// Addresses of a row operand: row (of the B T token rows), 32-bit (a row is below 2^24 elements).
// One instruction an address (a wide multiply-add) where 64-bit sums of offsets would be three.
__device__ __forceinline__ const char *row_at(const char *p, uint32_t row, uint32_t ld) {
  const char *q;
  asm("mad.wide.u32 %0, %1, %2, %3;" : "=l"(q) : "r"(row), "r"(ld), "l"(p));
  __builtin_assume(__isGlobal(q));
  return q;
}
template <typename T>
struct Rows {
  const char *p;  // the lane's channels of token row `row`
  uint32_t ld;    // bytes
  __device__ Rows(const void *base, long long ld_, uint32_t row, int ch)
      : ld((uint32_t)ld_ * (uint32_t)sizeof(T)) {
    p = row_at(static_cast<const char *>(base) + ch * (int)sizeof(T), row, ld);
  }
  __device__ T *operator[](uint32_t j) const { return reinterpret_cast<T *>(const_cast<char *>(row_at(p, j, ld))); }
};
// (left: tokens of the row of the batch from the first one on)
template <typename T, int V>
__device__ __forceinline__ void load_rows(typename Pack<T, V>::Raw (&v)[kTok], const void *base, long long ld,
                                          uint32_t row, int ch, bool full, int left) {
  const Rows<T> rows(base, ld, row, ch);
  if (full) {
#pragma unroll
    for (int j = 0; j < kTok; ++j) v[j] = Pack<T, V>::ld(rows[j]);
  } else {
#pragma unroll
    for (int j = 0; j < kTok; ++j) v[j] = j < left ? Pack<T, V>::ld(rows[j]) : Pack<T, V>::zero();
  }
}

__device__ __forceinline__ Span from_other_half(const Span &s) {
  return {__shfl_xor_sync(0xffffffffu, s.A, kLanes), __shfl_xor_sync(0xffffffffu, s.H, kLanes)};
}

// Leaves the warp's span, of its halves' (kBack: the upper one first).
template <bool kBack, bool kPacked>
__device__ __forceinline__ void leave(Span (*spans)[kLanes], int warp, int lane, int half, const Span &own,
                                      const Span &other) {
  if (half == (kBack ? 1 : 0)) spans[warp][lane] = then<kPacked>(own, other);
}

// A wait that gives up (after about a second; a test's sooner) tells the status word.  The kernels by TMA then leave
// their rounds: the bound that a round's end is compared with lies in shared memory, read behind the round's barrier
// (an instruction a round; a flag and a branch take 1 to 3 %).  The others run their remaining rounds on what is
// there, without exchanges.  Nothing in flight is left behind: a CTA waits for the copies that it began, and the CTAs
// of a cluster for one another and for what they were sent.  No barrier is armed again for which a wait was given up.
struct Lost {
  int end[2];  // by TMA: the bound of even and odd rounds.  One that is given up is set before the round's barrier.
  int gone;    // rows addressed one by one: no further exchange
  int owed;    // by thread 0: 4 + 2 parity + barrier of the last exchange that it gave up
};
__device__ __forceinline__ uint32_t wait_limit(const GP &p) { return p.inject ? 10000000u : 2000000000u; }
__device__ __forceinline__ void tell(const GP &p) {
  if (p.status) atomicExch(p.status, (int)RDN_ERR_TIMEOUT);
}
// tc::mbar_wait_cluster that looks without acquiring until the phase is over: an acquire at cluster scope drops
// the SM's L1 each time it looks.
__device__ __forceinline__ bool wait_cluster(uint64_t *bar, uint32_t parity, uint32_t limit) {
  const uint32_t t0 = (uint32_t)clock();
  while (true) {
    uint32_t over;
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "mbarrier.try_wait.parity.relaxed.cluster.shared::cta.b64 p, [%1], %2, 2000;\n"
        "selp.u32 %0, 1, 0, p;\n"
        "}\n"
        : "=r"(over)
        : "r"(tc::smem_u32(bar)), "r"(parity)
        : "memory");
    if (over) return tc::mbar_try_wait_cluster(bar, parity);
    if ((uint32_t)clock() - t0 > limit) return false;
  }
}

// Sends the composition of the CTA's warps' spans (in the order 0.. or, kBack, 7..) to the
// slot of this CTA in every CTA of the cluster, and waits until all have come.  The stores
// themselves tell the receiver's barrier: a barrier of the cluster would hold this thread
// until its global stores of the round before are done.  (A slot is written again two rounds
// later, by a CTA that has had this CTA's spans of the round between, sent when all its warps
// had read the slot.)  on: it takes part.  Returns whether it did, and its wait did not give up.
template <bool kBack, bool kPacked, int kN>
__device__ __forceinline__ bool exchange(const GP &p, const Span (*spans)[kN], Span (*tiles)[kN], uint64_t *bars,
                                         Lost &lost, bool on, int par, uint32_t phase, int rank) {
  uint64_t *bar = &bars[par];
  const int lane = threadIdx.x % kN, to = threadIdx.x / kN;
  static_assert(kThreads / kN >= kCluster, "lanes for each CTA of the cluster");
  if (threadIdx.x == 0 && on) tc::mbar_expect_tx(bar, (uint32_t)(p.nc * kN * sizeof(Span)));
  if (to < p.nc && on) {
    Span all = spans[kBack ? kWarps - 1 : 0][lane];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) all = then<kPacked>(all, spans[kBack ? kWarps - 1 - w : w][lane]);
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.b64 [%0], {%1, %2}, [%3];" ::"r"(
                     tc::map_rank(&tiles[rank][lane], to)),
                 "l"(all.A), "l"(all.H), "r"(tc::map_rank(bar, to))
                 : "memory");
  }
  __syncwarp();
  if (on && !wait_cluster(bar, phase, wait_limit(p))) {
    tell(p);
    on = false;
    if (threadIdx.x == 0) lost.owed = 4 + 2 * (int)phase + par;
  }
  return on;
}
// After the last barrier of the cluster: what the others sent for the exchange that was given up has come.  (What they
// sent for one that this CTA takes no part in came while they waited for it.)
__device__ __forceinline__ void drain_exchange(const GP &p, uint64_t *bars, const Lost &lost) {
  if (p.nc > 1 && threadIdx.x == 0 && lost.owed)
    wait_cluster(&bars[lost.owed & 1], (uint32_t)(lost.owed >> 1) & 1, wait_limit(p));
}
// Before the first exchange: the barriers are there, and every CTA of the cluster runs.
__device__ __forceinline__ void exchange_init(const GP &p, uint64_t *bars, Lost &lost, int rank) {
  if (p.nc == 1) return;
  if (threadIdx.x == 0) {
    lost = {{0, 0}, p.inject && rank == 0, 0};
    tc::mbar_init(&bars[0], 1);
    tc::mbar_init(&bars[1], 1);
    tc::fence_mbar_init();
  }
  __syncthreads();
  tc::cluster_sync();
}

// The state that comes into this warp's span; carry: into and out of the cluster's round.
template <bool kBack, bool kPacked, int kN>
__device__ __forceinline__ f2 fold(const Span (*spans)[kN], const Span (*tiles)[kN], int lane, int rank, int nc,
                                   int warp, f2 &carry) {
  f2 run = carry;
  if (nc > 1) {
    f2 h = carry;
#pragma unroll 1
    for (int q = 0; q < nc; ++q) {
      const int k = kBack ? nc - 1 - q : q;
      if (k == rank) run = h;
      h = over<kPacked>(tiles[k][lane], h);
    }
    carry = h;
  }
  const int before = kBack ? kWarps - 1 - warp : warp;  // warps whose spans come first
  int w = 0;
#pragma unroll 1
  for (; w < before; ++w) run = over<kPacked>(spans[kBack ? kWarps - 1 - w : w][lane], run);
  const f2 in = run;
  if (nc == 1) {
#pragma unroll 1
    for (; w < kWarps; ++w) run = over<kPacked>(spans[kBack ? kWarps - 1 - w : w][lane], run);
    carry = run;
  }
  return in;
}

// States of sequences without tokens: out = in, or 0.
template <int V, bool kPacked, typename At>
__device__ __forceinline__ void pass_through(const GP &p, const At &at, const float *in, float *out) {
  if (!out || !at.live || at.half) return;
  if (!kPacked) {
    const size_t o = (size_t)at.b * p.D + at.ch;
    if (p.T == 0 && at.rank == 0 && at.warp == 0) stf<V>(out + o, in ? ldf<V>(in + o) : both(0.f));
  } else {
    for (int s = at.rank * kWarps + at.warp; s < p.num_seqs; s += p.nc * kWarps)
      if (cu_at(p.cu, p.num_seqs, p.T, s + 1) <= cu_at(p.cu, p.num_seqs, p.T, s)) {
        const size_t o = (size_t)s * p.D + at.ch;
        stf<V>(out + o, in ? ldf<V>(in + o) : both(0.f));
      }
  }
}

// Whether a tile of packed tokens holds no first or last token of a sequence: the sequence (begin, end) of its
// first token, kept from round to round, answers it without a look at the table.
struct Inside {
  int begin = 0, end = 0;
  __device__ bool plain(int tile0, int tokens) const { return begin < tile0 && tile0 + tokens < end; }
  __device__ void move(const GP &p, int tile0) {  // to the tile at tile0
    if (tile0 < 0 || tile0 >= p.T || (begin <= tile0 && tile0 < end)) return;
    const SeqSpan q = find_seq(p.cu, p.num_seqs, p.T, 0, tile0);
    begin = (int)q.begin;
    end = (int)q.end;
  }
};

// ---- forward with rows addressed one by one.  8 x 2048 tokens of 1024 channels in fp32: 55 us, 4.8 TB/s; bound by
// the rounds' latency and instruction issue.
template <typename T, int V, bool kPacked>
__global__ void __launch_bounds__(kThreads, kFwdCtas) fwd_kernel(const GP p) {
  using Raw = typename Pack<T, V>::Raw;
  __shared__ Span kept[kTok][kThreads];  // the span up to each token of a thread
  __shared__ Span spans[2][kWarps][kLanes], tiles[2][kCluster][kLanes];
  __shared__ int2 mark[2][kPacked ? kTile : 1];
  __shared__ uint64_t bars[2];
  __shared__ Lost lost;
  const Place<V> at(p);
  const int me = threadIdx.x;
  const uint32_t row0 = (uint32_t)at.b * (uint32_t)p.T + (uint32_t)at.token();  // (B T is at most 2^30)
  const int nkept = (p.T + kKeep - 1) / kKeep, round = p.nc * kTile;
  const f2 k = rate<V>(p, at.ch);
  f2 carry = !kPacked && p.h0 ? ldf<V>(p.h0 + (size_t)at.b * p.D + at.ch) : both(0.f);
  pass_through<V, kPacked>(p, at, p.h0, p.hT);

  exchange_init(p, bars, lost, at.rank);
  int par = 0, tile0 = at.rank * kTile;
  uint32_t phase = 0;
  Inside inside;
  Raw xr[kTok], rr[kTok], ir[kTok];
  auto fetch = [&](int t) {
    const bool full = t + kTile <= p.T;
    const int left = p.T - t - at.token();
    load_rows<T, V>(rr, p.r, p.r_ld, row0 + t, at.ch, full, left);
    load_rows<T, V>(ir, p.i, p.i_ld, row0 + t, at.ch, full, left);
    load_rows<T, V>(xr, p.x, p.x_ld, row0 + t, at.ch, full, left);
  };
  fetch(tile0);
  for (int base = 0; base < p.T; base += round, tile0 += round, phase ^= par, par ^= 1) {
    const int left = p.T - tile0 - at.token();
    if (kPacked) inside.move(p, tile0);
    const bool marked = kPacked && !inside.plain(tile0, kTile);
    if (marked) {
      mark_tile(p, tile0, mark[par]);
      __syncthreads();
    }
    Span all = {both(1.f), both(0.f)};
    auto token = [&](int j) {
      const Gate g = gate<false>(get2<T, V>(rr[j]), get2<T, V>(ir[j]), k);
      const f2 a = one_minus<false>(g.u);
      f2 b = mul2(mul2(sqrt2(rest<false>(g.u)), g.si), get2<T, V>(xr[j]));
      const int start = marked ? mark[par][at.token() + j].x : -1;
      if (kPacked && start >= 0) {
        if (p.h0) b = fma2(a, ldf<V>(p.h0 + (size_t)start * p.D + at.ch), b);
        all = {both(-1.f), b};
      } else {
        step<kPacked>(all, a, b);
      }
      kept[j][me] = all;
    };
    if (tile0 + kTile <= p.T) {
#pragma unroll
      for (int j = 0; j < kTok; ++j) token(j);
    } else {
#pragma unroll
      for (int j = 0; j < kTok; ++j)
        if (j < left) token(j);
    }
    // the next round's rows are on their way while the spans are joined
    if (base + round < p.T) fetch(tile0 + round);
    const Span other = from_other_half(all);
    leave<false, kPacked>(spans[par], at.warp, at.lane, at.half, all, other);
    __syncthreads();
    if (p.nc > 1 && !exchange<false, kPacked>(p, spans[par], tiles[par], bars, lost, !lost.gone, par, phase, at.rank))
      lost.gone = 1;
    f2 in = fold<false, kPacked>(spans[par], tiles[par], at.lane, at.rank, p.nc, at.warp, carry);
    if (p.chunks && at.live && at.token() % kKeep == 0 && left > 0)
      stf<V>(p.chunks + ((size_t)at.b * nkept + (tile0 + at.token()) / kKeep) * p.D + at.ch, in);
    if (at.half) in = over<kPacked>(other, in);
    if (at.live) {
      if (p.y) {
        const Rows<T> y(p.y, p.y_ld, row0 + tile0, at.ch);
        if (tile0 + kTile <= p.T) {
#pragma unroll
          for (int j = 0; j < kTok; ++j) put2<T, V>(y[j], over<kPacked>(kept[j][me], in));
        } else {
#pragma unroll
          for (int j = 0; j < kTok; ++j)
            if (j < left) put2<T, V>(y[j], over<kPacked>(kept[j][me], in));
        }
      }
      if (p.hT) {
        if (marked) {
          for (int j = 0; j < kTok; ++j) {
            const int end = mark[par][at.token() + j].y;
            if (end >= 0) stf<V>(p.hT + (size_t)end * p.D + at.ch, over<kPacked>(kept[j][me], in));
          }
        } else if (!kPacked && left >= 1 && left <= kTok) {  // the row's last token
          stf<V>(p.hT + (size_t)at.b * p.D + at.ch, over<kPacked>(all, in));
        }
      }
    }
    __syncwarp();
  }
  if (p.nc > 1) tc::cluster_sync();  // (what this CTA sent has arrived)
  drain_exchange(p, bars, lost);
}

// ---- forward for bf16 rows on 16 bytes: tiles by TMA.  As fwd_kernel, but a warp takes kTok tokens of 64
// channels, so that a tile is 64 tokens of 128 bytes, and the tiles come to shared memory a round ahead
// (and go from there) as whole boxes: no addresses are worked out per row, which are a quarter of
// fwd_kernel's instructions, and the spans of a thread's tokens stay in its registers.
// 8 x 4096 tokens of 2048 channels: 129 us, 4.2 TB/s, 36 warp instructions for 32 elements (five of them special
// functions); bound by issue and by the units' number (256 on 152 SMs leave 16 % of them idle).
constexpr int kWide = 64, kTileTma = kKeep;  // channels and tokens of a box
constexpr int kTmaUnits = 36;
struct alignas(64) TileMap { unsigned char b[128]; };
struct FwdMaps { TileMap x, r, i, y; };
struct FwdTiles {
  __nv_bfloat16 in[2][3][kTileTma][kWide], y[kTileTma][kWide];
};

struct WidePlace {
  int lane, warp, rank, b, strip, ch;
  bool live;
  static constexpr int half = 0;
  __device__ explicit WidePlace(const GP &p) {
    lane = threadIdx.x & 31;
    warp = threadIdx.x >> 5;
    rank = blockIdx.x % p.nc;
    const int unit = blockIdx.x / p.nc;
    b = unit / p.strips;
    strip = (unit % p.strips) * kWide;
    live = strip + lane * 2 < p.D;
    ch = live ? strip + lane * 2 : strip;
  }
};

template <bool kPacked>
__global__ void __launch_bounds__(kThreads, kFwdCtas) fwd_tma_kernel(const GP p, const __grid_constant__ FwdMaps maps) {
  using bf = __nv_bfloat16;
  extern __shared__ __align__(128) unsigned char dynamic[];
  FwdTiles &sm = *reinterpret_cast<FwdTiles *>(dynamic + ((128 - (tc::smem_u32(dynamic) & 127)) & 127));
  __shared__ Span spans[2][kWarps][32], tiles[2][kCluster][32];
  __shared__ int2 mark[2][kPacked ? kTileTma : 1];
  __shared__ uint64_t bars[2], full[2];
  __shared__ Lost lost;
  const WidePlace at(p);
  const int round = p.nc * kTileTma, nkept = (p.T + kKeep - 1) / kKeep;
  auto fetch = [&](int t, int s) {  // by one thread
    tc::mbar_expect_tx(&full[s], (uint32_t)sizeof(sm.in[s]) + (p.inject && at.rank == 0 ? 16 : 0));
    tc::tma_load_3d(sm.in[s][0], &maps.r, at.strip, t, at.b, &full[s]);
    tc::tma_load_3d(sm.in[s][1], &maps.i, at.strip, t, at.b, &full[s]);
    tc::tma_load_3d(sm.in[s][2], &maps.x, at.strip, t, at.b, &full[s]);
  };
  int tile0 = at.rank * kTileTma;
  if (threadIdx.x == 0) {
    tc::mbar_init(&full[0], 1);
    tc::mbar_init(&full[1], 1);
    tc::mbar_init(&bars[0], 1);
    tc::mbar_init(&bars[1], 1);
    lost = {{p.T, p.T}, 0, 0};
    tc::fence_mbar_init();
    for (int s = 0; s < 2; ++s)
      if (s * round < p.T) fetch(tile0 + s * round, s);
  }
  const f2 k = rate<2>(p, at.ch);
  f2 carry = !kPacked && p.h0 ? ldf<2>(p.h0 + (size_t)at.b * p.D + at.ch) : both(0.f);
  pass_through<2, kPacked>(p, at, p.h0, p.hT);
  __syncthreads();
  if (p.nc > 1) tc::cluster_sync();  // the barriers are there, and every CTA of the cluster runs

  int par = 0;  // also the stage
  uint32_t phase = 0;
  Inside inside;
  int base = 0, end;
  do {
    const int first = at.warp * kTok, left = p.T - tile0 - first;
    if (kPacked) inside.move(p, tile0);
    const bool marked = kPacked && !inside.plain(tile0, kTileTma);
    if (marked) {
      mark_tile<kTileTma>(p, tile0, mark[par]);
      __syncthreads();
    }
    if (!tc::mbar_wait(&full[par], phase, wait_limit(p))) {
      tell(p);
      lost.end[par] = 0;
    }
    // (tokens past the row's end are zeros, which nothing that is kept follows)
    Span all = {both(1.f), both(0.f)}, kept[kTok];
#pragma unroll
    for (int j = 0; j < kTok; ++j) {
      const Gate g = gate<true>(get2<bf, 2>(Pack<bf, 2>::ld(&sm.in[par][0][first + j][at.lane * 2])),
                                get2<bf, 2>(Pack<bf, 2>::ld(&sm.in[par][1][first + j][at.lane * 2])), k);
      const f2 a = one_minus<true>(g.u);
      f2 b = mul2(mul2(sqrt2(rest<true>(g.u)), g.si),
                  get2<bf, 2>(Pack<bf, 2>::ld(&sm.in[par][2][first + j][at.lane * 2])));
      const int start = marked ? mark[par][first + j].x : -1;
      if (kPacked && start >= 0) {
        if (p.h0) b = fma2(a, ldf<2>(p.h0 + (size_t)start * p.D + at.ch), b);
        all = {both(-1.f), b};
      } else {
        step<kPacked>(all, a, b);
      }
      kept[j] = all;
    }
    spans[par][at.warp][at.lane] = all;
    __syncthreads();
    end = lost.end[par];
    if (threadIdx.x == 0 && base + 2 * round < end) fetch(tile0 + 2 * round, par);  // the stage has been read
    __syncwarp();
    if (p.nc > 1 && !exchange<false, kPacked>(p, spans[par], tiles[par], bars, lost, true, par, phase, at.rank))
      lost.end[par ^ 1] = 0;
    const f2 in = fold<false, kPacked>(spans[par], tiles[par], at.lane, at.rank, p.nc, at.warp, carry);
    if (p.chunks && at.live && at.warp == 0 && tile0 < p.T)
      stf<2>(p.chunks + ((size_t)at.b * nkept + tile0 / kKeep) * p.D + at.ch, in);
    if (p.y) {
      if (at.lane == 0) tc::bulk_wait_read();  // the round before has left the warp's rows
      __syncwarp();
#pragma unroll
      for (int j = 0; j < kTok; ++j) put2<bf, 2>(&sm.y[first + j][at.lane * 2], over<kPacked>(kept[j], in));
      tc::fence_async_smem();
      __syncwarp();
      if (at.lane == 0 && left > 0) {  // (what is past the tensor's ends is left out)
        tc::tma_store_3d(&maps.y, at.strip, tile0 + first, at.b, sm.y[first]);
        tc::bulk_commit();
      }
    }
    if (p.hT && at.live) {
      if (marked) {
        for (int j = 0; j < kTok; ++j) {
          const int end = mark[par][first + j].y;
          if (end >= 0) {
#pragma unroll
            for (int q = 0; q < kTok; ++q)
              if (q == j) stf<2>(p.hT + (size_t)end * p.D + at.ch, over<kPacked>(kept[q], in));
          }
        }
      } else if (!kPacked && left >= 1 && left <= kTok) {  // the row's last token
#pragma unroll
        for (int q = 0; q < kTok; ++q)
          if (q == left - 1) stf<2>(p.hT + (size_t)at.b * p.D + at.ch, over<kPacked>(kept[q], in));
      }
    }
    __syncwarp();
    base += round;
    tile0 += round;
    phase ^= par;
    par ^= 1;
  } while (base < end);
  if (at.lane == 0) tc::bulk_wait_all();
  if (threadIdx.x == 0) {  // the last round's copies and, where the rounds were left, the next one's have come
    tc::mbar_wait(&full[par ^ 1], phase ^ (uint32_t)(par ^ 1), wait_limit(p));
    if (base < p.T) tc::mbar_wait(&full[par], phase, wait_limit(p));
  }
  __syncwarp();
  if (p.nc > 1) tc::cluster_sync();  // (what this CTA sent has arrived)
  drain_exchange(p, bars, lost);
}

// dlam = sigmoid(lam) / softplus(lam) times the sum of w, here of w / ln 2.
__device__ __forceinline__ float dlam_of(float lam, float sum) {
  // (both are e^lam to the last digit where lam is far below zero)
  const float ratio = lam < -20.f ? 1.f : __fdividef(1.f, (1.f + expf(-lam)) * softplusf(lam));
  return sum * ratio * kLn2;
}
// The end of a backward: s, the CTA's sum of w / ln 2 (in `lead`, a thread of each lane), is joined over the
// cluster, its CTAs in order, and with one row of the batch that is dlam (a launch less: 3001 tokens of 1024
// channels in 7 sequences, forward and backward, 59.8 -> 56.1 us, in a graph 54.1 -> 51.8).
template <int V, int kN, typename At>
__device__ __forceinline__ void leave_sum(const GP &p, const At &at, bool lead, f2 s, f2 (*joined)[kN]) {
  if (p.nc > 1) {
    if (lead)
      asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(tc::map_rank(&joined[at.rank][at.lane], 0)), "l"(s)
                   : "memory");
    __syncwarp();
    tc::cluster_sync();  // (also: what this CTA sent before has arrived)
    if (at.rank) return;
    if (lead) {
      s = joined[0][at.lane];
      for (int q = 1; q < p.nc; ++q) s = add2(s, joined[q][at.lane]);
    }
  }
  if (!lead || !at.live) return;
  if (p.B > 1) {
    stf<V>(p.part + (size_t)at.b * p.D + at.ch, s);
  } else {
    float lo, hi;
    unpack2(s, lo, hi);
    stf<V>(p.dlam + at.ch, pack2(dlam_of(p.lam[at.ch], lo), V == 2 ? dlam_of(p.lam[at.ch + V - 1], hi) : 0.f));
  }
}

// What the first pass over a tile leaves for the second, in shared memory: thread-private, a
// pair of each at [token][thread].  (ms: m s; before: the state before each token.)
struct Kept {
  f2 sr[kTok][kThreads], si[kTok][kThreads], u[kTok][kThreads], ms[kTok][kThreads], before[kTok][kThreads];
};

// ---- backward with rows addressed one by one.  8 x 2048 tokens of 1024 channels in fp32: 94 us, 5.0 TB/s.
template <typename T, int V, bool kPacked>
__global__ void __launch_bounds__(kThreads, kBwdCtas) bwd_kernel(const GP p) {
  using Raw = typename Pack<T, V>::Raw;
  extern __shared__ __align__(128) unsigned char dynamic[];
  Kept &kept = *reinterpret_cast<Kept *>(dynamic);
  __shared__ Span fspans[2][kWarps][kLanes], spans[2][kWarps][kLanes], tiles[2][kCluster][kLanes];
  __shared__ int2 mark[2][kPacked ? kTile : 1];
  __shared__ f2 joined[kCluster][kLanes];
  __shared__ uint64_t bars[2];
  __shared__ Lost lost;
  const Place<V> at(p);
  const int me = threadIdx.x;
  const uint32_t row0 = (uint32_t)at.b * (uint32_t)p.T + (uint32_t)at.token();  // (B T is at most 2^30)
  const int nkept = (p.T + kKeep - 1) / kKeep, round = p.nc * kTile;
  const f2 k = rate<V>(p, at.ch), one = both(1.f);
  f2 carry = !kPacked && p.dhT ? ldf<V>(p.dhT + (size_t)at.b * p.D + at.ch) : both(0.f);
  f2 sum = both(0.f);
  pass_through<V, kPacked>(p, at, p.dhT, p.dh0);

  exchange_init(p, bars, lost, at.rank);
  int par = 0;
  uint32_t phase = 0;
  Inside inside;
  const int last = p.T > 0 ? (p.T - 1) / round * round : -1;
  int tile0 = last + at.rank * kTile;
  Raw rr[kTok], ir[kTok];
  auto fetch = [&](int t) {
    const bool full = t + kTile <= p.T;
    const int left = p.T - t - at.token();
    load_rows<T, V>(rr, p.r, p.r_ld, row0 + t, at.ch, full, left);
    load_rows<T, V>(ir, p.i, p.i_ld, row0 + t, at.ch, full, left);
  };
  if (last >= 0) fetch(tile0);
  for (int base = last; base >= 0; base -= round, tile0 -= round, phase ^= par, par ^= 1) {
    const int left = p.T - tile0 - at.token();
    const bool full = tile0 + kTile <= p.T;
    Raw xr[kTok], gr[kTok];
    load_rows<T, V>(xr, p.x, p.x_ld, row0 + tile0, at.ch, full, left);
    load_rows<T, V>(gr, p.dy, p.dy_ld, row0 + tile0, at.ch, full, left);
    f2 h = tile0 < p.T ? ldf<V>(p.chunks + ((size_t)at.b * nkept + tile0 / kKeep) * p.D + at.ch) : both(0.f);
    if (kPacked) inside.move(p, tile0);
    const bool marked = kPacked && !inside.plain(tile0, kTile);
    if (marked) {
      mark_tile(p, tile0, mark[par]);
      __syncthreads();
    }
    // this thread's span from a zero state, both ways
    Span fwd = {one, both(0.f)}, back = fwd;
    auto ahead = [&](int j) {
      const Gate g = gate<false>(get2<T, V>(rr[j]), get2<T, V>(ir[j]), k);
      kept.sr[j][me] = g.sr;
      kept.si[j][me] = g.si;
      kept.u[j][me] = g.u;
      const f2 a = one_minus<false>(g.u), ms = mul2(sqrt2(rest<false>(g.u)), g.si);
      kept.ms[j][me] = ms;
      f2 b = mul2(ms, get2<T, V>(xr[j]));
      const int start = marked ? mark[par][at.token() + j].x : -1;
      if (kPacked && start >= 0) {
        if (p.h0) b = fma2(a, ldf<V>(p.h0 + (size_t)start * p.D + at.ch), b);
        fwd = {both(-1.f), b};
      } else {
        step<kPacked>(fwd, a, b);
      }
    };
    auto behind = [&](int j) {
      const f2 a = one_minus<false>(kept.u[j][me]);
      const int end = marked ? mark[par][at.token() + j].y : -1;
      if (kPacked && end >= 0) back = {both(-1.f), p.dhT ? ldf<V>(p.dhT + (size_t)end * p.D + at.ch) : both(0.f)};
      step<kPacked>(back, a, mul2(a, get2<T, V>(gr[j])));
    };
    if (full) {
#pragma unroll
      for (int j = 0; j < kTok; ++j) ahead(j);
#pragma unroll
      for (int j = kTok - 1; j >= 0; --j) behind(j);
    } else {
#pragma unroll
      for (int j = 0; j < kTok; ++j)
        if (j < left) ahead(j);
#pragma unroll
      for (int j = kTok - 1; j >= 0; --j)
        if (j < left) behind(j);
    }
    // the next round's gates are on their way while the spans are joined
    if (base >= round) fetch(tile0 - round);
    const Span fother = from_other_half(fwd), other = from_other_half(back);
    leave<false, kPacked>(fspans[par], at.warp, at.lane, at.half, fwd, fother);
    leave<true, kPacked>(spans[par], at.warp, at.lane, at.half, back, other);
    __syncthreads();
    if (p.nc > 1 && !exchange<true, kPacked>(p, spans[par], tiles[par], bars, lost, !lost.gone, par, phase, at.rank))
      lost.gone = 1;
    f2 q = fold<true, kPacked>(spans[par], tiles[par], at.lane, at.rank, p.nc, at.warp, carry);
    for (int w = 0; w < at.warp; ++w) h = over<kPacked>(fspans[par][w][at.lane], h);
    if (at.half) h = over<kPacked>(fother, h);
    else q = over<kPacked>(other, q);
    auto again = [&](int j) {
      const int start = marked ? mark[par][at.token() + j].x : -1;
      if (kPacked && start >= 0) h = p.h0 ? ldf<V>(p.h0 + (size_t)start * p.D + at.ch) : both(0.f);
      kept.before[j][me] = h;
      h = fma2(one_minus<false>(kept.u[j][me]), h, mul2(kept.ms[j][me], get2<T, V>(xr[j])));
    };
    const Rows<T> dx(p.dx, p.dx_ld, row0 + tile0, at.ch), dr(p.dr, p.dr_ld, row0 + tile0, at.ch),
        di(p.di, p.di_ld, row0 + tile0, at.ch);
    auto grads = [&](int j) {
      const int2 f = marked ? mark[par][at.token() + j] : make_int2(-1, -1);
      if (kPacked && f.y >= 0) q = p.dhT ? ldf<V>(p.dhT + (size_t)f.y * p.D + at.ch) : both(0.f);
      const f2 u = kept.u[j][me], sr = kept.sr[j][me], ms = kept.ms[j][me];
      const f2 a = one_minus<false>(u), t = log2_decay(k, sr), b = mul2(ms, get2<T, V>(xr[j]));
      const f2 g = add2(get2<T, V>(gr[j]), q), ag = mul2(a, g);
      // w / ln 2 = a g t (h_{t-1} - a b / (1 - a^2)): 0 where a is 1, for t and b are
      const f2 w = mul2(mul2(ag, t), sub2(kept.before[j][me], mul2(mul2(a, b), rcp2(rest<false>(u)))));
      sum = add2(sum, w);
      q = ag;
      put2<T, V>(dx[j], mul2(g, ms));
      put2<T, V>(dr[j], mul2(w, each(sr, [](float s) { return fmaf(s, -kLn2, kLn2); })));
      put2<T, V>(di[j], mul2(mul2(g, b), one_minus<false>(kept.si[j][me])));
      if (kPacked && p.dh0 && f.x >= 0) stf<V>(p.dh0 + (size_t)f.x * p.D + at.ch, q);
    };
    if (at.live) {
      if (full) {
#pragma unroll
        for (int j = 0; j < kTok; ++j) again(j);
#pragma unroll
        for (int j = kTok - 1; j >= 0; --j) grads(j);
      } else {
#pragma unroll
        for (int j = 0; j < kTok; ++j)
          if (j < left) again(j);
#pragma unroll
        for (int j = kTok - 1; j >= 0; --j)
          if (j < left) grads(j);
      }
      if (!kPacked && p.dh0 && tile0 + at.token() == 0) stf<V>(p.dh0 + (size_t)at.b * p.D + at.ch, q);
    }
    __syncwarp();
  }
  // sum of w over this CTA's tokens, the spans in order
  __syncthreads();
  kept.u[0][me] = sum;
  __syncthreads();
  const bool lead = at.warp == 0 && at.half == 0;
  if (lead) {
    sum = kept.u[0][at.lane];
    for (int w = 1; w < 2 * kWarps; ++w) sum = add2(sum, kept.u[0][w * kLanes + at.lane]);
  }
  leave_sum<V, kLanes>(p, at, lead, sum, joined);
  drain_exchange(p, bars, lost);
}

// ---- backward for bf16 rows on 16 bytes: tiles by TMA, as fwd_tma_kernel.  The results take the inputs'
// places in the stage, from where they are copied out while the next round runs on the other.
// 8 x 4096 tokens of 2048 channels: 232 us, 4.0 TB/s, 67 warp instructions for 32 elements; bound as the forward.
struct BwdMaps { TileMap x, r, i, dy, dx, dr, di; };
struct BwdTiles {
  __nv_bfloat16 in[2][4][kTileTma][kWide];  // r, i, x, dy; then dr, di, dx
  f2 si[kTok][kThreads];
};

template <bool kPacked>
__global__ void __launch_bounds__(kThreads, kBwdCtas) bwd_tma_kernel(const GP p, const __grid_constant__ BwdMaps maps) {
  using bf = __nv_bfloat16;
  extern __shared__ __align__(128) unsigned char dynamic[];
  BwdTiles &sm = *reinterpret_cast<BwdTiles *>(dynamic + ((128 - (tc::smem_u32(dynamic) & 127)) & 127));
  __shared__ Span fspans[2][kWarps][32], spans[2][kWarps][32], tiles[2][kCluster][32];
  __shared__ int2 mark[2][kPacked ? kTileTma : 1];
  __shared__ f2 joined[kCluster][32];
  __shared__ uint64_t bars[2], full[2];
  __shared__ Lost lost;
  const WidePlace at(p);
  const int me = threadIdx.x, first = at.warp * kTok;
  const int round = p.nc * kTileTma, nkept = (p.T + kKeep - 1) / kKeep;
  auto fetch = [&](int t, int s) {  // by one thread
    tc::mbar_expect_tx(&full[s], (uint32_t)sizeof(sm.in[s]) + (p.inject && at.rank == 0 ? 16 : 0));
    tc::tma_load_3d(sm.in[s][0], &maps.r, at.strip, t, at.b, &full[s]);
    tc::tma_load_3d(sm.in[s][1], &maps.i, at.strip, t, at.b, &full[s]);
    tc::tma_load_3d(sm.in[s][2], &maps.x, at.strip, t, at.b, &full[s]);
    tc::tma_load_3d(sm.in[s][3], &maps.dy, at.strip, t, at.b, &full[s]);
  };
  const int last = (p.T - 1) / round * round;
  int tile0 = last + at.rank * kTileTma;
  if (threadIdx.x == 0) {
    tc::mbar_init(&full[0], 1);
    tc::mbar_init(&full[1], 1);
    tc::mbar_init(&bars[0], 1);
    tc::mbar_init(&bars[1], 1);
    lost = {{0, 0}, 0, 0};
    tc::fence_mbar_init();
    fetch(tile0, 0);
  }
  const f2 k = rate<2>(p, at.ch), one = both(1.f);
  f2 carry = !kPacked && p.dhT ? ldf<2>(p.dhT + (size_t)at.b * p.D + at.ch) : both(0.f);
  f2 sum = both(0.f);
  pass_through<2, kPacked>(p, at, p.dhT, p.dh0);
  __syncthreads();
  if (p.nc > 1) tc::cluster_sync();  // the barriers are there, and every CTA of the cluster runs

  int par = 0;  // also the stage
  uint32_t phase = 0;
  Inside inside;
  int base = last, end;
  do {
    const int left = p.T - tile0 - first;
    f2 h = tile0 < p.T ? ldf<2>(p.chunks + ((size_t)at.b * nkept + tile0 / kKeep) * p.D + at.ch) : both(0.f);
    if (kPacked) inside.move(p, tile0);
    const bool marked = kPacked && !inside.plain(tile0, kTileTma);
    if (marked) {
      mark_tile<kTileTma>(p, tile0, mark[par]);
      __syncthreads();
    }
    if (!tc::mbar_wait(&full[par], phase, wait_limit(p))) {
      tell(p);
      lost.end[par] = INT_MAX;
    }
    auto cell = [&](int which, int j) { return &sm.in[par][which][first + j][at.lane * 2]; };
    auto word = [&](int which, int j) -> uint32_t & { return *reinterpret_cast<uint32_t *>(cell(which, j)); };
    // this thread's span from a zero state, both ways
    Span fwd = {one, both(0.f)}, back = fwd;
    f2 u[kTok], ms[kTok];
#pragma unroll
    for (int j = 0; j < kTok; ++j) {
      const Gate g = gate<true>(get2<bf, 2>(Pack<bf, 2>::ld(cell(0, j))), get2<bf, 2>(Pack<bf, 2>::ld(cell(1, j))), k);
      float lo, hi;  // sigmoid(r) stays in the two cells that it came from
      unpack2(g.sr, lo, hi);
      word(0, j) = __float_as_uint(lo);
      word(1, j) = __float_as_uint(hi);
      sm.si[j][me] = g.si;
      // (a token past the row's end changes nothing: a = 1, no input)
      u[j] = j < left ? g.u : both(0.f);
      ms[j] = mul2(sqrt2(rest<true>(u[j])), g.si);
      const f2 a = one_minus<true>(u[j]);
      f2 b = mul2(ms[j], get2<bf, 2>(Pack<bf, 2>::ld(cell(2, j))));
      const int start = marked ? mark[par][first + j].x : -1;
      if (kPacked && start >= 0) {
        if (p.h0) b = fma2(a, ldf<2>(p.h0 + (size_t)start * p.D + at.ch), b);
        fwd = {both(-1.f), b};
      } else {
        step<kPacked>(fwd, a, b);
      }
    }
#pragma unroll
    for (int j = kTok - 1; j >= 0; --j) {
      const f2 a = one_minus<true>(u[j]);
      const int end = marked ? mark[par][first + j].y : -1;
      if (kPacked && end >= 0) back = {both(-1.f), p.dhT ? ldf<2>(p.dhT + (size_t)end * p.D + at.ch) : both(0.f)};
      step<kPacked>(back, a, mul2(a, get2<bf, 2>(Pack<bf, 2>::ld(cell(3, j)))));
    }
    fspans[par][at.warp][at.lane] = fwd;
    spans[par][at.warp][at.lane] = back;
    if (at.lane == 0) tc::bulk_wait_read();  // the round before has left the other stage
    __syncthreads();
    end = lost.end[par];
    if (threadIdx.x == 0 && base >= round) fetch(tile0 - round, par ^ 1);
    __syncwarp();
    if (p.nc > 1 && !exchange<true, kPacked>(p, spans[par], tiles[par], bars, lost, true, par, phase, at.rank))
      lost.end[par ^ 1] = INT_MAX;
    f2 q = fold<true, kPacked>(spans[par], tiles[par], at.lane, at.rank, p.nc, at.warp, carry);
#pragma unroll 1
    for (int w = 0; w < at.warp; ++w) h = over<kPacked>(fspans[par][w][at.lane], h);
    f2 before[kTok];  // the state before each token
#pragma unroll
    for (int j = 0; j < kTok; ++j) {
      const int start = marked ? mark[par][first + j].x : -1;
      if (kPacked && start >= 0) h = p.h0 ? ldf<2>(p.h0 + (size_t)start * p.D + at.ch) : both(0.f);
      before[j] = h;
      h = fma2(one_minus<true>(u[j]), h, mul2(ms[j], get2<bf, 2>(Pack<bf, 2>::ld(cell(2, j)))));
    }
#pragma unroll
    for (int j = kTok - 1; j >= 0; --j) {
      const int2 f = marked ? mark[par][first + j] : make_int2(-1, -1);
      if (kPacked && f.y >= 0) q = p.dhT ? ldf<2>(p.dhT + (size_t)f.y * p.D + at.ch) : both(0.f);
      const f2 sr = pack2(__uint_as_float(word(0, j)), __uint_as_float(word(1, j)));
      const f2 a = one_minus<true>(u[j]), t = log2_decay(k, sr);
      const f2 b = mul2(ms[j], get2<bf, 2>(Pack<bf, 2>::ld(cell(2, j))));
      const f2 g = add2(get2<bf, 2>(Pack<bf, 2>::ld(cell(3, j))), q), ag = mul2(a, g);
      // w / ln 2 = a g t (h_{t-1} - a b / (1 - a^2)): 0 where a is 1, for t and b are
      const f2 w = mul2(mul2(ag, t), sub2(before[j], mul2(mul2(a, b), rcp2(rest<true>(u[j])))));
      if (j < left) sum = add2(sum, w);
      q = ag;
      put2<bf, 2>(cell(2, j), mul2(g, ms[j]));
      put2<bf, 2>(cell(0, j), mul2(w, each(sr, [](float s) { return fmaf(s, -kLn2, kLn2); })));
      put2<bf, 2>(cell(1, j), mul2(mul2(g, b), one_minus<true>(sm.si[j][me])));
      if (kPacked && p.dh0 && at.live && f.x >= 0) stf<2>(p.dh0 + (size_t)f.x * p.D + at.ch, q);
    }
    tc::fence_async_smem();
    __syncwarp();
    if (at.lane == 0 && left > 0) {  // (what is past the tensors' ends is left out)
      tc::tma_store_3d(&maps.dr, at.strip, tile0 + first, at.b, sm.in[par][0][first]);
      tc::tma_store_3d(&maps.di, at.strip, tile0 + first, at.b, sm.in[par][1][first]);
      tc::tma_store_3d(&maps.dx, at.strip, tile0 + first, at.b, sm.in[par][2][first]);
      tc::bulk_commit();
    }
    if (!kPacked && p.dh0 && at.live && tile0 + first == 0) stf<2>(p.dh0 + (size_t)at.b * p.D + at.ch, q);
    __syncwarp();
    base -= round;
    tile0 -= round;
    phase ^= par;
    par ^= 1;
  } while (base >= end);
  if (at.lane == 0) tc::bulk_wait_all();
  if (threadIdx.x == 0) {  // the last round's copies and, where the rounds were left, the next one's have come
    tc::mbar_wait(&full[par ^ 1], phase ^ (uint32_t)(par ^ 1), wait_limit(p));
    if (base >= 0) tc::mbar_wait(&full[par], phase, wait_limit(p));
  }
  // sum of w over this CTA's tokens, the warps in order
  __syncthreads();
  sm.si[0][me] = sum;
  __syncthreads();
  const bool lead = at.warp == 0;
  if (lead) {
    sum = sm.si[0][at.lane];
    for (int w = 1; w < kWarps; ++w) sum = add2(sum, sm.si[0][w * 32 + at.lane]);
  }
  leave_sum<2, 32>(p, at, lead, sum, joined);
  drain_exchange(p, bars, lost);
}

// dlam from the sums of the batch's rows, in order: 16 interleaved sums, joined in order.
__global__ void __launch_bounds__(512) dlam_kernel(const GP p) {
  __shared__ float sh[16][32];
  const int ch = blockIdx.x * 32 + threadIdx.x;
  float a = 0.f;
  if (ch < p.D)
    for (int q = threadIdx.y; q < p.B; q += 16) a += p.part[(size_t)q * p.D + ch];
  sh[threadIdx.y][threadIdx.x] = a;
  __syncthreads();
  if (threadIdx.y || ch >= p.D) return;
#pragma unroll
  for (int y = 1; y < 16; ++y) a += sh[y][threadIdx.x];
  p.dlam[ch] = dlam_of(p.lam[ch], a);
}

// A token of each request: a thread has a pair of channels.  256 requests of 4096 channels: 5.2 us, 3.1 TB/s of
// states and rows; bound by the launch and the slot's and the state's loads one after the other.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads) step_kernel(const GP p) {
  const int ch = (blockIdx.x * kThreads + threadIdx.x) * V;
  if (ch >= p.D) return;
  const f2 k = rate<V>(p, ch);
  for (int row = blockIdx.y; row < p.B; row += gridDim.y) {
    const int slot = p.slots ? p.slots[row] : row;
    f2 y = both(0.f);
    if (slot >= 0 && slot < p.num_slots) {
      float *h = p.h + (size_t)slot * p.D + ch;
      const f2 x = get2<T, V>(Pack<T, V>::ld(static_cast<const T *>(p.x) + row * p.x_ld + ch));
      const Gate g = gate<false>(get2<T, V>(Pack<T, V>::ld(static_cast<const T *>(p.r) + row * p.r_ld + ch)),
                                 get2<T, V>(Pack<T, V>::ld(static_cast<const T *>(p.i) + row * p.i_ld + ch)), k);
      y = fma2(one_minus<false>(g.u), ldf<V>(h), mul2(mul2(sqrt2(rest<false>(g.u)), g.si), x));
      stf<V>(h, y);
    }
    put2<T, V>(static_cast<T *>(p.y) + row * p.y_ld + ch, y);
  }
}

// CTAs of a cluster for `units` rows of strips: what fills the places of the GPU (95 % of them: clusters
// do not take every SM) in one go.  Where the units fill them by themselves, two that share a
// unit even out what the last ones leave idle, until there are twice as many units as places
// (512 units of 4096 tokens: forward 145 us with two, 168 with one; 1024 units of 700: 66 and 60).
int cluster_of(int T, long long units, bool bwd) {
  const int tiles = (T + kTile - 1) / kTile, places = 152 * (bwd ? kBwdCtas : kFwdCtas) * 95 / 100;
  const long long nc = units >= 2 * places ? 1 : units > places ? 2 : places / units;
  const int most = tiles < 1 ? 1 : tiles < kCluster ? tiles : kCluster;
  return nc < most ? (int)nc : most;
}
long long units_of(const rdn_gscan_args &a, int V) {
  return (long long)a.B * ((a.D + kLanes * V - 1) / (kLanes * V));
}

GP params(const rdn_gscan_args &a, int V, bool bwd) {
  GP p{};
  p.B = a.B; p.T = a.T; p.D = a.D; p.c = a.c;
  p.strips = (a.D + kLanes * V - 1) / (kLanes * V);
  p.nc = cluster_of(a.T, units_of(a, V), bwd);
  p.num_seqs = a.num_seqs; p.cu = a.cu_seqlens;
  p.x_ld = a.x_ld; p.r_ld = a.r_ld; p.i_ld = a.i_ld; p.y_ld = a.y_ld;
  p.dy_ld = a.dy_ld; p.dx_ld = a.dx_ld; p.dr_ld = a.dr_ld; p.di_ld = a.di_ld;
  p.x = a.x; p.r = a.r; p.i = a.i; p.dy = a.dy;
  p.lam = a.lam; p.h0 = a.h0; p.dhT = a.dhT;
  p.y = a.y; p.dx = a.dx; p.dr = a.dr; p.di = a.di;
  p.hT = a.hT; p.chunks = a.h_chunks; p.dh0 = a.dh0;
  p.status = status_word();
  p.inject = fault_injection() == (bwd ? 4 : 3);
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

// A launch of p.nc CTAs a cluster, with `bytes` of dynamic shared memory.
template <auto kKernel, typename... Args>
cudaError_t go(const GP &p, int bytes, const char *name, cudaStream_t s, const Args &...args) {
  cudaError_t e = bytes ? let_smem<kKernel>(bytes) : cudaSuccess;
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)((long long)p.B * p.strips * p.nc));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = s;
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = p.nc;
  at.val.clusterDim.y = at.val.clusterDim.z = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  RDN_LAUNCH(name, s, (e = cudaLaunchKernelEx(&cfg, kKernel, p, args...)));
  return e;
}
template <typename T, int V>
cudaError_t run(const GP &p, bool bwd, const char *name, cudaStream_t s) {
  if (bwd)
    return p.cu ? go<bwd_kernel<T, V, true>>(p, sizeof(Kept), name, s)
                : go<bwd_kernel<T, V, false>>(p, sizeof(Kept), name, s);
  return p.cu ? go<fwd_kernel<T, V, true>>(p, 0, name, s) : go<fwd_kernel<T, V, false>>(p, 0, name, s);
}
cudaError_t run(const GP &p, bool bwd, int dtype, int V, const char *name, cudaStream_t s) {
  if (dtype == RDN_BF16)
    return V == 2 ? run<__nv_bfloat16, 2>(p, bwd, name, s) : run<__nv_bfloat16, 1>(p, bwd, name, s);
  return V == 2 ? run<float, 2>(p, bwd, name, s) : run<float, 1>(p, bwd, name, s);
}

// Tensor maps over [B][T][D] bf16 rows of distance ld, boxes of 64 channels and `tokens` tokens.
bool make_tiles(TileMap *m, const void *p, const rdn_gscan_args &a, long long ld, int tokens) {
  return rdn::make_rows_map(m, p, a.D, a.T, a.B, ld, kWide, tokens);
}
// bf16, an even D, rows (pointers and distances) on 16 bytes, distances that a map can hold, and enough strips:
// the other kernels' are half as wide, and with few of them fill more of the GPU (32 strips of 32768 tokens
// 199 us by TMA, 173 without; 16 strips of 777 tokens 15.2 and 13.1; 40 strips of 4096 tokens 34 and 38).
bool tma_ok(const rdn_gscan_args &a, std::initializer_list<const void *> ptrs, std::initializer_list<long long> lds) {
  if (a.dtype != RDN_BF16 || (a.D & 1) || a.T < 1) return false;
  if ((long long)a.B * ((a.D + kWide - 1) / kWide) < kTmaUnits) return false;
  for (const void *q : ptrs)
    if ((uintptr_t)q & 15) return false;
  for (long long ld : lds)
    if ((ld * 2) & 15 || ld * 2 * a.T >= (1ll << 40)) return false;
  return true;
}
bool fwd_tma_ok(const rdn_gscan_args &a) {
  return tma_ok(a, {a.x, a.r, a.i, a.y}, {a.x_ld, a.r_ld, a.i_ld, a.y_ld});
}
bool bwd_tma_ok(const rdn_gscan_args &a) {
  return tma_ok(a, {a.x, a.r, a.i, a.dy, a.dx, a.dr, a.di},
                {a.x_ld, a.r_ld, a.i_ld, a.dy_ld, a.dx_ld, a.dr_ld, a.di_ld});
}
// Strips, and CTAs of a cluster: what fills 95 % of the places in one go, and no more: a round costs a CTA more
// in a cluster (forward, 256 units of 4096 tokens 129 us with one, 135 with two; 128 units 71 with three, 95
// with one; 64 units of 16384 tokens 138 us with six, 159 with five, 185 with three); of 8 few clusters find a
// place (the same 64 units, before the gates were worked out in pairs: 148 us with six, 183 with eight).
int tma_strips(const rdn_gscan_args &a) { return (a.D + kWide - 1) / kWide; }
int tma_cluster(const rdn_gscan_args &a, bool bwd) {
  const long long units = (long long)a.B * tma_strips(a), places = 152 * (bwd ? kBwdCtas : kFwdCtas) * 95 / 100;
  const long long tiles = (a.T + kTileTma - 1) / kTileTma, nc = units > places ? 1 : places / units;
  const long long most = tiles < 1 ? 1 : tiles < 6 ? tiles : 6;
  return (int)(nc < most ? nc : most);
}
GP tma_params(GP p, const rdn_gscan_args &a, bool bwd) {
  p.strips = tma_strips(a);
  p.nc = tma_cluster(a, bwd);
  return p;
}
cudaError_t run_fwd_tma(const rdn_gscan_args &a, cudaStream_t s) {
  FwdMaps m{};
  if (!make_tiles(&m.x, a.x, a, a.x_ld, kTileTma) || !make_tiles(&m.r, a.r, a, a.r_ld, kTileTma) ||
      !make_tiles(&m.i, a.i, a, a.i_ld, kTileTma) || (a.y && !make_tiles(&m.y, a.y, a, a.y_ld, kTok)))
    return cudaErrorInvalidValue;
  const GP p = tma_params(params(a, 2, false), a, false);
  constexpr int kBytes = sizeof(FwdTiles) + 128;  // (tiles on 128 bytes)
  return p.cu ? go<fwd_tma_kernel<true>>(p, kBytes, "gscan_fwd_tma", s, m)
              : go<fwd_tma_kernel<false>>(p, kBytes, "gscan_fwd_tma", s, m);
}
cudaError_t run_bwd_tma(const rdn_gscan_args &a, GP p, cudaStream_t s) {
  BwdMaps m{};
  if (!make_tiles(&m.x, a.x, a, a.x_ld, kTileTma) || !make_tiles(&m.r, a.r, a, a.r_ld, kTileTma) ||
      !make_tiles(&m.i, a.i, a, a.i_ld, kTileTma) || !make_tiles(&m.dy, a.dy, a, a.dy_ld, kTileTma) ||
      !make_tiles(&m.dx, a.dx, a, a.dx_ld, kTok) || !make_tiles(&m.dr, a.dr, a, a.dr_ld, kTok) ||
      !make_tiles(&m.di, a.di, a, a.di_ld, kTok))
    return cudaErrorInvalidValue;
  p = tma_params(p, a, true);
  constexpr int kBytes = sizeof(BwdTiles) + 128;
  return p.cu ? go<bwd_tma_kernel<true>>(p, kBytes, "gscan_bwd_tma", s, m)
              : go<bwd_tma_kernel<false>>(p, kBytes, "gscan_bwd_tma", s, m);
}

size_t part_bytes(const rdn_gscan_args &a) { return a.B > 1 ? round256(sizeof(float) * (size_t)a.B * a.D) : 0; }

}  // namespace gscan

long long gscan_slots(const rdn_gscan_args &a) {
  return (long long)a.B * ((a.T + gscan::kKeep - 1) / gscan::kKeep);
}
// CTAs of a call at one channel a lane, the most it may take.
long long gscan_ctas(const rdn_gscan_args &a) {
  return gscan::units_of(a, 1) * gscan::kCluster;
}
size_t gscan_bwd_bytes(const rdn_gscan_args &a) {
  const size_t states = a.h_chunks ? 0 : round256(sizeof(float) * (size_t)gscan_slots(a) * a.D);
  return gscan::part_bytes(a) + states;
}

cudaError_t launch_gscan_fwd(const rdn_gscan_args &a, cudaStream_t s) {
  const size_t e = a.dtype == RDN_BF16 ? 2 : 4;
  if (gscan::fwd_tma_ok(a)) return gscan::run_fwd_tma(a, s);
  const int V = gscan::pairs_ok(a.D, e, {a.x, a.r, a.i, a.y}, {a.x_ld, a.r_ld, a.i_ld, a.y_ld}) ? 2 : 1;
  return gscan::run(gscan::params(a, V, false), false, a.dtype, V, "gscan_fwd", s);
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
  gscan::GP p = gscan::params(c, V, true);
  p.part = static_cast<float *>(a.workspace);
  p.dlam = a.dlam;
  const cudaError_t e =
      gscan::bwd_tma_ok(c) ? gscan::run_bwd_tma(c, p, s) : gscan::run(p, true, a.dtype, V, "gscan_bwd", s);
  if (e != cudaSuccess || a.B == 1) return e;
  RDN_LAUNCH("gscan_dlam", s, (gscan::dlam_kernel<<<(a.D + 31) / 32, dim3(32, 16), 0, s>>>(p)));
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
