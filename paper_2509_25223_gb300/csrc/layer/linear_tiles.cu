// linear_tiles.cu -- the matrix product of rdn_linear_* for results of many tiles.
// A pair of CTAs (two SMs) holds a tile of 256 x kBN of the result: each CTA 128 of its
// rows, with the rows of A it needs and half of B's, so that the pair's tensor cores
// (tcgen05.mma.cta_group::2) read each row of B from one of the two shared memories and
// a tile costs each SM as many shared-memory bytes as a 128 x 128 one.  Persistent CTAs
// walk over the tiles; one thread copies operand tiles (TMA, 128 bytes of k a stage), one
// thread of the pair issues the products, and eight warps of each CTA turn the previous
// tile's sums (TMEM, double buffered) into results meanwhile.
// 8192 cubed 1.88 PF/s; 16384 x 4096 by 2048 1.78 alone, 1.55 with bias, SiLU, residual and `pre` (402 MB more);
// in 8 bits 3.0.  Bound by the tensor cores under the power limit, and by the copies: with half of them left out
// it takes 5 to 10 % less, with four stages for six 2 to 9 % more.
#include "linear.cuh"

namespace rdn {
namespace lin {
namespace {

constexpr int kEpiWarps = 8, kThreads = 64 + 32 * kEpiWarps;
constexpr int kStageA = 128 * 128;

template <int kBN>
struct Smem {
  static constexpr int kStageB = kBN / 2 * 128, kStage = kStageA + kStageB;
  static constexpr int kStages = kBN == 256 ? 6 : 8;
  static constexpr int kBytes = 1024 + kStages * kStage;  // (tiles on 1024 bytes)
};

// A place in the ring of stages, and the parity of its use.
template <int kStages>
struct Ring {
  int s = 0;
  uint32_t phase = 0;
  __device__ void next() {
    if (++s == kStages) {
      s = 0;
      phase ^= 1;
    }
  }
};

struct Bars {
  uint64_t full[8], empty[8], done[2], taken[2], drained;
  uint32_t tmem;
  int dead;
};

// Tiles in groups of 8 rows of tiles, a column of the group after the other: the tiles at work
// at one time share few operand rows in L2.
__device__ __forceinline__ void tile_at(const GemmP &p, int t, int &tm, int &tn) {
  const int per = 8 * p.tiles_n, g = t / per, r = t - g * per;
  const int rows = min(8, p.tiles_m - g * 8);
  tn = r / rows;
  tm = g * 8 + r - tn * rows;
}

// ---- the epilogue: 32 columns of a lane's row at a time.  A lane reads and writes whole 32-byte
// sectors of its row where rows allow it (kSectors), 16 bytes or single elements else.
enum Access { kSingle = 0, kVectors = 1, kSectors = 2 };
struct alignas(32) U8 { uint32_t w[8]; };
__device__ __forceinline__ U8 ld32(const void *p) {
  U8 v;
  asm volatile("ld.global.L1::no_allocate.L2::evict_first.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(v.w[0]), "=r"(v.w[1]), "=r"(v.w[2]), "=r"(v.w[3]), "=r"(v.w[4]), "=r"(v.w[5]), "=r"(v.w[6]),
                 "=r"(v.w[7])
               : "l"(p));
  return v;
}
__device__ __forceinline__ void st32(void *p, const U8 &v) {
  asm volatile("st.global.L1::no_allocate.L2::evict_first.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p),
               "r"(v.w[0]), "r"(v.w[1]), "r"(v.w[2]), "r"(v.w[3]), "r"(v.w[4]), "r"(v.w[5]), "r"(v.w[6]), "r"(v.w[7])
               : "memory");
}

// 32 elements of a row, `cols` of them (a multiple of 8) there, as loaded.
template <typename T>
struct Row32 {
  static constexpr int kPer = 32 / sizeof(T), kN = 32 / kPer;  // elements of a U8, U8s of a row
  U8 v[kN];
  __device__ void load(const T *p, int cols, int access) {
    if (access == kSectors && cols >= 32) {
#pragma unroll
      for (int k = 0; k < kN; ++k) v[k] = ld32(p + k * kPer);
      return;
    }
#pragma unroll
    for (int k = 0; k < kN; ++k)
#pragma unroll
      for (int h = 0; h < 2; ++h) {  // 16 bytes each
        const int at = (2 * k + h) * (kPer / 2);
        uint4 u = make_uint4(0u, 0u, 0u, 0u);
        if (at < cols) {
          if (access != kSingle) {
            u = *reinterpret_cast<const uint4 *>(p + at);
          } else {
            float e[kPer / 2];
#pragma unroll
            for (int j = 0; j < kPer / 2; ++j) e[j] = to_f32<T>(p[at + j]);
            const auto w = Pack<T, kPer / 2>::put(e);
            u = *reinterpret_cast<const uint4 *>(&w);
          }
        }
        v[k].w[4 * h] = u.x; v[k].w[4 * h + 1] = u.y; v[k].w[4 * h + 2] = u.z; v[k].w[4 * h + 3] = u.w;
      }
  }
  __device__ void store(T *p, int cols, int access) const {
    if (access == kSectors && cols >= 32) {
#pragma unroll
      for (int k = 0; k < kN; ++k) st32(p + k * kPer, v[k]);
      return;
    }
#pragma unroll
    for (int k = 0; k < kN; ++k)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int at = (2 * k + h) * (kPer / 2);
        if (at >= cols) continue;
        const uint4 u = make_uint4(v[k].w[4 * h], v[k].w[4 * h + 1], v[k].w[4 * h + 2], v[k].w[4 * h + 3]);
        if (access != kSingle) {
          *reinterpret_cast<uint4 *>(p + at) = u;
        } else {
          float e[kPer / 2];
          typename Pack<T, kPer / 2>::Raw w;
          *reinterpret_cast<uint4 *>(&w) = u;
          Pack<T, kPer / 2>::get(w, e);
#pragma unroll
          for (int j = 0; j < kPer / 2; ++j) p[at + j] = from_f32<T>(e[j]);
        }
      }
  }
  __device__ void add_to(float (&o)[32]) const {
#pragma unroll
    for (int k = 0; k < kN; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if constexpr (sizeof(T) == 4) {
          o[8 * k + j] += __uint_as_float(v[k].w[j]);
        } else {
          o[16 * k + 2 * j] += __uint_as_float(v[k].w[j] << 16);
          o[16 * k + 2 * j + 1] += __uint_as_float(v[k].w[j] & 0xffff0000u);
        }
      }
  }
  __device__ void round_from(const float (&o)[32]) {
#pragma unroll
    for (int k = 0; k < kN; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if constexpr (sizeof(T) == 4) {
          v[k].w[j] = __float_as_uint(o[8 * k + j]);
        } else {
          const __nv_bfloat162 b = __floats2bfloat162_rn(o[16 * k + 2 * j], o[16 * k + 2 * j + 1]);
          v[k].w[j] = *reinterpret_cast<const uint32_t *>(&b);
        }
      }
  }
};

template <int kAct>
__device__ __forceinline__ void act32(float (&v)[32]) {
#pragma unroll
  for (int j = 0; j < 32; ++j) v[j] = act_of(kAct, v[j]);
}

// A warp's 32 rows x kCols columns from column n0 on; cols: [0] scales and [1] biases of its columns.
// A bf16 residual is loaded a chunk ahead (r: the first chunk's); fp32 ones would not leave registers.
template <typename T, int kCols, typename Taken>
__device__ __forceinline__ void finish(const GemmP &p, uint32_t ta, long long m, long long n0, float sx,
                                       const float (*cols)[kCols], Row32<__nv_bfloat16> r, int res_access, int y_access,
                                       int pre_access, Taken taken) {
  constexpr bool kAhead = sizeof(T) == 2;
  const Epilogue &e = p.e;
  const bool live = m < p.M;
  const T *res = e.res ? static_cast<const T *>(e.res) + m * e.res_ld + n0 : nullptr;
  T *y = static_cast<T *>(e.y) + m * e.y_ld + n0;
  __nv_bfloat16 *pre = e.pre ? e.pre + m * e.pre_ld + n0 : nullptr;
#pragma unroll 1
  for (int c = 0; c < kCols; c += 32) {
    const int left = (int)min((long long)32, p.N - n0 - c);  // columns of the chunk that exist
    float v[32];
    {
      float a[16], b[16];
      tc::tmem_ld16x2(ta + c, a, ta + c + 16, b);
#pragma unroll
      for (int j = 0; j < 16; ++j) { v[j] = a[j]; v[16 + j] = b[j]; }
    }
    if (c + 32 == kCols) taken();
    Row32<__nv_bfloat16> next;
    if constexpr (kAhead)
      if (res && live && c + 32 < kCols && p.N - n0 > c + 32)
        next.load(res + c + 32, (int)min((long long)32, p.N - n0 - c - 32), res_access);
    if (e.ws) {
#pragma unroll
      for (int j = 0; j < 32; j += 4) {
        const float4 s = *reinterpret_cast<const float4 *>(&cols[0][c + j]);
        v[j] *= sx * s.x; v[j + 1] *= sx * s.y; v[j + 2] *= sx * s.z; v[j + 3] *= sx * s.w;
      }
    }
    if (e.bias) {
#pragma unroll
      for (int j = 0; j < 32; j += 4) {
        const float4 s = *reinterpret_cast<const float4 *>(&cols[1][c + j]);
        v[j] += s.x; v[j + 1] += s.y; v[j + 2] += s.z; v[j + 3] += s.w;
      }
    }
    if (live && left > 0) {
      if (pre) {
        Row32<__nv_bfloat16> o;
        o.round_from(v);
        o.store(pre + c, left, pre_access);
      }
      if (e.act == 1) act32<1>(v);
      else if (e.act == 2) act32<2>(v);
      else if (e.act == 3) act32<3>(v);
      if (res) {
        if constexpr (kAhead) {
          r.add_to(v);
        } else {
          Row32<T> now;
          now.load(res + c, left, res_access);
          now.add_to(v);
        }
      }
      Row32<T> o;
      o.round_from(v);
      o.store(y + c, left, y_access);
    }
    if constexpr (kAhead) r = next;
    __syncwarp();
  }
}

template <int kBN, bool kFp8, bool kAmn, bool kBmn>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    tiles_kernel(const __grid_constant__ GemmP p, const __grid_constant__ Maps maps, int res_access, int y_access,
                 int pre_access) {
  using S = Smem<kBN>;
  constexpr int kStages = S::kStages;
  constexpr int kCols = kBN / 2;  // columns of an epilogue warp
  extern __shared__ unsigned char raw[];
  __shared__ Bars b;
  __shared__ alignas(16) float cols[kEpiWarps][2][kCols];
  unsigned char *tiles = raw + ((1024 - (tc::smem_u32(raw) & 1023)) & 1023);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = tc::cluster_rank();
  const int pairs = gridDim.x / 2, pair = blockIdx.x / 2, ntiles = p.tiles_m * p.tiles_n;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      tc::mbar_init(&b.full[s], 1);
      tc::mbar_init(&b.empty[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      tc::mbar_init(&b.done[s], 1);
      tc::mbar_init(&b.taken[s], 2 * kEpiWarps);
    }
    tc::mbar_init(&b.drained, 1);
    b.dead = 0;
    tc::fence_mbar_init();
  }
  __syncthreads();
  if (warp == 0) tmem_alloc<true>(&b.tmem, 2 * kBN);
  tc::fence_before_sync();
  __syncthreads();
  tc::cluster_sync();  // both CTAs' barriers and tensor memory are there
  tc::fence_after_sync();
  const uint32_t tmem = b.tmem;
  volatile int *dead = &b.dead;
  const uint32_t full0 = tc::map_rank(&b.full[0], 0);
  const long long limit = wait_limit(p);
  // A wait that gives up ends every role of the CTA at its next wait.
  auto fail = [&] {
    *dead = 1;
    if (p.status) atomicExch(p.status, (int)RDN_ERR_TIMEOUT);
  };

  if (warp == 0) {
    if (lane == 0) {
      Ring<kStages> at;
      long long n = 0;  // k blocks copied
      for (int t = pair; t < ntiles && !*dead; t += pairs) {
        int tm, tn;
        tile_at(p, t, tm, tn);
        const int ra = tm * 256 + (int)rank * 128, rb = tn * kBN + (int)rank * (kBN / 2);
        for (int kb = 0; kb < p.kblocks; ++kb, at.next(), ++n) {
          if (!tc::mbar_wait(&b.empty[at.s], at.phase ^ 1, limit)) fail();
          if (*dead) break;
          unsigned char *to = tiles + at.s * S::kStage;
          // both CTAs' copies complete on the first one's barrier
          if (rank == 0) tc::mbar_expect_tx(&b.full[at.s], 2 * S::kStage);
          const uint32_t bar = full0 + at.s * 8;
          load_tile<true, kAmn, kFp8, 128>(to, &maps.a, ra, kb, bar);
          load_tile<true, kBmn, kFp8, kBN / 2>(to + kStageA, &maps.b, rb, kb, bar);
        }
      }
      if (rank == 0)  // every copy has landed
        for (long long q = n > kStages ? n - kStages : 0; q < n; ++q)
          if (!tc::mbar_wait(&b.full[q % kStages], (uint32_t)(q / kStages) & 1, limit)) fail();
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      constexpr uint32_t idesc = idesc_of<kFp8>(256, kBN, kAmn, kBmn);
      const uint64_t da0 = tile_desc<kAmn>(tc::smem_u32(tiles)), db0 = tile_desc<kBmn>(tc::smem_u32(tiles) + kStageA);
      Ring<kStages> at;
      int it = 0;
      for (int t = pair; t < ntiles && !*dead; t += pairs, ++it) {
        const int acc = it & 1;
        if (!tc::mbar_wait_cluster(&b.taken[acc], (uint32_t)(it / 2 + 1) & 1, limit)) fail();
        if (*dead) break;
        tc::fence_after_sync();
        for (int kb = 0; kb < p.kblocks; ++kb, at.next()) {
          if (!tc::mbar_wait(&b.full[at.s], at.phase, limit)) {
            fail();
            break;
          }
          tc::fence_after_sync();
          const uint64_t to = tc::desc_off((uint32_t)(at.s * S::kStage));
#pragma unroll
          for (int j = 0; j < 4; ++j)
            mma_step<true, kFp8>(tmem + acc * kBN, da0 + to + tile_step<kAmn>(j), db0 + to + tile_step<kBmn>(j), idesc,
                                 kb + j > 0);
          commit<true>(&b.empty[at.s]);
        }
        if (!*dead && !(p.inject && it == 0)) commit<true>(&b.done[acc]);
      }
      // every product is done, whatever the others have given up meanwhile
      commit<true, 1>(&b.drained);
      if (!tc::mbar_wait(&b.drained, 0, limit)) fail();
    }
    __syncwarp();
  } else {
    const int quarter = warp & 3, part = (warp - 2) >> 2;
    float(*mine)[kCols] = cols[warp - 2];
    int it = 0;
    for (int t = pair; t < ntiles; t += pairs, ++it) {
      int tm, tn;
      tile_at(p, t, tm, tn);
      const int acc = it & 1;
      const long long m = (long long)tm * 256 + rank * 128 + quarter * 32 + lane;
      const long long n0 = (long long)tn * kBN + part * kCols;
      // what the sums meet is fetched before they are waited for
      const float sx = p.e.xs && m < p.M ? p.e.xs[m] : 1.f;
      for (int c = lane; c < kCols; c += 32) {
        const bool in = n0 + c < p.N;
        if (p.e.ws) mine[0][c] = in ? p.e.ws[n0 + c] : 0.f;
        if (p.e.bias)
          mine[1][c] = !in ? 0.f : p.e.bias_f32 ? static_cast<const float *>(p.e.bias)[n0 + c]
                                                : to_f32(static_cast<const __nv_bfloat16 *>(p.e.bias)[n0 + c]);
      }
      Row32<__nv_bfloat16> rb;
      const int have = (int)max(0ll, min((long long)32, p.N - n0));
      if (p.e.res && !p.e.out_f32 && m < p.M && have)
        rb.load(static_cast<const __nv_bfloat16 *>(p.e.res) + m * p.e.res_ld + n0, have, res_access);
      __syncwarp();
      bool ok = !*dead;
      if (ok && !tc::mbar_wait(&b.done[acc], (uint32_t)(it / 2) & 1, limit)) {
        fail();
        ok = false;
      }
      if (!__all_sync(0xffffffffu, ok)) break;
      tc::fence_after_sync();
      const uint32_t ta = tmem + ((uint32_t)(quarter * 32) << 16) + acc * kBN + part * kCols;
      auto taken = [&] {  // the sums are in registers: the next tile but one may be summed up in their place
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive_remote_relaxed(tc::map_rank(&b.taken[acc], 0));
      };
      if (p.e.out_f32) finish<float, kCols>(p, ta, m, n0, sx, mine, rb, res_access, y_access, pre_access, taken);
      else finish<__nv_bfloat16, kCols>(p, ta, m, n0, sx, mine, rb, res_access, y_access, pre_access, taken);
    }
    __syncwarp();
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::cluster_sync();  // nothing of the pair is in flight or will arrive at the other CTA
  if (warp == 0) tmem_free<true>(tmem, 2 * kBN);
}

// Rows (pointer and distance in bytes) on 32 bytes, 16 bytes or neither.
int access_of(const void *p, long long bytes) {
  const uintptr_t v = (uintptr_t)p | (uintptr_t)bytes;
  return v % 32 == 0 ? kSectors : v % 16 == 0 ? kVectors : kSingle;
}

template <int kBN, bool kFp8, bool kAmn, bool kBmn>
cudaError_t go(const Maps &maps, const GemmP &p, cudaStream_t s) {
  constexpr auto kern = tiles_kernel<kBN, kFp8, kAmn, kBmn>;
  cudaError_t e = let_smem<kern>(Smem<kBN>::kBytes);
  if (e != cudaSuccess) return e;
  const long long n = (long long)p.tiles_m * p.tiles_n;
  const int ctas = 2 * (int)(n < 76 ? n : 76);
  const size_t e_size = p.e.out_f32 ? 4 : 2;
  const int res = access_of(p.e.res, p.e.res_ld * e_size), y = access_of(p.e.y, p.e.y_ld * e_size);
  const int pre = access_of(p.e.pre, p.e.pre_ld * 2);
  RDN_LAUNCH("linear_tiles", s, (kern<<<ctas, kThreads, Smem<kBN>::kBytes, s>>>(p, maps, res, y, pre)));
  return cudaGetLastError();
}
template <int kBN>
cudaError_t pick(const Maps &maps, const GemmP &p, bool fp8, bool amn, bool bmn, cudaStream_t s) {
  if (fp8) return go<kBN, true, false, false>(maps, p, s);
  if (amn) return go<kBN, false, true, true>(maps, p, s);
  return bmn ? go<kBN, false, false, true>(maps, p, s) : go<kBN, false, false, false>(maps, p, s);
}

}  // namespace

cudaError_t run_tiles(const Operand &a, const Operand &b, GemmP p, bool fp8, cudaStream_t s) {
  // tiles of 256 x 128 where every pair of SMs has at most one of them (512 x 4096 by 2048: 14.4 us, of 256 x 256
  // 14.7); two rounds of them take longer than one of 256 x 256 (1024 x 4096: 23.9 and 15.4)
  p.tiles_m = (int)((p.M + 255) / 256);
  const int bn = (long long)p.tiles_m * ((p.N + 127) / 128) > 76 ? 256 : 128;
  p.tiles_n = (int)((p.N + bn - 1) / bn);
  Maps maps;
  if (!make_map(&maps.a, a, fp8 ? 1 : 2, 128) || !make_map(&maps.b, b, fp8 ? 1 : 2, bn / 2))
    return cudaErrorInvalidValue;
  return bn == 256 ? pick<256>(maps, p, fp8, a.mn, b.mn, s) : pick<128>(maps, p, fp8, a.mn, b.mn, s);
}

}  // namespace lin
}  // namespace rdn
