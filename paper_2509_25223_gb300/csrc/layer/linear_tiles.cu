// linear_tiles.cu -- the matrix product of rdn_linear_* for results of many tiles.
// A pair of CTAs (two SMs) holds a tile of 256 x kBN of the result: each CTA 128 of its
// rows, with the rows of A it needs and half of B's, so that the pair's tensor cores
// (tcgen05.mma.cta_group::2) read each row of B from one of the two shared memories and
// a tile costs each SM as many shared-memory bytes as a 128 x 128 one.  Persistent CTAs
// walk over the tiles; one thread copies operand tiles (TMA, 128 bytes of k a stage), one
// thread of the pair issues the products, and eight warps of each CTA turn the previous
// tile's sums (TMEM, double buffered) into results meanwhile.
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

// 16 columns n.. of row m, from the sums v.
__device__ __forceinline__ void put16(const Epilogue &e, long long m, long long n, long long N, float sx, float (&v)[16],
                                      bool wide) {
  const bool two = n + 16 <= N;  // (N is a multiple of 8)
  if (e.ws) {
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] *= sx * (n + j < N ? __ldg(e.ws + n + j) : 0.f);
  }
  if (e.bias) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (h && !two) break;
      float b[8];
      if (e.bias_f32) {
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = __ldg(static_cast<const float *>(e.bias) + n + 8 * h + j);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = to_f32(__ldg(static_cast<const __nv_bfloat16 *>(e.bias) + n + 8 * h + j));
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) v[8 * h + j] += b[j];
    }
  }
  using P8 = Pack<__nv_bfloat16, 8>;
  using P4 = Pack<float, 4>;
  auto half = [&](int h, float (&o)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = v[8 * h + j];
  };
  if (e.pre) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (!h || two) {
        float o[8];
        half(h, o);
        P8::st(e.pre + m * e.pre_ld + n + 8 * h, P8::put(o));
      }
  }
  if (e.act) {
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = act_of(e.act, v[j]);
  }
  if (e.res) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (h && !two) break;
      if (!e.out_f32) {
        const __nv_bfloat16 *q = static_cast<const __nv_bfloat16 *>(e.res) + m * e.res_ld + n + 8 * h;
        float b[8];
        if (wide) {
          P8::get(P8::ld(q), b);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) b[j] = to_f32(q[j]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v[8 * h + j] += b[j];
      } else {
        const float *q = static_cast<const float *>(e.res) + m * e.res_ld + n + 8 * h;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[8 * h + j] += q[j];
      }
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (h && !two) break;
    float o[8];
    half(h, o);
    if (!e.out_f32) {
      __nv_bfloat16 *q = static_cast<__nv_bfloat16 *>(e.y) + m * e.y_ld + n + 8 * h;
      if (wide) {
        P8::st(q, P8::put(o));
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) q[j] = from_f32<__nv_bfloat16>(o[j]);
      }
    } else {
      float *q = static_cast<float *>(e.y) + m * e.y_ld + n + 8 * h;
      if (wide) {
        float a[4] = {o[0], o[1], o[2], o[3]}, b[4] = {o[4], o[5], o[6], o[7]};
        P4::st(q, P4::put(a));
        P4::st(q + 4, P4::put(b));
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) q[j] = o[j];
      }
    }
  }
}

template <int kBN, bool kFp8, bool kAmn, bool kBmn>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
    tiles_kernel(const __grid_constant__ GemmP p, const __grid_constant__ Maps maps, int wide) {
  using S = Smem<kBN>;
  constexpr int kStages = S::kStages;
  extern __shared__ unsigned char raw[];
  __shared__ Bars b;
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
  // A wait that gives up ends every role of the CTA at its next wait.
  auto fail = [&] {
    *dead = 1;
    if (p.status) atomicExch(p.status, (int)RDN_ERR_TIMEOUT);
  };

  if (warp == 0) {
    if (lane == 0) {
      long long n = 0;  // k blocks copied
      for (int t = pair; t < ntiles && !*dead; t += pairs) {
        int tm, tn;
        tile_at(p, t, tm, tn);
        for (int kb = 0; kb < p.kblocks; ++kb, ++n) {
          const int s = (int)(n % kStages);
          if (!tc::mbar_wait(&b.empty[s], (uint32_t)(n / kStages + 1) & 1)) fail();
          if (*dead) break;
          unsigned char *at = tiles + s * S::kStage;
          // both CTAs' copies complete on the first one's barrier
          const uint32_t bar = tc::map_rank(&b.full[s], 0);
          if (rank == 0) tc::mbar_expect_tx(&b.full[s], 2 * S::kStage);
          load_tile<true, kAmn, kFp8, 128>(at, &maps.a, tm * 256 + (int)rank * 128, kb, bar);
          load_tile<true, kBmn, kFp8, kBN / 2>(at + kStageA, &maps.b, tn * kBN + (int)rank * (kBN / 2), kb, bar);
        }
      }
      if (rank == 0)  // every copy has landed
        for (long long q = n > kStages ? n - kStages : 0; q < n; ++q)
          if (!tc::mbar_wait(&b.full[q % kStages], (uint32_t)(q / kStages) & 1)) fail();
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      constexpr uint32_t idesc = idesc_of<kFp8>(256, kBN, kAmn, kBmn);
      long long n = 0;
      int it = 0;
      for (int t = pair; t < ntiles && !*dead; t += pairs, ++it) {
        const int acc = it & 1;
        if (!tc::mbar_wait_cluster(&b.taken[acc], (uint32_t)(it / 2 + 1) & 1, 2000000000ll)) fail();
        if (*dead) break;
        tc::fence_after_sync();
        for (int kb = 0; kb < p.kblocks; ++kb, ++n) {
          const int s = (int)(n % kStages);
          if (!tc::mbar_wait(&b.full[s], (uint32_t)(n / kStages) & 1)) fail();
          if (*dead) break;
          tc::fence_after_sync();
          const uint32_t at = tc::smem_u32(tiles + s * S::kStage);
          const uint64_t da = tile_desc<kAmn>(at), db = tile_desc<kBmn>(at + kStageA);
#pragma unroll
          for (int j = 0; j < 4; ++j)
            mma_step<true, kFp8>(tmem + acc * kBN, da + tile_step<kAmn>(j), db + tile_step<kBmn>(j), idesc, kb + j > 0);
          commit<true>(&b.empty[s]);
        }
        if (!*dead) commit<true>(&b.done[acc]);
      }
      if (*dead) {
        commit<true>(&b.drained);
        tc::mbar_wait(&b.drained, 0);
      }
    }
    __syncwarp();
  } else {
    const int quarter = warp & 3, part = (warp - 2) >> 2;
    constexpr int kCols = kBN / 2;  // columns of a warp
    int it = 0;
    for (int t = pair; t < ntiles; t += pairs, ++it) {
      int tm, tn;
      tile_at(p, t, tm, tn);
      const int acc = it & 1;
      bool ok = !*dead;
      if (ok && !tc::mbar_wait(&b.done[acc], (uint32_t)(it / 2) & 1)) {
        fail();
        ok = false;
      }
      if (!__all_sync(0xffffffffu, ok)) break;
      tc::fence_after_sync();
      const long long m = (long long)tm * 256 + rank * 128 + quarter * 32 + lane;
      const float sx = p.e.xs && m < p.M ? p.e.xs[m] : 1.f;
      const long long n0 = (long long)tn * kBN + part * kCols;
      const uint32_t ta = tmem + ((uint32_t)(quarter * 32) << 16) + acc * kBN + part * kCols;
#pragma unroll 1
      for (int c = 0; c < kCols; c += 32) {
        float v0[16], v1[16];
        tc::tmem_ld16x2(ta + c, v0, ta + c + 16, v1);
        if (c + 32 == kCols) {  // the sums are in registers: the next tile but one may be summed up here
          tc::fence_before_sync();
          __syncwarp();
          if (lane == 0) tc::mbar_arrive_remote_relaxed(tc::map_rank(&b.taken[acc], 0));
        }
        if (m < p.M) {
          if (n0 + c < p.N) put16(p.e, m, n0 + c, p.N, sx, v0, wide);
          if (n0 + c + 16 < p.N) put16(p.e, m, n0 + c + 16, p.N, sx, v1, wide);
        }
        __syncwarp();
      }
    }
    __syncwarp();
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::cluster_sync();  // nothing of the pair is in flight or will arrive at the other CTA
  if (warp == 0) tmem_free<true>(tmem, 2 * kBN);
}

template <int kBN, bool kFp8, bool kAmn, bool kBmn>
cudaError_t go(const Maps &maps, const GemmP &p, bool wide, cudaStream_t s) {
  auto kern = tiles_kernel<kBN, kFp8, kAmn, kBmn>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<kBN>::kBytes);
  if (e != cudaSuccess) return e;
  const long long n = (long long)p.tiles_m * p.tiles_n;
  const int ctas = 2 * (int)(n < 76 ? n : 76);
  RDN_LAUNCH("linear_tiles", s, (kern<<<ctas, kThreads, Smem<kBN>::kBytes, s>>>(p, maps, wide)));
  return cudaGetLastError();
}
template <int kBN>
cudaError_t pick(const Maps &maps, const GemmP &p, bool fp8, bool amn, bool bmn, bool wide, cudaStream_t s) {
  if (fp8) return go<kBN, true, false, false>(maps, p, wide, s);
  if (amn) return go<kBN, false, true, true>(maps, p, wide, s);
  return bmn ? go<kBN, false, false, true>(maps, p, wide, s) : go<kBN, false, false, false>(maps, p, wide, s);
}

}  // namespace

cudaError_t run_tiles(const Operand &a, const Operand &b, GemmP p, bool fp8, cudaStream_t s) {
  // tiles of 256 x 128 where those of 256 x 256 would leave pairs of SMs idle
  p.tiles_m = (int)((p.M + 255) / 256);
  const int bn = (long long)p.tiles_m * ((p.N + 255) / 256) >= 60 ? 256 : 128;
  p.tiles_n = (int)((p.N + bn - 1) / bn);
  Maps maps;
  if (!make_map(&maps.a, a, fp8 ? 1 : 2, 128) || !make_map(&maps.b, b, fp8 ? 1 : 2, bn / 2)) return cudaErrorInvalidValue;
  const size_t e = p.e.out_f32 ? 4 : 2;
  const bool wide = (((uintptr_t)p.e.y | (uintptr_t)p.e.res | (p.e.y_ld * e) | (p.e.res ? p.e.res_ld * e : 0)) & 15) == 0;
  return bn == 256 ? pick<256>(maps, p, fp8, a.mn, b.mn, wide, s) : pick<128>(maps, p, fp8, a.mn, b.mn, wide, s);
}

}  // namespace lin
}  // namespace rdn
