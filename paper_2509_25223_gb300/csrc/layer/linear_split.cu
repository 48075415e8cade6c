// linear_split.cu -- the matrix product of rdn_linear_* for results of few tiles: few tokens
// (the weights stream from HBM once), or few output channels.
// The roles are turned: rows of the tensor core's left operand (128 a tile) are the result's
// contiguous columns, so that a lane of the accumulator is a column and every store and
// load of the epilogue is coalesced; the result's rows (tokens) are the right operand, 16 to
// 128 a tile.  The sum over k is split over the CTAs of a cluster (up to 8), as many as
// fill the GPU; each leaves its sums in its own shared memory, and each then adds all
// the CTAs' sums, in order, for its share of the tile's rows, and finishes those.
// 1 row by 65536, K = 4096: 82 us, 6.5 TB/s of weights; 1 by 6144, K = 2048: 7.4 us, where launch, first copy, join
// and store follow one another.
#include "linear.cuh"

namespace rdn {
namespace lin {
namespace {

constexpr int kThreads = 256, kStageA = 128 * 128;

// (two CTAs on an SM: clusters of several do not take every SM, and what one waits for the other hides)
template <int kBN>
struct Smem {
  static constexpr int kStage = kStageA + kBN * 128;
  static constexpr int kStages = kBN <= 32 ? 5 : kBN == 64 ? 4 : 3;
  static constexpr int kBytes = 1024 + kStages * kStage;
  static_assert(kBN * 128 * 4 <= kStages * kStage, "the sums take the stages' place");
  static_assert(2 * (kBytes + 2048) <= 227 * 1024, "two CTAs an SM");
};

// 4 elements from p on: in one access where `vec`.
__device__ __forceinline__ void load4(float (&v)[4], const void *p, bool f32, bool vec) {
  if (f32) {
    const float *q = static_cast<const float *>(p);
    if (vec) Pack<float, 4>::get(Pack<float, 4>::ld(q), v);
    else
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = q[j];
  } else {
    const __nv_bfloat16 *q = static_cast<const __nv_bfloat16 *>(p);
    if (vec) Pack<__nv_bfloat16, 4>::get(Pack<__nv_bfloat16, 4>::ld(q), v);
    else
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = to_f32(q[j]);
  }
}
__device__ __forceinline__ void store4(void *p, const float (&v)[4], bool f32, bool vec) {
  if (f32) {
    float *q = static_cast<float *>(p);
    if (vec) Pack<float, 4>::st(q, Pack<float, 4>::put(v));
    else
#pragma unroll
      for (int j = 0; j < 4; ++j) q[j] = v[j];
  } else {
    __nv_bfloat16 *q = static_cast<__nv_bfloat16 *>(p);
    if (vec) Pack<__nv_bfloat16, 4>::st(q, Pack<__nv_bfloat16, 4>::put(v));
    else
#pragma unroll
      for (int j = 0; j < 4; ++j) q[j] = from_f32<__nv_bfloat16>(v[j]);
  }
}
__device__ __forceinline__ const void *at4(const void *p, long long i, bool f32) {
  return static_cast<const char *>(p) + i * (f32 ? 4 : 2);
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
               : "r"(addr)
               : "memory");
  return v;
}

// (A: columns of the result, p.N; B: its rows, p.M;  vec: rows of y, res allow accesses of 4 elements)
template <int kBN, bool kFp8, bool kAmn, bool kBmn>
__global__ void __launch_bounds__(kThreads, 2)
    split_kernel(const __grid_constant__ GemmP p, const __grid_constant__ Maps maps, int vec) {
  using S = Smem<kBN>;
  constexpr int kStages = S::kStages, kTmem = kBN < 32 ? 32 : kBN;
  extern __shared__ unsigned char raw[];
  __shared__ uint64_t full[kStages], empty[kStages], done, drained;
  __shared__ uint32_t slot;
  __shared__ int dead_;
  unsigned char *tiles = raw + ((1024 - (tc::smem_u32(raw) & 1023)) & 1023);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int q = blockIdx.x % p.splits, unit = blockIdx.x / p.splits;
  const int tn = unit % p.tiles_n, tm = unit / p.tiles_n;
  const int kb0 = (int)((long long)q * p.kblocks / p.splits), kb1 = (int)((long long)(q + 1) * p.kblocks / p.splits);
  auto copy = [&](int n) {  // this CTA's k block n
    const int s = n % kStages;
    unsigned char *at = tiles + s * S::kStage;
    tc::mbar_expect_tx(&full[s], S::kStage);
    load_tile<false, kAmn, kFp8, 128>(at, &maps.a, tn * 128, kb0 + n, tc::smem_u32(&full[s]));
    load_tile<false, kBmn, kFp8, kBN>(at + kStageA, &maps.b, tm * kBN, kb0 + n, tc::smem_u32(&full[s]));
  };
  const int count = kb1 - kb0;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      tc::mbar_init(&full[s], 1);
      tc::mbar_init(&empty[s], 1);
    }
    tc::mbar_init(&done, 1);
    tc::mbar_init(&drained, 1);
    dead_ = 0;
    tc::fence_mbar_init();
    for (int n = 0; n < min(count, kStages); ++n) copy(n);  // ahead of everything else
  }
  __syncwarp();
  if (warp == 1) tc::tmem_alloc(&slot, kTmem);
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = slot;
  volatile int *dead = &dead_;
  const long long limit = wait_limit(p);
  auto fail = [&] {
    *dead = 1;
    if (p.status) atomicExch(p.status, (int)RDN_ERR_TIMEOUT);
  };

  if (warp == 0) {
    if (lane == 0) {
      int n = min(count, kStages);
      for (; n < count; ++n) {
        if (!tc::mbar_wait(&empty[n % kStages], (uint32_t)(n / kStages + 1) & 1, limit)) fail();
        if (*dead) break;
        copy(n);
      }
      for (int c = n > kStages ? n - kStages : 0; c < n; ++c)  // every copy has landed
        if (!tc::mbar_wait(&full[c % kStages], (uint32_t)(c / kStages) & 1, limit)) fail();
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0) {
      constexpr uint32_t idesc = idesc_of<kFp8>(128, kBN, kAmn, kBmn);
      for (int n = 0; n < count; ++n) {
        const int s = n % kStages;
        if (!tc::mbar_wait(&full[s], (uint32_t)(n / kStages) & 1, limit)) fail();
        if (*dead) break;
        tc::fence_after_sync();
        const uint32_t at = tc::smem_u32(tiles + s * S::kStage);
        const uint64_t da = tile_desc<kAmn>(at), db = tile_desc<kBmn>(at + kStageA);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          mma_step<false, kFp8>(tmem, da + tile_step<kAmn>(j), db + tile_step<kBmn>(j), idesc, n + j > 0);
        tc::mma_commit(&empty[s]);
      }
      if (!p.inject) tc::mma_commit(&done);
      if (!tc::mbar_wait(&done, 0, limit)) {
        fail();
        tc::mma_commit(&drained);  // (the products are done all the same, or never)
        tc::mbar_wait(&drained, 0, limit);
      }
    }
    __syncwarp();
  }

  // what the sums meet: this lane's 4 columns, and the warp's first row of the residual
  const Epilogue &e = p.e;
  const long long n0 = (long long)tn * 128 + lane * 4;
  const bool in = n0 < p.N;  // (N is a multiple of 8)
  const int rows = (int)min((long long)kBN, p.M - (long long)tm * kBN);
  const int r0 = q * rows / p.splits + warp, r1 = (q + 1) * rows / p.splits;
  float sw[4] = {1.f, 1.f, 1.f, 1.f}, bias[4] = {0.f, 0.f, 0.f, 0.f}, res[4] = {0.f, 0.f, 0.f, 0.f};
  auto row_res = [&](int r) {
    if (e.res && r < r1) load4(res, at4(e.res, ((long long)tm * kBN + r) * e.res_ld + n0, e.out_f32), e.out_f32, vec);
  };
  if (in) {
    if (e.ws) load4(sw, e.ws + n0, true, false);
    if (e.bias) load4(bias, at4(e.bias, n0, e.bias_f32), e.bias_f32, false);
    row_res(r0);
  }
  __syncthreads();  // the products are done (or given up)
  tc::fence_after_sync();
  float *part = reinterpret_cast<float *>(tiles);  // [rows of the result][128 columns]
  if (warp >= 4) {
    const int quarter = warp & 3;
#pragma unroll
    for (int c = 0; c < kBN; c += 16) {
      if (c >= rows) break;
      float v[16];
      tc::tmem_ld16(tmem + ((uint32_t)(quarter * 32) << 16) + c, v);
#pragma unroll
      for (int j = 0; j < 16; ++j) part[(c + j) * 128 + quarter * 32 + lane] = v[j];
    }
    tc::fence_before_sync();
  }
  if (p.splits > 1) tc::cluster_sync();
  else __syncthreads();

  if (in && !*dead) {
    for (int r = r0; r < r1; r += kThreads / 32) {
      const long long m = (long long)tm * kBN + r;
      float4 w[8];
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k < p.splits) w[k] = ld_cluster4(tc::map_rank(part + r * 128 + lane * 4, k));
      float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < 8; ++k)  // in order
        if (k < p.splits) {
          v[0] += w[k].x; v[1] += w[k].y; v[2] += w[k].z; v[3] += w[k].w;
        }
      const float sx = e.ws ? e.xs[m] : 1.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = fmaf(v[j], sx * sw[j], bias[j]);
      if (e.pre) store4(e.pre + m * e.pre_ld + n0, v, false, true);
      if (e.act == 1) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = act_of(1, v[j]);
      } else if (e.act == 2) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = act_of(2, v[j]);
      } else if (e.act == 3) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = act_of(3, v[j]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] += res[j];
      row_res(r + kThreads / 32);
      store4(const_cast<void *>(at4(e.y, m * e.y_ld + n0, e.out_f32)), v, e.out_f32, vec);
    }
  }
  __syncwarp();
  // the others have read this CTA's sums (nothing that it wrote is waited for)
  if (p.splits > 1)
    asm volatile("barrier.cluster.arrive.relaxed.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
  if (warp == 1) tc::tmem_dealloc(tmem, kTmem);
}

template <int kBN, bool kFp8, bool kAmn, bool kBmn>
cudaError_t go(const Maps &maps, const GemmP &p, cudaStream_t s) {
  constexpr auto kern = split_kernel<kBN, kFp8, kAmn, kBmn>;
  cudaError_t e = let_smem<kern>(Smem<kBN>::kBytes);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)((long long)p.tiles_m * p.tiles_n * p.splits));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = Smem<kBN>::kBytes;
  cfg.stream = s;
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = p.splits;
  at.val.clusterDim.y = at.val.clusterDim.z = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  // rows on 4 elements
  const size_t by = p.e.out_f32 ? 16 : 8, el = p.e.out_f32 ? 4 : 2;
  auto on = [&](const void *q, long long ld) { return !q || (((uintptr_t)q | (ld * el)) & (by - 1)) == 0; };
  const int vec = on(p.e.y, p.e.y_ld) && on(p.e.res, p.e.res_ld);
  RDN_LAUNCH("linear_split", s, (e = cudaLaunchKernelEx(&cfg, kern, p, maps, vec)));
  return e;
}
template <int kBN>
cudaError_t pick(const Maps &maps, const GemmP &p, bool fp8, bool amn, bool bmn, cudaStream_t s) {
  if (fp8) return go<kBN, true, false, false>(maps, p, s);
  if constexpr (kBN >= 64) {
    if (bmn) return go<kBN, false, true, true>(maps, p, s);
  }
  return amn ? go<kBN, false, true, false>(maps, p, s) : go<kBN, false, false, false>(maps, p, s);
}

// Parts of the sum over k: as many as give an SM one CTA (a cluster needs SMs side by side, so fewer than 152 in
// all; 128 rows by 4096, K = 2048: four parts 8.6 us, five 10.2, seven 11.4; 256 by 1280: six 7.8, seven 10.0), or
// two, where the parts stay long and would be few (512 by 2048, K = 2048: two 12.1 us, four 10.9, five 16.2) or the
// tiles are narrow, so that one CTA's stages are too few bytes on their way (1 by 4096, K = 4096: four 9.2, six 8.2).
int splits_of(long long tiles, int kblocks, int bn) {
  const int most = (bn == 16 && kblocks >= 32) || tiles <= 8 ? 8 : 6;
  int one = 1, two = 1;
  for (int s = 2; s <= most && s <= kblocks; ++s) {
    if (tiles * s <= (s == 4 ? 144 : 136)) one = s;
    if (tiles * s <= (s <= 3 ? 288 : s == 6 ? 240 : 256)) two = s;
  }
  return kblocks >= 8 * one && (one < 4 || bn <= 32) ? two : one;
}

// Rows of a tile: all of them, at most 128 (an MN-major operand's boxes are 64 wide).
int rows_of(const Operand &a) {
  return a.rows <= 16 && !a.mn ? 16 : a.rows <= 32 && !a.mn ? 32 : a.rows <= 64 ? 64 : 128;
}

}  // namespace

// Up to 64 rows run_tiles multiplies mostly zeros (1 by 16384, K = 4096: 25.5 us here, 39 there; 64 by 16384 28.0 and
// 28.9).  Beyond, the join costs more than what it lets the SMs share unless the tiles are few or k is long (split
// and tiles: 1280 by 1024, 80 tiles, K = 512 9.1 and 7.0 us, 1024 10.2 and 9.5, 2048 12.4 and 14.0; 512 by 4096,
// 128 tiles, K = 2048 15.0 and 14.3, 4096 21.6 and 23.4; 1024 by 1024, 64 tiles, 512 7.8 and 7.1, 1024 9.3 and 9.4).
bool split_fits(const Operand &a, const Operand &b, int kblocks) {
  const long long tiles = (a.rows + 127) / 128 * ((b.rows + 127) / 128);
  return a.rows <= 64 || tiles <= (kblocks < 16 ? 48 : kblocks < 32 ? 64 : kblocks < 64 ? 96 : 128);
}

// (a holds the result's rows, b its columns, as for run_tiles)
cudaError_t run_split(const Operand &a, const Operand &b, GemmP p, bool fp8, cudaStream_t s) {
  const int bn = rows_of(a);
  p.tiles_m = (int)((p.M + bn - 1) / bn);
  p.tiles_n = (int)((p.N + 127) / 128);
  p.splits = splits_of((long long)p.tiles_m * p.tiles_n, p.kblocks, bn);
  Maps maps;
  if (!make_map(&maps.a, b, fp8 ? 1 : 2, 128) || !make_map(&maps.b, a, fp8 ? 1 : 2, bn))
    return cudaErrorInvalidValue;
  switch (bn) {
    case 16: return pick<16>(maps, p, fp8, b.mn, a.mn, s);
    case 32: return pick<32>(maps, p, fp8, b.mn, a.mn, s);
    case 64: return pick<64>(maps, p, fp8, b.mn, a.mn, s);
    default: return pick<128>(maps, p, fp8, b.mn, a.mn, s);
  }
}

}  // namespace lin
}  // namespace rdn
