// linear_split.cu -- the matrix product of rdn_linear_* for results of few tiles: few tokens
// (the weights stream from HBM once), or few output channels.
// The roles are turned: rows of the tensor core's left operand (128 a tile) are the result's
// contiguous columns, so that a lane of the accumulator is a column and every store and
// load of the epilogue is coalesced; the result's rows (tokens) are the right operand, 16 to
// 128 a tile.  The sum over k is split over the CTAs of a cluster (up to 8), as many as
// fill the GPU; each leaves its sums in its own shared memory, and each then adds all
// the CTAs' sums, in order, for its share of the tile's rows, and finishes those.
#include "linear.cuh"

namespace rdn {
namespace lin {
namespace {

constexpr int kThreads = 256, kStageA = 128 * 128;

template <int kBN>
struct Smem {
  static constexpr int kStage = kStageA + kBN * 128;
  static constexpr int kStages = kBN == 128 ? 6 : 8;
  static constexpr int kBytes = 1024 + kStages * kStage;
  static_assert(kBN * 128 * 4 <= kStages * kStage, "the sums take the stages' place");
};

// (A: columns of the result, p.N; B: its rows, p.M)
template <int kBN, bool kFp8, bool kAmn, bool kBmn>
__global__ void __launch_bounds__(kThreads, 1)
    split_kernel(const __grid_constant__ GemmP p, const __grid_constant__ Maps maps) {
  using S = Smem<kBN>;
  constexpr int kStages = S::kStages, kTmem = kBN < 32 ? 32 : kBN;
  extern __shared__ unsigned char raw[];
  __shared__ uint64_t full[kStages], empty[kStages], done;
  __shared__ uint32_t slot;
  __shared__ int dead_;
  unsigned char *tiles = raw + ((1024 - (tc::smem_u32(raw) & 1023)) & 1023);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int q = blockIdx.x % p.splits, unit = blockIdx.x / p.splits;
  const int tn = unit % p.tiles_n, tm = unit / p.tiles_n;
  const int kb0 = (int)((long long)q * p.kblocks / p.splits), kb1 = (int)((long long)(q + 1) * p.kblocks / p.splits);

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      tc::mbar_init(&full[s], 1);
      tc::mbar_init(&empty[s], 1);
    }
    tc::mbar_init(&done, 1);
    dead_ = 0;
    tc::fence_mbar_init();
  }
  __syncthreads();
  if (warp == 0) tc::tmem_alloc(&slot, kTmem);
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = slot;
  volatile int *dead = &dead_;
  auto fail = [&] {
    *dead = 1;
    if (p.status) atomicExch(p.status, (int)RDN_ERR_TIMEOUT);
  };

  if (warp == 0) {
    if (lane == 0) {
      int n = 0;
      for (int kb = kb0; kb < kb1; ++kb, ++n) {
        const int s = n % kStages;
        if (!tc::mbar_wait(&empty[s], (uint32_t)(n / kStages + 1) & 1)) fail();
        if (*dead) break;
        unsigned char *at = tiles + s * S::kStage;
        tc::mbar_expect_tx(&full[s], S::kStage);
        load_tile<false, kAmn, kFp8, 128>(at, &maps.a, tn * 128, kb, tc::smem_u32(&full[s]));
        load_tile<false, kBmn, kFp8, kBN>(at + kStageA, &maps.b, tm * kBN, kb, tc::smem_u32(&full[s]));
      }
      for (int c = n > kStages ? n - kStages : 0; c < n; ++c)  // every copy has landed
        if (!tc::mbar_wait(&full[c % kStages], (uint32_t)(c / kStages) & 1)) fail();
    }
    __syncwarp();
  } else if (warp == 1) {
    if (lane == 0) {
      constexpr uint32_t idesc = idesc_of<kFp8>(128, kBN, kAmn, kBmn);
      int n = 0;
      for (int kb = kb0; kb < kb1; ++kb, ++n) {
        const int s = n % kStages;
        if (!tc::mbar_wait(&full[s], (uint32_t)(n / kStages) & 1)) fail();
        if (*dead) break;
        tc::fence_after_sync();
        const uint32_t at = tc::smem_u32(tiles + s * S::kStage);
        const uint64_t da = tile_desc<kAmn>(at), db = tile_desc<kBmn>(at + kStageA);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          mma_step<false, kFp8>(tmem, da + tile_step<kAmn>(j), db + tile_step<kBmn>(j), idesc, n + j > 0);
        tc::mma_commit(&empty[s]);
      }
      tc::mma_commit(&done);
      if (!tc::mbar_wait(&done, 0)) fail();
    }
    __syncwarp();
  }
  __syncthreads();  // the products are done (or given up)
  tc::fence_after_sync();
  float *part = reinterpret_cast<float *>(tiles);  // [kBN rows of the result][128 columns]
  if (warp >= 4) {
    const int quarter = warp & 3;
#pragma unroll
    for (int c = 0; c < kBN; c += 16) {
      float v[16];
      tc::tmem_ld16(tmem + ((uint32_t)(quarter * 32) << 16) + c, v);
#pragma unroll
      for (int j = 0; j < 16; ++j) part[(c + j) * 128 + quarter * 32 + lane] = v[j];
    }
    tc::fence_before_sync();
  }
  if (p.splits > 1) tc::cluster_sync();
  else __syncthreads();

  const Epilogue &e = p.e;
  const int i = threadIdx.x & 127;
  const long long n = (long long)tn * 128 + i;
  const int r0 = q * kBN / p.splits, r1 = (q + 1) * kBN / p.splits;
  if (n < p.N && !*dead) {
    const float sw = e.ws ? e.ws[n] : 1.f;
    const float bias = !e.bias ? 0.f : e.bias_f32 ? static_cast<const float *>(e.bias)[n]
                                                  : to_f32(static_cast<const __nv_bfloat16 *>(e.bias)[n]);
    for (int r = r0 + (threadIdx.x >> 7); r < r1; r += 2) {
      const long long m = (long long)tm * kBN + r;
      if (m >= p.M) break;
      float v = 0.f;
      if (p.splits > 1) {
        float w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (k < p.splits)
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(w[k]) : "r"(tc::map_rank(part + r * 128 + i, k)) : "memory");
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (k < p.splits) v += w[k];
      } else {
        v = part[r * 128 + i];
      }
      if (e.ws) v *= e.xs[m] * sw;
      if (e.bias) v += bias;
      if (e.pre) e.pre[m * e.pre_ld + n] = from_f32<__nv_bfloat16>(v);
      v = act_of(e.act, v);
      if (e.out_f32) {
        if (e.res) v += static_cast<const float *>(e.res)[m * e.res_ld + n];
        static_cast<float *>(e.y)[m * e.y_ld + n] = v;
      } else {
        if (e.res) v += to_f32(static_cast<const __nv_bfloat16 *>(e.res)[m * e.res_ld + n]);
        static_cast<__nv_bfloat16 *>(e.y)[m * e.y_ld + n] = from_f32<__nv_bfloat16>(v);
      }
    }
  }
  __syncwarp();
  if (p.splits > 1) tc::cluster_sync();  // the others have read this CTA's sums
  else __syncthreads();
  if (warp == 0) tc::tmem_dealloc(tmem, kTmem);
}

template <int kBN, bool kFp8, bool kAmn, bool kBmn>
cudaError_t go(const Maps &maps, const GemmP &p, cudaStream_t s) {
  auto kern = split_kernel<kBN, kFp8, kAmn, kBmn>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<kBN>::kBytes);
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
  RDN_LAUNCH("linear_split", s, (e = cudaLaunchKernelEx(&cfg, kern, p, maps)));
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

}  // namespace

// (a holds the result's rows, b its columns, as for run_tiles)
cudaError_t run_split(const Operand &a, const Operand &b, GemmP p, bool fp8, cudaStream_t s) {
  // rows a tile: all of them, at most 128 (an MN-major operand's boxes are 64 wide)
  const int bn = p.M <= 16 && !a.mn ? 16 : p.M <= 32 && !a.mn ? 32 : p.M <= 64 ? 64 : 128;
  p.tiles_m = (int)((p.M + bn - 1) / bn);
  p.tiles_n = (int)((p.N + 127) / 128);
  const long long tiles = (long long)p.tiles_m * p.tiles_n;
  p.splits = 1;
  while (p.splits < 8 && tiles * (p.splits + 1) <= 152 && p.splits < p.kblocks) ++p.splits;
  Maps maps;
  if (!make_map(&maps.a, b, fp8 ? 1 : 2, 128) || !make_map(&maps.b, a, fp8 ? 1 : 2, bn)) return cudaErrorInvalidValue;
  switch (bn) {
    case 16: return pick<16>(maps, p, fp8, b.mn, a.mn, s);
    case 32: return pick<32>(maps, p, fp8, b.mn, a.mn, s);
    case 64: return pick<64>(maps, p, fp8, b.mn, a.mn, s);
    default: return pick<128>(maps, p, fp8, b.mn, a.mn, s);
  }
}

}  // namespace lin
}  // namespace rdn
