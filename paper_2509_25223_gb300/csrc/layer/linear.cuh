// linear.cuh -- what the matrix products of rdn_linear_* share: operands and their
// tensor maps, the tensor-core instructions in both element types and for one CTA
// or a pair, and the epilogue.
#pragma once
#include "launch.cuh"
#include "rows.cuh"
#include "status.cuh"
#include "tc_common.cuh"

namespace rdn {
namespace lin {

// An operand of a product: `rows` indexes of the result by `k` of the sum.  K-major: a row is
// k consecutive elements, rows ld apart; MN-major (transposed): stored [k][rows], ld between k.
struct Operand {
  const void *p;
  long long rows, k, ld;
  bool mn;
};

// The result's side of a product: out[m][n] = act(acc * xs[m] * ws[n] + bias[n]) + res[m][n].
struct Epilogue {
  const float *xs, *ws;
  const void *bias, *res;
  void *y;
  __nv_bfloat16 *pre;
  long long res_ld, y_ld, pre_ld;
  int act;                // 0 none, 1 SiLU, 2 sigmoid, 3 GELU
  int bias_f32, out_f32;  // element types (res as y)
};

struct GemmP {
  long long M, N;  // the result's rows and columns
  int kblocks, tiles_m, tiles_n, splits;
  Epilogue e;
  int *status;
  int inject;  // a test: the first tile's sums are not signalled
};
// A wait gives up after about a second, in a test sooner.
__device__ __forceinline__ long long wait_limit(const GemmP &p) { return p.inject ? 10000000ll : 2000000000ll; }

struct alignas(64) Map { unsigned char b[128]; };
struct Maps { Map a, b; };

// 128-byte wide boxes in the 128-byte swizzle: K-major `box` rows of 128 bytes of k, MN-major
// 64 k of 64 rows' elements.  Out of range reads as zero.
bool make_map(Map *m, const Operand &o, int elem, int box);

// The normal distribution function, with its own digits below zero too, where 1 + erf cancels (at -5 to 4 % of it, from
// -6 on to nothing): with a = |p|, that of -a is e^(-a^2 / 2) times a function of a that falls slowly, t Q(t) with
// t = 1 / (1 + 0.297 a) and the Q of degree 7 that has the least largest relative error for a <= 13.4 (the
// exponential is 0 beyond), fitted by reweighted least squares: 1.7e-7.  (erfcf spills 240 bytes a thread in tiles_kernel:
// 16384 x 4096 by 2048 with GELU 197 -> 258 us.)  e: the exponential.
__device__ __forceinline__ float normal_cdf(float p, float &e) {
  e = ex2(p * p * (-0.5f * kLog2e));
  const float t = rcp_approx(fmaf(fabsf(p), 0.29698485f, 1.f));
  float q = fmaf(3.5107624e-2f, t, -1.6009493e-1f);
  q = fmaf(q, t, 2.2027846e-1f);
  q = fmaf(q, t, -6.520926e-2f);
  q = fmaf(q, t, 1.3434237e-1f);
  q = fmaf(q, t, 9.737199e-2f);
  q = fmaf(q, t, 1.1979145e-1f);
  q = fmaf(q, t, 1.1841221e-1f);
  q = e * (t * q);
  return p < 0.f ? q : 1.f - q;
}
__device__ __forceinline__ float act_of(int act, float p) {
  float e;
  if (act == 1) return siluf(p);
  if (act == 2) return sigmoidf(p);
  if (act == 3) return p * normal_cdf(p, e);
  return p;
}
// The activation's derivative.
__device__ __forceinline__ float act_grad(int act, float p) {
  if (act == 0) return 1.f;
  if (act == 3) {
    float e;
    const float cdf = normal_cdf(p, e);
    return fmaf(p * 0.39894228f, e, cdf);
  }
  const float s = sigmoidf(p);
  return act == 2 ? s * (1.f - s) : s * fmaf(p, 1.f - s, 1.f);
}

// ---- tensor-core pieces for a CTA (kPair = false) or a pair of CTAs
template <bool kPair>
__device__ __forceinline__ void tma_2d(void *dst, const Map *map, int c0, int c1, uint32_t bar) {
  if constexpr (kPair)
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2"
        " [%0], [%1, {%2, %3}], [%4];" ::"r"(tc::smem_u32(dst)), "l"(map), "r"(c0), "r"(c1), "r"(bar)
        : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3}], [%4];" ::"r"(tc::smem_u32(dst)), "l"(map), "r"(c0), "r"(c1), "r"(bar)
        : "memory");
}

// D (+)= A B^T for one step of 32 bytes of k (16 bf16 or 32 e4m3), by one thread of the CTA
// (of the pair's first CTA).
template <bool kPair, bool kFp8>
__device__ __forceinline__ void mma_step(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
#define RDN_MMA(GROUP, KIND)                                                    \
  asm volatile(                                                                 \
      "{\n"                                                                     \
      ".reg .pred p;\n"                                                         \
      "setp.ne.b32 p, %4, 0;\n"                                                 \
      "tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], %1, %2, %3, p;\n"  \
      "}\n" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate)               \
      : "memory")
  if constexpr (kPair && kFp8) RDN_MMA("2", "f8f6f4");
  else if constexpr (kPair) RDN_MMA("2", "f16");
  else if constexpr (kFp8) RDN_MMA("1", "f8f6f4");
  else RDN_MMA("1", "f16");
#undef RDN_MMA
}
// Instruction descriptor: fp32 results; bf16 (format 1) or e4m3 (format 0) operands.
template <bool kFp8>
__host__ __device__ constexpr uint32_t idesc_of(int M, int N, bool a_mn, bool b_mn) {
  return (1u << 4) | (kFp8 ? 0u : (1u << 7) | (1u << 10)) | (a_mn ? tc::kAMajorMN : 0u) | (b_mn ? tc::kBMajorMN : 0u) |
         ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
// Arrives on `bar` (of a pair: of the CTAs in kTo) once this thread's products so far are done.
template <bool kPair, int kTo = 3>
__device__ __forceinline__ void commit(uint64_t *bar) {
  if constexpr (kPair)
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
            tc::smem_u32(bar)),
        "h"((uint16_t)kTo)
        : "memory");
  else
    tc::mma_commit(bar);
}
template <bool kPair>
__device__ __forceinline__ void tmem_alloc(uint32_t *slot, uint32_t cols) {
  if constexpr (kPair) {
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc::smem_u32(slot)), "r"(cols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  } else {
    tc::tmem_alloc(slot, cols);
  }
}
template <bool kPair>
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t cols) {
  if constexpr (kPair)
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols) : "memory");
  else
    tc::tmem_dealloc(addr, cols);
}

constexpr int kAtom = 64 * 128;  // bytes of 64 rows (K-major) or 64 k (MN-major) of 128 bytes
// The descriptor of an operand tile in shared memory, and its advance per 32 bytes of k (16 rows of an
// MN-major tile).
template <bool kMN>
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr) {
  return kMN ? tc::sdesc_sw128_mn(addr, kAtom) : tc::sdesc_sw128(addr);
}
template <bool kMN>
__device__ __forceinline__ uint64_t tile_step(int j) { return tc::desc_off(kMN ? 2048u * j : 32u * j); }

// One k block (128 bytes of k, K-major; 64 k, MN-major) of `rows` rows from row r0 of an operand.
template <bool kPair, bool kMN, bool kFp8, int kRows>
__device__ __forceinline__ void load_tile(unsigned char *dst, const Map *map, int r0, int kb, uint32_t bar) {
  if constexpr (kMN) {
#pragma unroll
    for (int q = 0; q < kRows / 64; ++q) tma_2d<kPair>(dst + q * kAtom, map, r0 + q * 64, kb * 64, bar);
  } else {
    tma_2d<kPair>(dst, map, kb * (kFp8 ? 128 : 64), r0, bar);
  }
}

cudaError_t run_tiles(const Operand &a, const Operand &b, GemmP p, bool fp8, cudaStream_t s);
cudaError_t run_split(const Operand &a, const Operand &b, GemmP p, bool fp8, cudaStream_t s);
// Whether run_split is the faster one.
bool split_fits(const Operand &a, const Operand &b, int kblocks);
// out = A B^T by the kernel that suits the sizes.
cudaError_t run_product(const Operand &a, const Operand &b, GemmP p, bool fp8, cudaStream_t s);

}  // namespace lin
}  // namespace rdn
