// rows.cuh -- pieces shared by the operators around the recurrence (conv.cu,
// scan.cu, scan_bwd.cu, norm.cu): vectors of consecutive elements, the
// activations and packed-sequence lookups.
#pragma once
#include "common.cuh"

namespace rdn {

// V consecutive elements, kept packed as loaded: one 16-byte access for
// V = 16 / sizeof(T), single elements for V = 1.
template <typename T, int V>
struct Pack;
template <>
struct Pack<float, 4> {
  using Raw = float4;
  __device__ static Raw zero() { return make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ static Raw ld(const float *p) { return *reinterpret_cast<const float4 *>(p); }
  __device__ static void get(const Raw &a, float (&v)[4]) {
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  }
  __device__ static Raw put(const float (&v)[4]) { return make_float4(v[0], v[1], v[2], v[3]); }
  __device__ static void st(float *p, const Raw &a) { *reinterpret_cast<float4 *>(p) = a; }
};
template <>
struct Pack<__nv_bfloat16, 8> {
  using Raw = uint4;
  __device__ static Raw zero() { return make_uint4(0u, 0u, 0u, 0u); }
  __device__ static Raw ld(const __nv_bfloat16 *p) { return *reinterpret_cast<const uint4 *>(p); }
  __device__ static void get(const Raw &a, float (&v)[8]) {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // a bf16 is the high half of its fp32
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  __device__ static Raw put(const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t *>(&b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ static void st(__nv_bfloat16 *p, const Raw &a) { *reinterpret_cast<uint4 *>(p) = a; }
};
template <>
struct Pack<__nv_bfloat16, 4> {
  using Raw = uint2;
  __device__ static Raw zero() { return make_uint2(0u, 0u); }
  __device__ static Raw ld(const __nv_bfloat16 *p) { return *reinterpret_cast<const uint2 *>(p); }
  __device__ static void get(const Raw &a, float (&v)[4]) {
    v[0] = __uint_as_float(a.x << 16);
    v[1] = __uint_as_float(a.x & 0xffff0000u);
    v[2] = __uint_as_float(a.y << 16);
    v[3] = __uint_as_float(a.y & 0xffff0000u);
  }
  __device__ static Raw put(const float (&v)[4]) {
    const __nv_bfloat162 lo = __floats2bfloat162_rn(v[0], v[1]), hi = __floats2bfloat162_rn(v[2], v[3]);
    return make_uint2(*reinterpret_cast<const uint32_t *>(&lo), *reinterpret_cast<const uint32_t *>(&hi));
  }
  __device__ static void st(__nv_bfloat16 *p, const Raw &a) { *reinterpret_cast<uint2 *>(p) = a; }
};
template <typename T>
struct Pack<T, 1> {
  using Raw = T;
  __device__ static Raw zero() { return from_f32<T>(0.f); }
  __device__ static Raw ld(const T *p) { return *p; }
  __device__ static void get(const Raw &a, float (&v)[1]) { v[0] = to_f32<T>(a); }
  __device__ static Raw put(const float (&v)[1]) { return from_f32<T>(v[0]); }
  __device__ static void st(T *p, const Raw &a) { *p = a; }
};
// elements of one 16-byte access
template <typename T>
constexpr int kVec = 16 / (int)sizeof(T);

constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Pairs of fp32 values in one register pair: one issue slot for two operations
// (the FMA pipe's rate is the same; the slots go to the exponentials and loads).
typedef unsigned long long f2;
__device__ __forceinline__ f2 pack2(float lo, float hi) {
  f2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpack2(f2 v, float &lo, float &hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
  f2 r;
  asm("fma.rn.ftz.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
  f2 r;
  asm("mul.rn.ftz.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
  f2 r;
  asm("add.rn.ftz.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float sum2(f2 v) {
  float lo, hi;
  unpack2(v, lo, hi);
  return lo + hi;
}

__device__ __forceinline__ float sigmoidf(float x) { return __fdividef(1.f, 1.f + __expf(-x)); }
__device__ __forceinline__ float siluf(float x) { return x * sigmoidf(x); }

// sigmoid and silu of a pair, and silu's derivative.  (The exponent is rounded: below zero the
// sigmoid's relative error is up to 7.3e-8 |x| + 7e-7.)
__device__ __forceinline__ f2 sigmoid2(f2 x) {
  float a, b;
  unpack2(mul2(x, pack2(-kLog2e, -kLog2e)), a, b);
  unpack2(add2(pack2(ex2(a), ex2(b)), pack2(1.f, 1.f)), a, b);
  return pack2(rcp_approx(a), rcp_approx(b));
}
__device__ __forceinline__ f2 silu2(f2 x) { return mul2(x, sigmoid2(x)); }
__device__ __forceinline__ f2 silu_grad2(f2 x) {
  const f2 s = sigmoid2(x), one = pack2(1.f, 1.f);
  return mul2(s, fma2(x, fma2(s, pack2(-1.f, -1.f), one), one));
}
// V elements as pairs (V = 1: with a zero)
template <int V>
__device__ __forceinline__ void to_pairs(const float (&v)[V], f2 (&p)[(V + 1) / 2]) {
#pragma unroll
  for (int e = 0; e < V; e += 2) p[e / 2] = pack2(v[e], e + 1 < V ? v[e + 1 < V ? e + 1 : e] : 0.f);
}
template <int V>
__device__ __forceinline__ void from_pairs(const f2 (&p)[(V + 1) / 2], float (&v)[V]) {
#pragma unroll
  for (int e = 0; e < V; e += 2) {
    float lo, hi;
    unpack2(p[e / 2], lo, hi);
    v[e] = lo;
    if (e + 1 < V) v[e + 1 < V ? e + 1 : e] = hi;
  }
}

// Packed sequences: token s of the offsets table, clamped into [0, T] (a table
// that breaks the ordering gives unspecified results, but stays in bounds).
__device__ __forceinline__ int cu_at(const int *cu, int num_seqs, int T, int s) {
  return s <= 0 ? 0 : s >= num_seqs ? T : min(max(__ldg(cu + s), 0), T);
}

// A sequence of a call: rows [begin, end) of its B * T token rows.
struct SeqSpan {
  int s;              // sequence: the row of the state tensors
  long long begin, end;
};
// The sequence that holds token t of batch row b (t < T): with a table, the
// last s with cu[s] <= t.
__device__ __forceinline__ SeqSpan find_seq(const int *cu, int num_seqs, int T, int b, int t) {
  if (!cu) return {b, (long long)b * T, (long long)(b + 1) * T};
  int lo = 0, hi = num_seqs - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (cu_at(cu, num_seqs, T, mid) <= t) lo = mid;
    else hi = mid - 1;
  }
  return {lo, cu_at(cu, num_seqs, T, lo), max(cu_at(cu, num_seqs, T, lo + 1), t + 1)};
}

inline size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }

}  // namespace rdn
