// Softmax statistics of a row of logits, gathered in any order of parts (internal; token_logprobs.cu, lm_logprobs.cu).
//
// With a reference m (here the largest logit seen) and t_i = (x_i - m) log2(e) / T for logits x at temperature T:
//   S = sum 2^t_i,  A = sum t_i 2^t_i;
//   log p_i = (x_i - m) / T - ln S,  entropy = -sum p_i log p_i = ln S - (A / S) ln 2 (two terms >= 0, no cancellation).
// The difference comes before the scale: it is exact near the reference, and a logit of the type's lowest value overflows
// to -inf at most, never the other way.  Both sums and their merges are in 32 bits; a change of reference by d (in t) is
// S -> 2^d S, A -> 2^d (A + d S).  A part that has seen no number has m = -inf, S = A = 0.  Exponents are kept at -200 and
// above, where 2^t is 0 in 32 bits, so that a logit of -inf adds 0 to both; NaN and +inf make S NaN.
#pragma once

#include <cuda_runtime.h>

#include "ptd_device.cuh"

namespace ptd {

constexpr float kLeastExponent = -200.f;
constexpr float kLn2 = 0.693147180559945309f;

struct RowSums {
  float ref, s, a;
};

// max that keeps NaN
__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}

__device__ __forceinline__ RowSums merge_sums(const RowSums& x, const RowSums& y, float scale) {
  const float r = fmaxf(x.ref, y.ref);
  // (-inf - -inf counts as the least)
  const float dx = fmaxf((x.ref - r) * scale, kLeastExponent), dy = fmaxf((y.ref - r) * scale, kLeastExponent);
  const float ex = ptx_exp2(dx), ey = ptx_exp2(dy);
  // products rounded before the sum: the same bits whichever is x, so that all lanes of a merge have the same
  return {r, __fadd_rn(__fmul_rn(ex, x.s), __fmul_rn(ey, y.s)),
          __fadd_rn(__fmul_rn(ex, fmaf(dx, x.s, x.a)), __fmul_rn(ey, fmaf(dy, y.s, y.a)))};
}

// The sums of a warp's lanes together, to every lane (the same bits: pairs are added, and a sum does not depend on its order).
// With lanes < 32 the lanes' values repeat every `lanes`, and one period counts.
template <int kLanes>
__device__ __forceinline__ RowSums merge_lanes(const RowSums& x, float scale) {
  const uint32_t u = __float_as_uint(x.ref);
  const uint32_t most = __reduce_max_sync(0xffffffffu, (u & 0x80000000u) ? ~u : (u | 0x80000000u));   // in the order of floats
  const float r = __uint_as_float((most & 0x80000000u) ? (most & 0x7FFFFFFFu) : ~most);
  const float d = fmaxf((x.ref - r) * scale, kLeastExponent), e = ptx_exp2(d);   // (-inf - -inf counts as the least)
  float s = e * x.s, a = e * fmaf(d, x.s, x.a);
#pragma unroll
  for (int o = 1; o < kLanes; o <<= 1) {
    s += __shfl_xor_sync(0xffffffffu, s, o);
    a += __shfl_xor_sync(0xffffffffu, a, o);
  }
  return {r, s, a};
}

// A thread's sums, in packed pairs.
struct ThreadSums {
  float most = -INFINITY;   // the largest logit seen
  float neg = 0.f;          // -most (0: none yet)
  unsigned long long s = 0ull, a = 0ull;

  __device__ __forceinline__ void raise(float m, float scale) {
    if (!(m > most)) return;
    const float d = fmaxf((most - m) * scale, kLeastExponent), e = ptx_exp2(d);
    s = f2_mul(s, f2_pack(e, e));   // 2^d (a + d s) = 2^d a + d (2^d s)
    a = f2_fma(f2_pack(d, d), s, f2_mul(a, f2_pack(e, e)));
    most = m, neg = -m;
  }
  // Adds N logits (even; none above `most`).  They are summed by themselves first: a row's sum then has a rounding per block of
  // N rather than one per pair.
  template <int N>
  __device__ __forceinline__ void add(const float (&x)[N], unsigned long long scale2) {
    const unsigned long long neg2 = f2_pack(neg, neg);
    unsigned long long bs = 0ull, ba = 0ull;
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      float t0, t1;
      f2_unpack(f2_mul(f2_add(f2_pack(x[i], x[i + 1]), neg2), scale2), t0, t1);
      t0 = max_nan(t0, kLeastExponent), t1 = max_nan(t1, kLeastExponent);
      const unsigned long long e = f2_pack(ptx_exp2(t0), ptx_exp2(t1));
      bs = f2_add(bs, e);
      ba = f2_fma(f2_pack(t0, t1), e, ba);
    }
    s = f2_add(s, bs);
    a = f2_add(a, ba);
  }
  __device__ __forceinline__ RowSums sums() const {
    float s0, s1, a0, a1;
    f2_unpack(s, s0, s1);
    f2_unpack(a, a0, a1);
    return {most, s0 + s1, a0 + a1};
  }
};

// A finished row: ln S, and what log p_i and the entropy are made of.  log p_i takes its difference in natural units, so that
// what is within 32 bits there stays so.
struct RowResult {
  float ref, ln_s, entropy;
  __device__ __forceinline__ explicit RowResult(const RowSums& x)
      : ref(x.ref), ln_s(logf(x.s)), entropy(x.s == 0.f ? 0.f : logf(x.s) - x.a / x.s * kLn2) {}
  // log p of a logit x; -inf for every one of a row of -inf
  __device__ __forceinline__ float logprob(float x, float inv_temperature) const {
    return ref == -INFINITY && !(ln_s != ln_s) ? -INFINITY : (x - ref) * inv_temperature - ln_s;
  }
};

}  // namespace ptd
