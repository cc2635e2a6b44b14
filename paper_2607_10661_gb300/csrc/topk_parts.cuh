// Pieces shared by the kernels that select the largest logits of a row (topk.cu, token_logprobs.cu): ordered keys, vectors of
// logits, and the k-th largest of a warp's values (internal).
//
// Order: a 64-bit key (order-preserving bits of the fp32 value) << 32 | ~index, so a larger key is a larger value
// or, on equal values, a lower index.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "ptd_device.cuh"

namespace ptd {
namespace topk {

__device__ __forceinline__ uint32_t ordered_bits(float f) {
  uint32_t u = __float_as_uint(f);
  if (u == 0x80000000u) u = 0u;   // -0.0 == +0.0
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ float from_ordered(uint32_t o) {
  const uint32_t u = (o & 0x80000000u) ? (o & 0x7FFFFFFFu) : ~o;
  return __uint_as_float(u);
}

__device__ __forceinline__ uint64_t make_key(uint32_t ord, uint32_t idx) {
  return ((uint64_t)ord << 32) | (uint64_t)(~idx);
}

// Largest key of the warp: the largest high word (one warp reduction), then the largest low
// word among the lanes that hold it (a second one).
__device__ __forceinline__ uint64_t warp_max_u64(uint64_t v) {
  const uint32_t hi = (uint32_t)(v >> 32);
  const uint32_t mhi = __reduce_max_sync(0xffffffffu, hi);
  const uint32_t mlo = __reduce_max_sync(0xffffffffu, hi == mhi ? (uint32_t)v : 0u);
  return ((uint64_t)mhi << 32) | mlo;
}

template <typename T>
struct Vec;
template <>
struct Vec<__nv_bfloat16> {
  static constexpr int kN = 8;
  __device__ __forceinline__ static void unpack(const uint4& v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f[2 * j] = __uint_as_float(w[j] << 16);
      f[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
    }
  }
  __device__ __forceinline__ static float scalar(const __nv_bfloat16* p) {
    return __uint_as_float((uint32_t)(*reinterpret_cast<const uint16_t*>(p)) << 16);
  }
};
template <>
struct Vec<float> {
  static constexpr int kN = 4;
  __device__ __forceinline__ static void unpack(const uint4& v, float (&f)[8]) {
    f[0] = __uint_as_float(v.x);
    f[1] = __uint_as_float(v.y);
    f[2] = __uint_as_float(v.z);
    f[3] = __uint_as_float(v.w);
  }
  __device__ __forceinline__ static float scalar(const float* p) { return *p; }
};

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
// Lane-wise maximum of two bf16 pairs in one instruction (exact: a maximum only compares)
__device__ __forceinline__ uint32_t bf16x2_max(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
constexpr uint32_t kBf16x2NegInf = 0xFF80FF80u;

// The largest logit of a 16-byte vector.
template <typename T>
__device__ __forceinline__ float vec_max(const uint4& x) {
  if constexpr (sizeof(T) == 2) {
    const uint32_t h = bf16x2_max(bf16x2_max(x.x, x.y), bf16x2_max(x.z, x.w));
    return fmaxf(bf16_lo(h), bf16_hi(h));
  } else {
    return fmax3(__uint_as_float(x.x), __uint_as_float(x.y), fmaxf(__uint_as_float(x.z), __uint_as_float(x.w)));
  }
}

// The k-th largest of the warp's 32 order-preserving values (0 = a lane without one), or 0 when
// fewer than k lanes hold one: one warp maximum and one ballot per distinct value, equal values
// counted together.  Any x with k elements >= x bounds the warp's top-k from below.
__device__ __forceinline__ uint32_t kth_largest_ord(uint32_t v, int k) {
  int count = 0;
  for (int s = 0; s < k; ++s) {
    const uint32_t m = __reduce_max_sync(0xffffffffu, v);
    if (m == 0u) return 0u;
    count += __popc(__ballot_sync(0xffffffffu, v == m));
    if (count >= k) return m;
    if (v == m) v = 0u;
  }
  return 0u;
}

// The k-th largest (k <= 32) of 32 shared values, by every warp on its own: a lane's value with
// k - 1 values before it (larger, or equal at a lower lane).
__device__ __forceinline__ uint32_t kth_of_32(const uint32_t* v_s, int k) {
  const int lane = threadIdx.x & 31;
  const uint32_t mine = v_s[lane];
  int before = 0;
#pragma unroll
  for (int i = 0; i < 32; i += 4) {
    const uint4 o = *reinterpret_cast<const uint4*>(v_s + i);
    before += (o.x > mine || (o.x == mine && i < lane)) + (o.y > mine || (o.y == mine && i + 1 < lane)) +
              (o.z > mine || (o.z == mine && i + 2 < lane)) + (o.w > mine || (o.w == mine && i + 3 < lane));
  }
  const uint32_t at = __ballot_sync(0xffffffffu, before == k - 1);
  return __shfl_sync(0xffffffffu, mine, __ffs(at) - 1);
}

}  // namespace topk
}  // namespace ptd
