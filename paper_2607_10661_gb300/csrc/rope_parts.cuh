// Pieces shared by the kernels that apply the rotary encoding (tree_rope.cu, prompt_rope.cu): elements and
// 16-byte vectors of fp32 or bf16, and the cosine and sine of an angle.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "tree_rope.cuh"

namespace ptd {
namespace rope {

template <typename T>
__device__ __forceinline__ float ld(const T* p);
template <>
__device__ __forceinline__ float ld<float>(const float* p) { return *p; }
template <>
__device__ __forceinline__ float ld<__nv_bfloat16>(const __nv_bfloat16* p) { return __bfloat162float(*p); }
template <typename T>
__device__ __forceinline__ void st(T* p, float x);
template <>
__device__ __forceinline__ void st<float>(float* p, float x) { *p = x; }
template <>
__device__ __forceinline__ void st<__nv_bfloat16>(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// One 16-byte vector of T: 16 / sizeof(T) elements, widened to fp32.
template <typename T>
struct Vec {
  static constexpr int N = 16 / sizeof(T);
  float x[N];
};
template <typename T>
__device__ __forceinline__ Vec<T> unpack16(const uint4& u) {
  Vec<T> r;
  if constexpr (sizeof(T) == 2) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r.x[2 * i] = __uint_as_float(w[i] << 16);
      r.x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  } else {
    r.x[0] = __uint_as_float(u.x), r.x[1] = __uint_as_float(u.y), r.x[2] = __uint_as_float(u.z),
    r.x[3] = __uint_as_float(u.w);
  }
  return r;
}
template <typename T>
__device__ __forceinline__ uint4 pack16(const Vec<T>& r) {
  if constexpr (sizeof(T) == 2) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(r.x[2 * i], r.x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  } else {
    return make_uint4(__float_as_uint(r.x[0]), __float_as_uint(r.x[1]), __float_as_uint(r.x[2]), __float_as_uint(r.x[3]));
  }
}

// cos and sin of pos * f_j, f_j in 2^-64 turns: the product modulo 2^64 is the angle modulo a turn, with no loss for any
// position but that of f_j itself (2^-53 of it, so pos * 2^-53 of the angle).  Its top 24 bits, a float, go through
// sincospif, the next eight (|e| < 2^-21) are added to first order; what is left is 2^-32 of a turn.
__device__ __forceinline__ void turn_of(const RopeFreqs& freqs, int pos, int j, float& c, float& s) {
  const int turn = (int)(((unsigned long long)(long long)pos * freqs.turns[j]) >> 32);   // of 2^-32, in [-1/2, 1/2)
  const float e = (float)(turn & 255) * (6.2831853f / 4294967296.f);
  float s0, c0;
  sincospif((float)(turn & ~255) * (1.f / 2147483648.f), &s0, &c0);
  s = fmaf(e, c0, s0);
  c = fmaf(-e, s0, c0);
}

}  // namespace rope
}  // namespace ptd
