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

// The norm of a head that lies across `lanes` lanes (a power of two, whole within its aligned group of lanes), each with
// two vectors: 1 / sqrt(mean_D(x^2) + eps).  Every lane of the warp takes part; the lanes' sums meet pairwise, so that all
// have the same.
template <typename T>
__device__ __forceinline__ float norm_of_head(const Vec<T>& x, const Vec<T>& y, int lanes, float inv_d, float eps) {
  float s0 = 0.f, s1 = 0.f;
#pragma unroll
  for (int i = 0; i < Vec<T>::N; ++i) s0 = fmaf(x.x[i], x.x[i], s0), s1 = fmaf(y.x[i], y.x[i], s1);
  float s = s0 + s1;
  for (int o = lanes >> 1; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return __frsqrt_rn(fmaf(s, inv_d, eps));
}
template <typename T>
__device__ __forceinline__ void scale_by(Vec<T>& x, float r, const Vec<T>& w) {
#pragma unroll
  for (int i = 0; i < Vec<T>::N; ++i) x.x[i] *= r * w.x[i];
}

// Norm and rotation of a head's D elements by one warp, element by element (dst may be src: the warp has read the
// row for the norm before it writes, and a pair before it writes that).
template <typename T>
__device__ __forceinline__ void norm_and_turn_row(const T* src, T* dst, const T* w, int D, float eps, const float* cos_s,
                                                  const float* sin_s) {
  const int lane = threadIdx.x & 31, half = D / 2;
  float s = 0.f;
  for (int i = lane; i < D; i += 32) {
    const float x = ld(src + i);
    s = fmaf(x, x, s);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  const float norm = __frsqrt_rn(fmaf(s, 1.f / (float)D, eps));
  for (int j = lane; j < half; j += 32) {
    const float a = ld(src + j) * (norm * ld(w + j)), b = ld(src + j + half) * (norm * ld(w + j + half));
    st(dst + j, a * cos_s[j] - b * sin_s[j]);
    st(dst + j + half, a * sin_s[j] + b * cos_s[j]);
  }
}

}  // namespace rope
}  // namespace ptd
