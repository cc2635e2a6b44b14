// Pieces shared by the kernels that apply the rotary encoding (tree_rope.cu, prompt_rope.cu): elements and
// 16-byte vectors of fp32 or bf16, and the cosine and sine of an angle.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "ptd_device.cuh"
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

// Norm and rotation of a head in one: with r = 1 / sqrt(mean(x^2) + eps), weights w and the angle's (c, s), the pair (x, y) =
// (x_j, x_{j+D/2}) becomes r (x w_j c - y w_{j+D/2} s), r (x w_j s + y w_{j+D/2} c).  The four products of weights and
// angle do not depend on the head, so they are tables in shared memory: [4][D / 2] floats for the queries' weights, then the
// same for the keys', the columns of a thread's vector in runs of four so that neighbouring lanes read neighbouring runs.
constexpr int kNormTables = 8;   // of D / 2 floats: -w' s, w c, w s, w' c of the queries, of the keys

// Column x of a table: of vector x / N, its element x % N.
template <typename T>
__device__ __forceinline__ int norm_column(int x, int half) {
  constexpr int N = 16 / (int)sizeof(T);
  const int lane = x / N, c = x % N;
  return N == 4 ? x : ((c >> 2) * (half / N) + lane) * 4 + (c & 3);
}
// The weights of column x (row pointers of the queries' and the keys'), and that column of both sets of tables at `table`.
struct NormWeights {
  float q_lo, q_hi, k_lo, k_hi;
};
template <typename T>
__device__ __forceinline__ NormWeights load_norm_weights(const void* q_weight, const void* k_weight, size_t row, int x, int half) {
  const T *q = static_cast<const T*>(q_weight) + row + x, *k = static_cast<const T*>(k_weight) + row + x;
  return {ld(q), ld(q + half), ld(k), ld(k + half)};
}
template <typename T>
__device__ __forceinline__ void make_norm_columns(float* table, const NormWeights& w, int x, int half, float c, float s) {
  float* t = table + norm_column<T>(x, half);
  t[0] = -w.q_hi * s;
  t[half] = w.q_lo * c;
  t[2 * half] = w.q_lo * s;
  t[3 * half] = w.q_hi * c;
  t[4 * half] = -w.k_hi * s;
  t[5 * half] = w.k_lo * c;
  t[6 * half] = w.k_lo * s;
  t[7 * half] = w.k_hi * c;
}

// A 16-byte vector as packed pairs of fp32, and back.
template <typename T>
struct Pairs {
  static constexpr int N = 8 / (int)sizeof(T);   // pairs
  unsigned long long x[N];
};
template <typename T>
__device__ __forceinline__ Pairs<T> unpack_pairs(const uint4& u) {
  Pairs<T> r;
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < Pairs<T>::N; ++i) {
    if constexpr (sizeof(T) == 2)
      r.x[i] = f2_pack(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
    else
      r.x[i] = f2_pack(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
  }
  return r;
}
template <typename T>
__device__ __forceinline__ uint4 pack_pairs(const Pairs<T>& r) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < Pairs<T>::N; ++i) {
    float lo, hi;
    f2_unpack(r.x[i], lo, hi);
    if constexpr (sizeof(T) == 2) {
      w[i] = pack_bf16x2(lo, hi);
    } else {
      w[2 * i] = __float_as_uint(lo), w[2 * i + 1] = __float_as_uint(hi);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// r of a head that lies across `lanes` lanes (a power of two, whole within its aligned group of lanes), each with two
// vectors.  Every lane of the warp takes part; the lanes' sums meet pairwise, so that all have the same.
template <typename T>
__device__ __forceinline__ float norm_of_head(const uint4& lo, const uint4& hi, int lanes, float inv_d, float eps) {
  const Pairs<T> x = unpack_pairs<T>(lo), y = unpack_pairs<T>(hi);
  unsigned long long s2 = 0ull, t2 = 0ull;
#pragma unroll
  for (int i = 0; i < Pairs<T>::N; ++i) s2 = f2_fma(x.x[i], x.x[i], s2), t2 = f2_fma(y.x[i], y.x[i], t2);
  float s0, s1;
  f2_unpack(f2_add(s2, t2), s0, s1);
  float s = s0 + s1;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    if (o < lanes) s += __shfl_xor_sync(0xffffffffu, s, o);
  return __frsqrt_rn(fmaf(s, inv_d, eps));
}
// The two vectors of columns j .. and j + D / 2 .. of a head, normed and turned in place; table: of the head's weights.
template <typename T>
__device__ __forceinline__ void norm_and_turn(uint4& lo, uint4& hi, float r, const float* table, int j, int half) {
  const Pairs<T> x = unpack_pairs<T>(lo), y = unpack_pairs<T>(hi);
  const float* t = table + norm_column<T>(j, half);
  const unsigned long long r2 = f2_pack(r, r);
  Pairs<T> a, b;
#pragma unroll
  for (int i = 0; i < Pairs<T>::N; i += 2) {   // a run of four columns
    const float* run = t + (i >> 1) * (half / Pairs<T>::N / 2 * 4);
    const ulonglong2 ns = *reinterpret_cast<const ulonglong2*>(run), c = *reinterpret_cast<const ulonglong2*>(run + half);
    const ulonglong2 s = *reinterpret_cast<const ulonglong2*>(run + 2 * half), d = *reinterpret_cast<const ulonglong2*>(run + 3 * half);
    a.x[i] = f2_mul(r2, f2_fma(x.x[i], c.x, f2_mul(y.x[i], ns.x)));
    b.x[i] = f2_mul(r2, f2_fma(x.x[i], s.x, f2_mul(y.x[i], d.x)));
    a.x[i + 1] = f2_mul(r2, f2_fma(x.x[i + 1], c.y, f2_mul(y.x[i + 1], ns.y)));
    b.x[i + 1] = f2_mul(r2, f2_fma(x.x[i + 1], s.y, f2_mul(y.x[i + 1], d.y)));
  }
  lo = pack_pairs<T>(a);
  hi = pack_pairs<T>(b);
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
