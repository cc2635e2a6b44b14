// Rotary encoding of packed tokens and their K/V into cache slots, one layer.
//
// Token n at position p = positions[n]: the pair (x_j, x_{j+D/2}) of its query and key heads turns by
// p * base^(-2j/D) (RoFormer's rotation in the rotate-half layout; the angle's arithmetic is in
// rope_parts.cuh); the rotated keys and the values go to cache row slots[n].  A row is cut into items of two
// 16-byte vectors, columns j and j + D/2; a CTA takes the items of a run of tokens, kItems per thread at a
// time, and asks for them before it forms its tokens' (cos, sin) tables.
//
// What bounds it: the reads and writes, (2 Hq + 4 Hkv) D elements a token: 8192 tokens of 32/8 heads (bf16, D = 128,
// 201 MB) 31.7 us in graph replays, 6.3 TB/s, and 34.0 among other passes, 20000 tokens 72.0 us, 6.8 TB/s; for few tokens
// latency: 8 tokens 2.1 us.  (Streaming loads, __ldcs, were 1.5 % slower.)
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "launch.cuh"
#include "prompt.cuh"
#include "ptd_device.cuh"
#include "rope_parts.cuh"
#include "row_division.cuh"

namespace ptd {
namespace pr {

using namespace rope;

constexpr int kMaxTokens = 8;   // of one CTA

// kItems of each thread in flight, kCtas on an SM.
template <typename T, int kThreads, int kItems, int kCtas>
__global__ void __launch_bounds__(kThreads, kCtas)
    prompt_rope_kernel(const PromptRopeParams p, const __grid_constant__ RopeFreqs freqs, int tokens_per_cta,
                       GroupDivisor by_token, GroupDivisor by_chunks) {
  __shared__ float cos_s[kMaxTokens * kMaxRopeHalf], sin_s[kMaxTokens * kMaxRopeHalf];
  __shared__ int slot_s[kMaxTokens];
  constexpr int V = Vec<T>::N;
  const int t = threadIdx.x, n0 = blockIdx.x * tokens_per_cta, tokens = min(tokens_per_cta, p.n_tokens - n0);
  const int half = p.head_dim / 2, chunks = half / V, per_token = (p.hq + 2 * p.hkv) * chunks, items = tokens * per_token;
  const int D = p.head_dim, hq = p.hq, hkv = p.hkv;
  if (t == 0) grid_launch_dependents();
  grid_dependency_wait();   // q, k, v, the slots and the cache belong to the stream's previous work
  // item e: its token (of this CTA), head (q heads, then k heads, then v heads) and first column
  auto place_of = [&](int e, int& n, int& h, int& j) {
    n = tokens > 1 ? divide_by_group(e, by_token) : 0;
    const int r = e - n * per_token;
    h = divide_by_group(r, by_chunks);
    j = (r - h * chunks) * V;
  };
  const int first_slot = p.slots[n0 + min(t, tokens - 1)];
  uint4 lo[kItems], hi[kItems];
  auto load_items = [&](int e0) {
#pragma unroll
    for (int u = 0; u < kItems; ++u) {
      const int e = e0 + u * kThreads;
      if (e < items) {
        int i, h, j;
        place_of(e, i, h, j);
        const size_t n = (size_t)(n0 + i);
        const T* src = h < hq ? static_cast<const T*>(p.q) + n * p.q_stride + (size_t)h * D + j
                       : h < hq + hkv ? static_cast<const T*>(p.k) + n * p.k_stride + (size_t)(h - hq) * D + j
                                      : static_cast<const T*>(p.v) + n * p.v_stride + (size_t)(h - hq - hkv) * D + j;
        lo[u] = *reinterpret_cast<const uint4*>(src);   // plain loads: q may also be written
        hi[u] = *reinterpret_cast<const uint4*>(src + half);
      }
    }
  };
  load_items(t);
  if (t < tokens) {
    const bool fits = first_slot >= 0 && first_slot < p.layer_rows;
    slot_s[t] = fits ? first_slot : -1;
    if (!fits && first_slot != -1) atomicMax(p.dev_status, (int)PTD_ERR_INVALID_BATCH);
  }
  for (int x = t; x < tokens * half; x += kThreads)
    turn_of(freqs, p.positions[n0 + x / half], x % half, cos_s[x], sin_s[x]);
  __syncthreads();
  for (int e0 = t;; load_items(e0)) {
#pragma unroll
    for (int u = 0; u < kItems; ++u) {
      const int e = e0 + u * kThreads;
      if (e >= items) continue;
      int i, h, j;
      place_of(e, i, h, j);
      const int slot = slot_s[i];
      if (slot < 0) continue;
      uint4 a = lo[u], b = hi[u];
      if (h < hq + hkv) {
        const Vec<T> x = unpack16<T>(a), y = unpack16<T>(b);
        Vec<T> rx, ry;
#pragma unroll
        for (int c = 0; c < V; ++c) {
          const float cs = cos_s[i * half + j + c], sn = sin_s[i * half + j + c];
          rx.x[c] = x.x[c] * cs - y.x[c] * sn;
          ry.x[c] = x.x[c] * sn + y.x[c] * cs;
        }
        a = pack16(rx);
        b = pack16(ry);
      }
      T* dst;
      if (h < hq) {
        dst = static_cast<T*>(p.q_out) + (size_t)(n0 + i) * p.q_out_stride + (size_t)h * D + j;
      } else {
        const size_t row = (size_t)slot * hkv;
        dst = h < hq + hkv ? static_cast<T*>(p.k_layer) + (row + (h - hq)) * D + j
                           : static_cast<T*>(p.v_layer) + (row + (h - hq - hkv)) * D + j;
      }
      *reinterpret_cast<uint4*>(dst) = a;
      *reinterpret_cast<uint4*>(dst + half) = b;
    }
    e0 += kItems * kThreads;
    if (e0 - t >= items) break;
  }
}

// Rows that are not 16-byte vectors: one element at a time, one CTA per token.
constexpr int kScalarThreads = 256;
template <typename T>
__global__ void __launch_bounds__(kScalarThreads)
    prompt_rope_scalar_kernel(const PromptRopeParams p, const __grid_constant__ RopeFreqs freqs) {
  __shared__ float cos_s[kMaxRopeHalf], sin_s[kMaxRopeHalf];
  const size_t n = blockIdx.x;
  const int t = threadIdx.x, D = p.head_dim, half = D / 2;
  if (t == 0) grid_launch_dependents();
  grid_dependency_wait();   // q, k, v, the slots and the cache belong to the stream's previous work
  const int slot = p.slots[n];
  if (slot < 0 || slot >= p.layer_rows) {
    if (t == 0 && slot != -1) atomicMax(p.dev_status, (int)PTD_ERR_INVALID_BATCH);
    return;
  }
  for (int j = t; j < half; j += kScalarThreads) turn_of(freqs, p.positions[n], j, cos_s[j], sin_s[j]);
  __syncthreads();
  const T* q = static_cast<const T*>(p.q) + n * p.q_stride;
  const T* k = static_cast<const T*>(p.k) + n * p.k_stride;
  const T* v = static_cast<const T*>(p.v) + n * p.v_stride;
  T* qo = static_cast<T*>(p.q_out) + n * p.q_out_stride;
  T* ko = static_cast<T*>(p.k_layer) + (size_t)slot * p.hkv * D;
  T* vo = static_cast<T*>(p.v_layer) + (size_t)slot * p.hkv * D;
  for (int e = t; e < (p.hq + p.hkv) * half; e += kScalarThreads) {
    const bool isq = e < p.hq * half;
    const int e2 = isq ? e : e - p.hq * half;
    const int h = e2 / half, j = e2 - h * half;
    const T* src = (isq ? q : k) + (size_t)h * D;
    T* dst = (isq ? qo : ko) + (size_t)h * D;
    const float a = ld(src + j), b = ld(src + j + half);
    const float c = cos_s[j], s = sin_s[j];
    st(dst + j, a * c - b * s);
    st(dst + j + half, a * s + b * c);
  }
  for (int e = t; e < p.hkv * D; e += kScalarThreads) vo[e] = v[e];
}

template <typename T, int kThreads, int kItems, int kCtas>
cudaError_t launch(const PromptRopeParams& p, const RopeFreqs& freqs, int chunks, int per_token, int sms, cudaStream_t stream) {
  // as many tokens a CTA as fill the items of its threads, fewer where the CTAs would not fill the SMs
  int tokens = kItems * kThreads / per_token;
  const int64_t fill = p.n_tokens / (kCtas * (int64_t)sms);
  if (tokens > fill) tokens = (int)fill;
  tokens = tokens < 1 ? 1 : (tokens > kMaxTokens ? kMaxTokens : tokens);
  return launch_chained(prompt_rope_kernel<T, kThreads, kItems, kCtas>, dim3((unsigned)((p.n_tokens + tokens - 1) / tokens)),
                        dim3(kThreads), 0, stream, 0, p, freqs, tokens, group_divisor(per_token), group_divisor(chunks));
}

}  // namespace pr

cudaError_t launch_prompt_rope(const PromptRopeParams& p, bool bf16, const RopeFreqs& freqs, int sms,
                               cudaStream_t stream) {
  const int64_t es = bf16 ? 2 : 4;
  const auto al16 = [](const void* x) { return (reinterpret_cast<uintptr_t>(x) & 15u) == 0; };
  const bool aligned = al16(p.q) && al16(p.k) && al16(p.v) && al16(p.q_out) && al16(p.k_layer) && al16(p.v_layer) &&
                       (p.q_stride * es | p.k_stride * es | p.v_stride * es | p.q_out_stride * es) % 16 == 0;
  const int vec = bf16 ? 8 : 4, half = p.head_dim / 2;
  // (2^22 items a token: the bound of the kernel's quotients)
  if (aligned && half % vec == 0 && ((int64_t)p.hq + 2 * (int64_t)p.hkv) * (half / vec) < (1 << 22)) {
    const int chunks = half / vec, per_token = (p.hq + 2 * p.hkv) * chunks;
    // While all CTAs have a place at once a token is done soonest by many threads, then small CTAs turn over best.
    // Measured (us, 384 threads of one item each and 128 of three, bf16 with D = 128; SMs 152): 8 tokens of 32/8 heads
    // 2.1 and 2.6, 300 2.9 and 4.0, 600 3.2 and 4.1, [the rule's bound] 620 4.2 and 4.5, 1000 5.0 and 4.6, 8192 37.3 and
    // 31.5; of 64/8 heads 500 4.6 and 6.6, 8000 57.1 and 49.1; fp32 4000 31.8 and 30.3.
    if (p.n_tokens <= 4 * (int64_t)sms)
      return bf16 ? pr::launch<__nv_bfloat16, 384, 1, 4>(p, freqs, chunks, per_token, sms, stream)
                  : pr::launch<float, 384, 1, 4>(p, freqs, chunks, per_token, sms, stream);
    return bf16 ? pr::launch<__nv_bfloat16, 128, 3, 8>(p, freqs, chunks, per_token, sms, stream)
                : pr::launch<float, 128, 3, 8>(p, freqs, chunks, per_token, sms, stream);
  }
  const auto kernel = bf16 ? pr::prompt_rope_scalar_kernel<__nv_bfloat16> : pr::prompt_rope_scalar_kernel<float>;
  return launch_chained(kernel, dim3((unsigned)p.n_tokens), dim3(pr::kScalarThreads), 0, stream, 0, p, freqs);
}

}  // namespace ptd
