// Norms of query and key heads, rotary encoding and the append of packed tokens, one layer, one pass.
//
// The mathematics is in rope_parts.cuh: r = 1 / sqrt(mean(x^2) + eps) of a head multiplies its rotation by tables of weight
// times cosine and sine.  One CTA per token: a head is cut into items of two 16-byte vectors, columns j and j + D / 2, its
// items lie in neighbouring lanes and their squares meet in shuffles; a thread asks for kItems of them before the CTA
// forms its token's tables.
//
// What bounds it: the reads and writes, as in prompt_rope.cu, and next to them the instructions (an item's norm, its rotation
// and its addresses are some 110; with cosine, sine and weights applied one after the other and every address formed from the
// item's number they were 280, and 8192 tokens of 32/8 heads, bf16, D = 128, took 41.3 us).  GB300, graph replays: those 33.2 us, 6.06
// TB/s; 8000 tokens of 64/8 heads 50.7, 4000 in fp32 31.8, 8 tokens 2.5.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "launch.cuh"
#include "prompt.cuh"
#include "ptd_device.cuh"
#include "rope_parts.cuh"

namespace ptd {
namespace pn {

using namespace rope;

// A token's slot, or -1 (nothing is written; another one than -1 is reported).
__device__ __forceinline__ int slot_of(const PromptRopeParams& p, int n) {
  const int slot = p.slots[n];
  if (slot >= 0 && slot < p.layer_rows) return slot;
  if (threadIdx.x == 0 && slot != -1) atomicMax(p.dev_status, (int)PTD_ERR_INVALID_BATCH);
  return -1;
}

// kHalf: D / 2 (0: p's).  kItems of each thread in flight, of at most kMost threads.
template <typename T, int kHalf, int kMost, int kItems, int kCtas>
__global__ void __launch_bounds__(kMost, kCtas)
    prompt_norm_rope_kernel(const __grid_constant__ PromptRopeParams p, const __grid_constant__ RopeFreqs freqs) {
  constexpr int V = 16 / (int)sizeof(T);
  __shared__ __align__(16) float tables[kNormTables * (kHalf > 0 ? kHalf : kMaxRopeHalf)];
  const int t = threadIdx.x, threads = blockDim.x, half = kHalf > 0 ? kHalf : p.head_dim / 2, D = 2 * half, chunks = half / V;   // a power of two
  const size_t n = blockIdx.x;
  grid_dependency_wait();   // q, k, v, the slots and the cache belong to the stream's previous work
  const int log2c = kHalf > 0 ? (kHalf / V == 8 ? 3 : 4) : __ffs(chunks) - 1;
  const int q_items = p.hq << log2c, qk_items = (p.hq + p.hkv) << log2c, items = (p.hq + 2 * p.hkv) << log2c;
  const T* q_row = static_cast<const T*>(p.q) + n * p.q_stride;
  const T* k_row = static_cast<const T*>(p.k) + n * p.k_stride;
  const T* v_row = static_cast<const T*>(p.v) + n * p.v_stride;
  auto at_of = [&](int e) { return (e >> log2c) * D + (e & (chunks - 1)) * V; };   // an item's first element in its row
  uint4 lo[kItems], hi[kItems];
  auto load_items = [&](int e0) {
#pragma unroll
    for (int u = 0; u < kItems; ++u) {
      const int e = e0 + u * threads;
      lo[u] = hi[u] = make_uint4(0u, 0u, 0u, 0u);
      if (e < items) {
        const T* src = e < q_items ? q_row + at_of(e) : e < qk_items ? k_row + at_of(e - q_items) : v_row + at_of(e - qk_items);
        lo[u] = *reinterpret_cast<const uint4*>(src);   // plain loads: q may also be written
        hi[u] = *reinterpret_cast<const uint4*>(src + half);
      }
    }
  };
  load_items(t);
  const int slot = slot_of(p, (int)n);
  for (int x = t; x < half; x += threads) {
    const NormWeights w = load_norm_weights<T>(p.norms.q_weight, p.norms.k_weight, 0, x, half);
    float c, s;
    turn_of(freqs, p.positions[n], x, c, s);
    make_norm_columns<T>(tables, w, x, half, c, s);
  }
  // The next grid may be placed from here on (500 tokens 3.9 us, 4.8 where its CTAs had waited from the start).
  if (t == 0) grid_launch_dependents();
  if (slot < 0) return;   // the whole CTA
  __syncthreads();
  T* q_to = static_cast<T*>(p.q_out) + n * p.q_out_stride;
  T* k_to = static_cast<T*>(p.k_layer) + (size_t)slot * p.hkv * D;
  T* v_to = static_cast<T*>(p.v_layer) + (size_t)slot * p.hkv * D;
  const float inv_d = 1.f / (float)D;
  for (int e0 = t;; load_items(e0)) {
#pragma unroll
    for (int u = 0; u < kItems; ++u) {
      const int e = e0 + u * threads;
      const bool isq = e < q_items;
      T* dst = isq ? q_to + at_of(e) : k_to + at_of(e - q_items);
      if (e - (t & 31) < qk_items) {   // not a warp of values: every lane takes part
        const float r = norm_of_head<T>(lo[u], hi[u], chunks, inv_d, p.norms.eps);
        if (e < qk_items) norm_and_turn<T>(lo[u], hi[u], r, tables + (isq ? 0 : 4 * half), (e & (chunks - 1)) * V, half);
      }
      if (e >= qk_items) dst = v_to + at_of(e - qk_items);
      if (e < items) {
        *reinterpret_cast<uint4*>(dst) = lo[u];
        *reinterpret_cast<uint4*>(dst + half) = hi[u];
      }
    }
    e0 += kItems * threads;
    if (e0 - t >= items) break;
  }
}

// Rows that are not 16-byte vectors, or heads whose items are not a power of two: a warp per head, element by element.
constexpr int kScalarThreads = 256;
template <typename T>
__global__ void __launch_bounds__(kScalarThreads)
    prompt_norm_rope_scalar_kernel(const __grid_constant__ PromptRopeParams p, const __grid_constant__ RopeFreqs freqs) {
  __shared__ float cos_s[kMaxRopeHalf], sin_s[kMaxRopeHalf];
  const size_t n = blockIdx.x;
  const int t = threadIdx.x, D = p.head_dim;
  if (t == 0) grid_launch_dependents();
  grid_dependency_wait();   // q, k, v, the slots and the cache belong to the stream's previous work
  const int slot = slot_of(p, (int)n);
  if (slot < 0) return;
  for (int j = t; j < D / 2; j += kScalarThreads) turn_of(freqs, p.positions[n], j, cos_s[j], sin_s[j]);
  __syncthreads();
  const T* q = static_cast<const T*>(p.q) + n * p.q_stride;
  const T* k = static_cast<const T*>(p.k) + n * p.k_stride;
  const T* v = static_cast<const T*>(p.v) + n * p.v_stride;
  T* q_to = static_cast<T*>(p.q_out) + n * p.q_out_stride;
  T* k_to = static_cast<T*>(p.k_layer) + (size_t)slot * p.hkv * D;
  T* v_to = static_cast<T*>(p.v_layer) + (size_t)slot * p.hkv * D;
  for (int h = t >> 5; h < p.hq + p.hkv; h += kScalarThreads / 32) {
    const bool isq = h < p.hq;
    const T* src = isq ? q + (size_t)h * D : k + (size_t)(h - p.hq) * D;
    T* dst = isq ? q_to + (size_t)h * D : k_to + (size_t)(h - p.hq) * D;
    norm_and_turn_row(src, dst, static_cast<const T*>(isq ? p.norms.q_weight : p.norms.k_weight), D, p.norms.eps, cos_s, sin_s);
  }
  for (int e = t; e < p.hkv * D; e += kScalarThreads) v_to[e] = v[e];
}

template <typename T, int kHalf>
cudaError_t launch(const PromptRopeParams& p, const RopeFreqs& freqs, int sms, cudaStream_t stream) {
  const dim3 grid((unsigned)p.n_tokens);
  const int64_t items = ((int64_t)p.hq + 2 * (int64_t)p.hkv) * (p.head_dim / 2) * (int64_t)sizeof(T) / 16;
  const auto threads_of = [&](int most, int each) {   // whole warps
    const int64_t n = (items + 32 * each - 1) / (32 * each) * 32;
    return dim3((unsigned)(n < most ? n : most));
  };
  // While all CTAs have a place at once a token is done soonest by many threads, then small CTAs turn over best.  Measured (us,
  // one item a thread and three; 32/8 heads bf16, D = 128): 8 tokens 2.5 and 3.0, 400 3.2 and 3.9, [the rule's bound] 500 4.3 and
  // 4.8, 1000 6.4 and 5.3; 592 of 16/8 heads fp32, D = 64 2.9 and 3.9.  Two or four items of 128 threads: 8192 tokens 35.5, 35.4
  // (three: 33.2), three of 96: 34.5, of 224 for 64/8 heads 57.0 (50.7).
  const dim3 wide = threads_of(384, 1);
  if (p.n_tokens * (int64_t)wide.x <= 3 * 384 * (int64_t)sms)
    return launch_chained(prompt_norm_rope_kernel<T, kHalf, 384, 1, 3>, grid, wide, 0, stream, 0, p, freqs);
  return launch_chained(prompt_norm_rope_kernel<T, kHalf, 128, 3, 8>, grid, threads_of(128, 3), 0, stream, 0, p, freqs);
}

template <typename T>
cudaError_t launch_typed(const PromptRopeParams& p, const RopeFreqs& freqs, int sms, cudaStream_t stream) {
  constexpr int64_t es = sizeof(T);
  constexpr int vec = 16 / (int)es;
  const auto al16 = [](const void* x) { return (reinterpret_cast<uintptr_t>(x) & 15u) == 0; };
  const bool aligned = al16(p.q) && al16(p.k) && al16(p.v) && al16(p.q_out) && al16(p.k_layer) && al16(p.v_layer) &&
                       (p.q_stride * es | p.k_stride * es | p.v_stride * es | p.q_out_stride * es) % 16 == 0;
  const int half = p.head_dim / 2, chunks = half / vec;   // (at most 32: D <= 256)
  if (aligned && half % vec == 0 && (chunks & (chunks - 1)) == 0)
    return half == 64 ? launch<T, 64>(p, freqs, sms, stream) : launch<T, 0>(p, freqs, sms, stream);
  return launch_chained(prompt_norm_rope_scalar_kernel<T>, dim3((unsigned)p.n_tokens), dim3(kScalarThreads), 0, stream, 0, p, freqs);
}

}  // namespace pn

cudaError_t launch_prompt_norm_rope(const PromptRopeParams& p, bool bf16, const RopeFreqs& freqs, int sms, cudaStream_t stream) {
  return bf16 ? pn::launch_typed<__nv_bfloat16>(p, freqs, sms, stream) : pn::launch_typed<float>(p, freqs, sms, stream);
}

}  // namespace ptd
