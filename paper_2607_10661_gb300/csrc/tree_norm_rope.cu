// Norms of query and key heads, rotary encoding and the append of a tree's rows, in one pass over some layers.
//
// The mathematics is in rope_parts.cuh, the positions are tree_rope.cu's.  A node's rows of q, k and v in a layer are contiguous;
// a CTA has one node in some layers and asks for all its rows at once, as bulk copies into shared memory, before it looks
// the node up and forms its tables (of weights and angles, one set a layer).  Then its threads take the heads item by
// item (two 16-byte vectors, columns j and j + D / 2, a head's items in neighbouring lanes); the values go from shared memory
// to the cache by bulk copies, through no register.
//
// What bounds it: the reads and writes and, for few layers, the chain tree, parents, slot, angles, tables; with the rows of all
// CTAs on their way at once the one hides most of the other.  GB300, graph replays (cold: after 512 MB of other writes, launch
// included): 63 nodes, 32 layers of 32/8 heads, bf16, 49.5 MB 9.4 us (5.3 TB/s), cold 17.5; one layer 3.9; 128 nodes, 32
// layers of 64/8 heads 32.4 (5.2 TB/s).  Items loaded to registers, three a thread, as tree_rope.cu does: 11.5, cold
// 19.7, 4.3 and 37.5.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "launch.cuh"
#include "ptd_device.cuh"
#include "rope_parts.cuh"
#include "tree_place.cuh"
#include "tree_rope.cuh"

namespace ptd {
namespace tn {

using namespace rope;
using tr::find_place;
using tr::kThreads;
using tr::Place;

constexpr int kCtas = 5;                         // of an SM
constexpr size_t kMostSmem = 42 * 1024;          // of one of them: rows and tables of its layers (under the 48 KB of any kernel)

__device__ __forceinline__ bool place_of_node(const TreeNormRopeParams& p, int n, bool first, int* par_s, Place& at) {
  return find_place(p.node_offsets, p.parents, p.ctx_lens, p.batch, n, p.page_size, p.seq_capacity, p.num_pages, p.block_table,
                    p.max_pages, first, par_s, p.positions_out, p.dev_status, at) && at.fits;
}

// Bulk copy shared -> global (both 16-byte aligned, size a multiple of 16), and the wait for all of this thread's.
__device__ __forceinline__ void bulk_store(void* dst, uint32_t src, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(reinterpret_cast<uint64_t>(dst)), "r"(src), "r"(bytes)
               : "memory");
}
__device__ __forceinline__ void bulk_store_drain() {
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
  asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
}

// kHalf: D / 2 (0: p's).
template <typename T, int kHalf>
__global__ void __launch_bounds__(kThreads, kCtas)
    tree_norm_rope_kernel(const __grid_constant__ TreeNormRopeParams p, const __grid_constant__ RopeFreqs freqs) {
  constexpr int V = 16 / (int)sizeof(T);
  extern __shared__ __align__(128) uint8_t smem[];   // [layers][q, k, v rows], then [layers][kNormTables][half] floats
  __shared__ int par_s[kThreads];
  __shared__ __align__(8) uint64_t rows_bar_s;
  __shared__ int abort_s;
  const int t = threadIdx.x, n = blockIdx.x;
  const int half = kHalf > 0 ? kHalf : p.head_dim / 2, D = 2 * half, chunks = half / V;   // a power of two
  const int log2c = __ffs(chunks) - 1, l0 = blockIdx.y * p.layers_per_cta, layers = min(p.num_layers - l0, p.layers_per_cta);
  const uint32_t q_bytes = (uint32_t)(p.hq * D) * sizeof(T), kv_bytes = (uint32_t)(p.hkv * D) * sizeof(T);
  const uint32_t unit = q_bytes + 2 * kv_bytes, bar = smem_u32(&rows_bar_s), rows = smem_u32(smem);
  float* tables = reinterpret_cast<float*>(smem + (size_t)p.layers_per_cta * unit);
  if (t == 0) {
    mbar_init(bar, 1);
    fence_mbar_init();
    abort_s = 0;
  }
  grid_dependency_wait();   // the trees, q, k, v and the cache belong to the stream's previous work
  if (t == 0) {
    mbar_arrive_expect_tx(bar, (uint32_t)layers * unit);
    for (int l = 0; l < layers; ++l) {
      const size_t node = (size_t)(l0 + l) * p.n_total + n;
      const uint32_t dst = rows + (uint32_t)l * unit;
      bulk_load(dst, static_cast<const uint8_t*>(p.q) + node * q_bytes, q_bytes, bar);
      bulk_load(dst + q_bytes, static_cast<const uint8_t*>(p.k) + node * kv_bytes, kv_bytes, bar);
      bulk_load(dst + q_bytes + kv_bytes, static_cast<const uint8_t*>(p.v) + node * kv_bytes, kv_bytes, bar);
    }
  }
  Place at;
  const bool there = place_of_node(p, n, l0 == 0, par_s, at);   // (a barrier: the mbarrier is set up)
  if (there)
    for (int x = t; x < layers * half; x += kThreads) {
      const int l = x / half, j = x - l * half;
      const NormWeights w = load_norm_weights<T>(p.norms.q_weight, p.norms.k_weight, (size_t)(l0 + l) * D, j, half);
      float c, s;
      turn_of(freqs, at.pos, j, c, s);
      make_norm_columns<T>(tables + l * (kNormTables * half), w, j, half, c, s);
    }
  if (t == 0) grid_launch_dependents();
  __syncthreads();   // the tables
  if (!mbar_wait(bar, 0u, &abort_s, p.dev_status)) {   // the copies land before the CTA may end
    mbar_drain(bar, 0u, kWaitLimitNs);
    return;
  }
  if (!there) return;   // nothing is written
  const uint32_t cache_row = (uint32_t)(p.hkv * D);
  if (t == 0)
    for (int l = 0; l < layers; ++l)
      bulk_store(static_cast<T*>(p.v_cache) + ((size_t)(l0 + l) * p.layer_rows + at.row) * cache_row,
                 rows + (uint32_t)l * unit + q_bytes + kv_bytes, kv_bytes);
  const int q_items = p.hq << log2c, per_layer = (p.hq + p.hkv) << log2c, items = layers * per_layer;
  const float inv_d = 1.f / (float)D;
  int l = 0, r = t;   // of item e: its layer and place there
  for (int e = t; e - (t & 31) < items; e += kThreads, r += kThreads) {   // every lane of a warp takes part
    while (r >= per_layer) r -= per_layer, ++l;
    const int h = r >> log2c, j = (r & (chunks - 1)) * V;
    const bool in = e < items, isq = r < q_items;
    const T* src = reinterpret_cast<const T*>(smem + (size_t)(in ? l : 0) * unit) + (in ? h : 0) * D + j;
    uint4 a = *reinterpret_cast<const uint4*>(src), b = *reinterpret_cast<const uint4*>(src + half);
    const float norm = norm_of_head<T>(a, b, chunks, inv_d, p.norms.eps);
    if (!in) continue;
    norm_and_turn<T>(a, b, norm, tables + (l * kNormTables + (isq ? 0 : 4)) * half, j, half);
    T* dst = isq ? static_cast<T*>(p.q_out) + (((size_t)(l0 + l) * p.n_total + n) * p.hq + h) * D + j
                 : static_cast<T*>(p.k_cache) + ((size_t)(l0 + l) * p.layer_rows + at.row) * cache_row + (size_t)(h - p.hq) * D + j;
    *reinterpret_cast<uint4*>(dst) = a;
    *reinterpret_cast<uint4*>(dst + half) = b;
  }
  if (t == 0) bulk_store_drain();
}

// Rows that are not 16-byte vectors, heads whose items are not a power of two, or rows that do not fit (64/64 heads of bf16, 32/32 of
// fp32 at D = 128): a warp per head, element by element, one CTA per (node, layer).  63 nodes, 8 layers of those heads: 28.8 us
// and 15.6 in graph replays, 49.5 MB each.
template <typename T>
__global__ void __launch_bounds__(kThreads)
    tree_norm_rope_scalar_kernel(const __grid_constant__ TreeNormRopeParams p, const __grid_constant__ RopeFreqs freqs) {
  __shared__ int par_s[kThreads];
  __shared__ float cos_s[kMaxRopeHalf], sin_s[kMaxRopeHalf];
  const int n = blockIdx.x, t = threadIdx.x, l = blockIdx.y, D = p.head_dim;
  if (t == 0) grid_launch_dependents();
  grid_dependency_wait();   // the trees, q, k, v and the cache belong to the stream's previous work
  Place at;
  if (!place_of_node(p, n, l == 0, par_s, at)) return;
  for (int j = t; j < D / 2; j += kThreads) turn_of(freqs, at.pos, j, cos_s[j], sin_s[j]);
  __syncthreads();
  const size_t node = (size_t)l * p.n_total + n, row = ((size_t)l * p.layer_rows + at.row) * p.hkv * D;
  const T* q = static_cast<const T*>(p.q) + node * p.hq * D;
  const T* k = static_cast<const T*>(p.k) + node * p.hkv * D;
  const T* v = static_cast<const T*>(p.v) + node * p.hkv * D;
  for (int h = t >> 5; h < p.hq + p.hkv; h += kThreads / 32) {
    const bool isq = h < p.hq;
    const T* src = isq ? q + (size_t)h * D : k + (size_t)(h - p.hq) * D;
    T* dst = isq ? static_cast<T*>(p.q_out) + (node * p.hq + h) * D : static_cast<T*>(p.k_cache) + row + (size_t)(h - p.hq) * D;
    norm_and_turn_row(src, dst, static_cast<const T*>(isq ? p.norms.q_weight : p.norms.k_weight) + (size_t)l * D, D, p.norms.eps,
                      cos_s, sin_s);
  }
  for (int e = t; e < p.hkv * D; e += kThreads) static_cast<T*>(p.v_cache)[row + e] = v[e];
}

template <typename T, int kHalf>
cudaError_t launch(TreeNormRopeParams p, const RopeFreqs& freqs, size_t per_layer, int sms, cudaStream_t stream) {
  // As many layers a CTA as give all CTAs a place at once, no more than its shared memory holds.
  int layers = (int)(kMostSmem / per_layer);
  const int64_t places = kCtas * (int64_t)sms, fill = ((int64_t)p.n_total * p.num_layers + places - 1) / places;
  if (layers > fill) layers = (int)fill;
  p.layers_per_cta = layers < 1 ? 1 : (layers > p.num_layers ? p.num_layers : layers);
  return launch_chained(tree_norm_rope_kernel<T, kHalf>, dim3(p.n_total, (p.num_layers + p.layers_per_cta - 1) / p.layers_per_cta),
                        dim3(kThreads), p.layers_per_cta * per_layer, stream, 0, p, freqs);
}

template <typename T>
cudaError_t launch_typed(const TreeNormRopeParams& p, const RopeFreqs& freqs, int sms, cudaStream_t stream) {
  constexpr int vec = 16 / (int)sizeof(T);
  const auto al16 = [](const void* x) { return (reinterpret_cast<uintptr_t>(x) & 15u) == 0; };
  const bool aligned = al16(p.q) && al16(p.q_out) && al16(p.k) && al16(p.v) && al16(p.k_cache) && al16(p.v_cache);
  const int half = p.head_dim / 2, chunks = half / vec;   // (at most 32: D <= 256)
  const int64_t per_layer = ((int64_t)p.hq + 2 * (int64_t)p.hkv) * p.head_dim * (int64_t)sizeof(T) + kNormTables * half * (int64_t)sizeof(float);
  if (aligned && half % vec == 0 && (chunks & (chunks - 1)) == 0 && per_layer <= (int64_t)kMostSmem)
    return half == 64 ? launch<T, 64>(p, freqs, (size_t)per_layer, sms, stream) : launch<T, 0>(p, freqs, (size_t)per_layer, sms, stream);
  return launch_chained(tree_norm_rope_scalar_kernel<T>, dim3(p.n_total, p.num_layers), dim3(kThreads), 0, stream, 0, p, freqs);
}

}  // namespace tn

cudaError_t launch_tree_norm_rope(TreeNormRopeParams p, bool bf16, const RopeFreqs& freqs, int sms, cudaStream_t stream) {
  return bf16 ? tn::launch_typed<__nv_bfloat16>(p, freqs, sms, stream) : tn::launch_typed<float>(p, freqs, sms, stream);
}

}  // namespace ptd
