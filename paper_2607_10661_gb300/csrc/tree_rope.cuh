// Internal launcher of the tree-position / rotary-encoding / K-V append kernel.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

namespace ptd {
constexpr int kMaxRopeHalf = 128;   // D / 2 for D <= 256
struct RopeFreqs {
  unsigned long long turns[kMaxRopeHalf];   // base^(-2i/D) / 2 pi, in 2^-64
};
// The norms of the query and key heads before the rotation: weights [layers of the call][D], NULL: none.
struct HeadNorms {
  const void* q_weight;
  const void* k_weight;
  float eps;
};
cudaError_t launch_tree_rope(const int32_t* node_offsets, const int32_t* parents, const int32_t* ctx_lens,
                             int batch, int n_total, bool bf16, int head_dim, int hq, int hkv, void* q, const void* k,
                             const void* v, void* k_cache, void* v_cache, int layer_begin, int num_layers,
                             int page_size, int seq_capacity,
                             int num_pages, const int32_t* block_table, int max_pages, const RopeFreqs& freqs,
                             int32_t* positions_out, int32_t* dev_status, int sms, cudaStream_t stream);

struct TreeNormRopeParams {
  const int32_t* node_offsets;
  const int32_t* parents;
  const int32_t* ctx_lens;
  int batch, n_total, num_layers, layers_per_cta;   // (the last is the launcher's)
  int head_dim, hq, hkv;
  const void* q;        // [num_layers][n_total][hq][D]
  void* q_out;          // q itself, or apart from q, k and v
  const void* k;
  const void* v;
  HeadNorms norms;      // weights [num_layers][D]
  void* k_cache;        // the first layer's
  void* v_cache;
  int64_t layer_rows;
  int page_size, seq_capacity, num_pages, max_pages;
  const int32_t* block_table;
  int32_t* positions_out;
  int32_t* dev_status;
};
cudaError_t launch_tree_norm_rope(TreeNormRopeParams p, bool bf16, const RopeFreqs& freqs, int sms, cudaStream_t stream);
}  // namespace ptd
