// Internal launch parameters of the prompt kernels (not part of the C ABI).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

#include "prompt_geometry.cuh"
#include "tree_rope.cuh"

namespace ptd {

struct PromptSlotsParams {
  const int32_t* token_offsets;
  const int32_t* ctx_lens;
  int batch;
  PromptBounds bounds;
  int page_size, page_log2, seq_capacity, num_pages, max_pages;
  const int32_t* block_table;
  // the page pool: free_pages NULL without one
  int32_t* free_pages;
  const int32_t* free_count;
  const int32_t* held;
  int32_t* new_held;
  int32_t* new_free_count;
  int32_t* table_out;
  int32_t* slots;
  int32_t* positions;
  int32_t* dev_status;
};
cudaError_t launch_prompt_slots(const PromptSlotsParams& p, int sms, cudaStream_t stream);

struct PromptRopeParams {
  const int32_t* slots;
  const int32_t* positions;
  int n_tokens, head_dim, hq, hkv;
  const void* q;
  const void* k;
  const void* v;
  void* q_out;
  int64_t q_stride, k_stride, v_stride, q_out_stride;   // elements
  void* k_layer;      // the layer's first row
  void* v_layer;
  int64_t layer_rows;
  int32_t* dev_status;
  HeadNorms norms;    // weights [D]
};
cudaError_t launch_prompt_rope(const PromptRopeParams& p, bool bf16, const RopeFreqs& freqs, int sms,
                               cudaStream_t stream);
// The same with norms (called by it).
cudaError_t launch_prompt_norm_rope(const PromptRopeParams& p, bool bf16, const RopeFreqs& freqs, int sms, cudaStream_t stream);

struct PromptAttnParams {
  const void* q;
  void* out;
  const void* k;               // the cache's base pointers
  const void* v;
  float* part_o;               // split keys: partials [piece][D / 4][rows of a block][4], O unnormalised
  float* part_ml;              // [piece][rows][2]: running max in log2 units, row sum
  const int32_t* token_offsets;
  const int32_t* ctx_lens;
  const int32_t* block_table;
  int32_t* dev_status;
  PromptBounds bounds;
  int64_t q_stride;            // elements between tokens of q
  int batch, hq, hkv, head_dim, layer;
  int sub;                     // query heads of one KV head that share a tile (a divisor of hq / hkv)
  int tile_heads;              // hq / sub: head tiles
  int tiles_per_kv;            // head tiles per KV head
  int tile_tokens;             // tokens per M tile (tile_tokens * sub rows of it are used)
  int block_tokens;            // tokens per block: one or two M tiles
  int tile_rows;               // rows of an M tile in the partials
  int key_tile, key_tile_log2; // keys per tile
  int level_step;              // of the blocks' order (prompt_geometry.cuh)
  IndexDivisor by_block, by_heads, by_kv, by_splits, by_sub;   // block_tokens, tile_heads, tiles_per_kv, splits, sub
  int blocks;                  // upper bound of the batch's blocks of tokens (per head tile)
  int places;                  // of the blocks' partials (per head tile)
  int cut_ctas;                // CTAs at a time of a cut by the lengths on the device (PromptCut); 0: none
  int most_shares;             // of such a cut: what the scratch and the grid have room for
  CutCosts costs;
  int splits, piece_tiles;     // a block's keys are cut into pieces of piece_tiles key tiles, at most `splits` (1: uncut)
  int page_size, page_log2, seq_capacity, num_pages, max_pages;
  float scale_log2;            // scale * log2(e)
};

// Chooses the tiles and the cut of the keys from the host-known sizes, with `scratch` bytes at hand: sets sub,
// tile_heads, tiles_per_kv, tile_tokens, block_tokens, tile_rows, key_tile, level_step, blocks, piece_tiles, splits and cut_ctas.
// Returns the scratch that the cut takes (0: unsplit).
size_t plan_prompt_attention(PromptAttnParams& p, bool bf16, size_t scratch, int sms);
// bf16, D = 128.  map_k, map_v: boxes of 64 columns of one KV head and 128 rows (or a page's); map_q: of 64
// columns, `sub` heads and tile_tokens tokens; 128-byte swizzle.
cudaError_t launch_prompt_attn_tc(const CUtensorMap& map_k, const CUtensorMap& map_v, const CUtensorMap& map_q,
                                  const PromptAttnParams& p, cudaStream_t stream);
// fp32, D = 32, 64 or 128.
cudaError_t launch_prompt_attn_simt(const PromptAttnParams& p, cudaStream_t stream);
// The merge of split blocks, after either.
cudaError_t launch_prompt_attn_merge(const PromptAttnParams& p, bool bf16, cudaStream_t stream);

}  // namespace ptd
