// Internal launcher of the LM head with log probabilities (not part of the C ABI).
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

namespace ptd {
struct RowSums;

// How the product's tiles go to CTAs: phases of at most `per_phase` row tiles; in a phase of R row tiles CTA i has row tile
// i % R and, with C = ctas / R lanes, the vocabulary tiles i / R, i / R + C, ... (none for i / R >= C).
struct LmLogprobsPlan {
  int ctas, row_tiles, per_phase, tile_tokens, vocab_tiles;
  int box_rows;   // rows of H that are loaded of a tile: a multiple of 8, the others of the tile are anything
  int stages;     // of the ring
  int keys;       // kept of each row's part (>= k)
};
LmLogprobsPlan plan_lm_logprobs(int rows, int vocab, int d_model, int k, int sms);
size_t lm_logprobs_workspace_bytes(int rows, int vocab, int k, int sms);   // for any d_model

struct LmLogprobsParams {
  int rows, d_model, vocab, k;
  float scale;                // log2(e) / temperature
  float inv_temperature;
  const int32_t* tokens;
  float* logprob;
  float* entropy;             // or NULL
  int32_t* top_idx;
  float* top_val;
  int32_t* dev_status;
  LmLogprobsPlan plan;
  void* workspace;
};
// map_h, map_w: boxes of 64 columns and plan.box_rows or plan.tile_tokens rows, 128-byte swizzle.
constexpr int kLmTileRows = 128;
cudaError_t launch_lm_logprobs(const CUtensorMap& map_h, const CUtensorMap& map_w, const LmLogprobsParams& p, cudaStream_t stream);
}  // namespace ptd
