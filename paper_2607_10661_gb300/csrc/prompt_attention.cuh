// Pieces shared by the prompt-attention kernels: a CTA's work unit and its key range.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "prompt.cuh"

namespace ptd {
namespace pa {

// A block of tokens of one sequence under one head tile, and a piece of its keys.
struct Unit {
  int b, token0, tokens;   // sequence; the block's first token within it, and how many
  int row0;                // token0's row in q and out
  int ctx;                 // C_b
  int head0, kv;           // first query head, KV head
  int tiles;               // key tiles of the block
  int tile0, tile1;        // those of this piece
};

// Key tiles [k0, k1) of piece s of S.
__device__ __forceinline__ void piece_range(int tiles, int s, int S, int& k0, int& k1) {
  k0 = (int)((int64_t)tiles * s / S);
  k1 = (int)((int64_t)tiles * (s + 1) / S);
}

// Sequence b's blocks (none if it is out of range).
__device__ __forceinline__ PromptBlocks blocks_of(const PromptAttnParams& p, int b) {
  const int off0 = p.token_offsets[b], off1 = p.token_offsets[b + 1], ctx = p.ctx_lens[b];
  return prompt_sequence_ok(p.bounds, off0, off1, ctx) ? prompt_blocks(ctx, off1 - off0, p.block_tokens) : PromptBlocks{0, 0};
}

// A key above every block's (a warp's answer); `seq` as find_prompt_block takes it.
template <typename Seq>
__device__ __forceinline__ int max_block_key(const Seq& seq, int batch) {
  int m = 0;
  for (int b = threadIdx.x & 31; b < batch; b += 32) {
    const PromptBlocks s = seq(b);
    m = max(m, s.first + s.count);
  }
  return (int)__reduce_max_sync(0xffffffffu, (unsigned)m);
}

// Block y / tile_heads of the batch under head tile y % tile_heads, with all of its keys (a warp's answer).
// False: there is none.
template <typename Seq>
__device__ __forceinline__ bool find_unit(const PromptAttnParams& p, const Seq& seq, int max_key, int y, Unit& u) {
  const int block = y / p.tile_heads, tile = y - block * p.tile_heads;
  int i;
  if (!find_prompt_block(WarpLanes{}, seq, p.batch, max_key, block, &u.b, &i)) return false;
  const int off0 = p.token_offsets[u.b], n = p.token_offsets[u.b + 1] - off0;
  u.ctx = p.ctx_lens[u.b];
  u.token0 = i * p.block_tokens;
  u.tokens = min(p.block_tokens, n - u.token0);
  u.row0 = off0 + u.token0;
  u.head0 = tile * p.sub;
  u.kv = tile / p.tiles_per_kv;
  u.tiles = (u.ctx + u.token0 + u.tokens + p.key_tile - 1) / p.key_tile;
  u.tile0 = 0;
  u.tile1 = u.tiles;
  return true;
}

}  // namespace pa
}  // namespace ptd
