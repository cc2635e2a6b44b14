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

// Sequence b of the batch.
__device__ __forceinline__ PromptSequence load_sequence(const PromptAttnParams& p, int b) {
  const int off0 = p.token_offsets[b], off1 = p.token_offsets[b + 1], ctx = p.ctx_lens[b];
  if (!prompt_sequence_ok(p.bounds, off0, off1, ctx)) return {0, 0, 0, {0, 0}};
  return {off0, off1 - off0, ctx, prompt_blocks(ctx, off1 - off0, p.block_tokens)};
}

// A warp's walk over the batch's units.  Batches of up to 32 sequences are in registers, one a lane.
struct Units {
  PromptSequence mine;
  PromptCursor cur;
  __device__ __forceinline__ Units(const PromptAttnParams& p) : mine{0, 0, 0, {0, 0}}, cur{0, 0, 0} {
    const int lane = threadIdx.x & 31;
    if (lane < p.batch) mine = load_sequence(p, lane);
  }
  // Block y / tile_heads of the batch under head tile y % tile_heads, with all of its keys (every lane gets it).
  // False: there is none.
  __device__ __forceinline__ bool find(const PromptAttnParams& p, int y, Unit& u) {
    const int block = (int)((unsigned)y / (unsigned)p.tile_heads), tile = y - block * p.tile_heads;
    int i;
    PromptSequence s;
    auto load = [&](int b) { return p.batch <= 32 ? mine : load_sequence(p, b); };
    if (!find_prompt_block(WarpLanes{}, load, p.batch, p.level_step, block, cur, u.b, i, s)) return false;
    u.ctx = s.ctx;
    u.token0 = i * p.block_tokens;
    u.tokens = min(p.block_tokens, s.tokens - u.token0);
    u.row0 = s.row0 + u.token0;
    u.head0 = tile * p.sub;
    u.kv = (int)((unsigned)tile / (unsigned)p.tiles_per_kv);
    u.tiles = (u.ctx + u.token0 + u.tokens + p.key_tile - 1) >> p.key_tile_log2;
    u.tile0 = 0;
    u.tile1 = u.tiles;
    return true;
  }
};

}  // namespace pa
}  // namespace ptd
