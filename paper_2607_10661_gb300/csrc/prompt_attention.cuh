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
  int tile0, tile1;        // key tiles of the piece
  bool whole;              // all that the block has: no partials
  int place;               // of the partials: (the block's place * tile_heads + head tile) * splits + piece
};

// Sequence b of the batch (read from L2, which has it before any grid that waits for the batch's writer goes on: the
// merge reads it before its own wait).
__device__ __forceinline__ PromptSequence load_sequence(const PromptAttnParams& p, int b, bool& bad) {
  const int off0 = __ldcg(p.token_offsets + b), off1 = __ldcg(p.token_offsets + b + 1), ctx = __ldcg(p.ctx_lens + b);
  if (!prompt_sequence_ok(p.bounds, off0, off1, ctx)) {
    bad = true;
    return {0, 0, 0, {0, 0}};
  }
  return {off0, off1 - off0, ctx, prompt_blocks(ctx, off1 - off0, p.block_tokens, p.by_block)};
}

// A warp's walk over the batch's units.  Batches of up to 32 sequences are in registers, one a lane (one sequence
// alone in every lane); lane l also keeps how many blocks have level l or a higher one.
struct Units {
  PromptSequence mine;
  PromptCursor cur;
  int from_level;
  bool bad;   // some sequence is out of range (of those that the lane has looked at)
  __device__ __forceinline__ Units(const PromptAttnParams& p) : mine{0, 0, 0, {0, 0}}, cur{0, 0, 0, 0, 0}, from_level(0), bad(false) {
    const int lane = threadIdx.x & 31, m = lane * p.level_step;
#pragma unroll 1
    for (int b0 = 0; b0 < p.batch; b0 += 32) {
      const int b = p.batch == 1 ? 0 : b0 + lane;
      PromptSequence s = {0, 0, 0, {0, 0}};
      if (b < p.batch) s = load_sequence(p, b, bad);
      if (b0 == 0) mine = s;
      if (prompt_has_levels(p.batch)) {
#pragma unroll 1
        for (int i = 0; i < min(32, p.batch - b0); ++i)
          from_level += blocks_from({__shfl_sync(0xffffffffu, s.blocks.first, i), __shfl_sync(0xffffffffu, s.blocks.count, i)}, m);
      }
    }
  }
  // Unit number x: piece x % splits of block (x / splits) / tile_heads of the batch under head tile (x / splits) %
  // tile_heads (every lane gets it).  False: there is none.
  __device__ __forceinline__ bool find(const PromptAttnParams& p, int x, Unit& u) {
    const int y = divide(x, p.by_splits), piece = x - y * p.splits;
    const int block = divide(y, p.by_heads), tile = y - block * p.tile_heads;
    int i;
    PromptSequence s;
    auto load = [&](int b) { return p.batch <= 32 ? mine : load_sequence(p, b, bad); };
    auto level_of = [&](int n, int& upto, int& above) {
      const int level = max(0, 31 - __clz(__ballot_sync(0xffffffffu, from_level > n)));
      upto = __shfl_sync(0xffffffffu, from_level, level);
      above = level < kLevels - 1 ? __shfl_sync(0xffffffffu, from_level, level + 1) : 0;
      return level;
    };
    if (!find_prompt_block(WarpLanes{}, load, level_of, p.batch, p.level_step, block, cur, u.b, i, s)) return false;
    u.ctx = s.ctx;
    u.token0 = i * p.block_tokens;
    u.tokens = min(p.block_tokens, s.tokens - u.token0);
    u.row0 = s.row0 + u.token0;
    u.head0 = tile * p.sub;
    u.kv = divide(tile, p.by_kv);
    const int tiles = (u.ctx + u.token0 + u.tokens + p.key_tile - 1) >> p.key_tile_log2;
    u.tile0 = piece * p.piece_tiles;
    u.tile1 = min(tiles, u.tile0 + p.piece_tiles);
    u.whole = u.tile0 == 0 && u.tile1 == tiles;
    u.place = ((block_place(s.row0, u.b, p.by_block) + i) * p.tile_heads + tile) * p.splits + piece;
    return u.tile1 > u.tile0;
  }
};

}  // namespace pa
}  // namespace ptd
