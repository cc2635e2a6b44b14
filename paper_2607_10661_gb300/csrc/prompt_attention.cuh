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
  int place;               // of the partials: (the block's place * tile_heads + head tile) * splits + piece, or a share's
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

// Key tiles of a sequence of one block.
__device__ __forceinline__ int sequence_tiles(const PromptAttnParams& p, const PromptSequence& s) {
  return s.tokens > 0 ? (s.ctx + s.tokens + p.key_tile - 1) >> p.key_tile_log2 : 0;
}

// The cut of the batch by its lengths (prompt_geometry.cuh), and how many key tiles come before sequence `of`; `mine` is
// sequence `lane`.  Warp-collective.
struct LengthCut {
  PromptCut cut;
  int before;
  __device__ __forceinline__ LengthCut(const PromptAttnParams& p, const PromptSequence& mine, int of, bool& bad) : before(0) {
    const int lane = threadIdx.x & 31;
    int units = 0, longest = 0, tiles = 0;
#pragma unroll 1
    for (int b0 = 0; b0 < p.batch; b0 += 32) {
      const int b = b0 + lane, n = b < p.batch ? sequence_tiles(p, b0 == 0 ? mine : load_sequence(p, b, bad)) : 0;
      tiles += (int)__reduce_add_sync(0xffffffffu, (unsigned)n);
      before += (int)__reduce_add_sync(0xffffffffu, b < of ? (unsigned)n : 0u);
      units += __popc(__ballot_sync(0xffffffffu, n > 0));
      longest = max(longest, (int)__reduce_max_sync(0xffffffffu, (unsigned)n));
    }
    before *= p.tile_heads;
    cut = prompt_cut(tiles * p.tile_heads, units * p.tile_heads, longest, p.cut_ctas);
  }
};

// A warp's walk over the batch's units.  Batches of up to 32 sequences are in registers, one a lane (one sequence
// alone in every lane); lane l also keeps how many blocks have level l or a higher one.
struct Units {
  PromptSequence mine;
  PromptCursor cur;
  int from_level;
  PromptCut cut;                      // by the lengths
  int share, begin, at, end;          // the share last asked for: its key tiles, and the next of them
  int b0, before;                     // the sequence group of `at`, and the key tiles before it
  bool bad;   // some sequence is out of range (of those that the lane has looked at)
  __device__ __forceinline__ Units(const PromptAttnParams& p)
      : mine{0, 0, 0, {0, 0}}, cur{0, 0, 0, 0, 0}, from_level(0), cut{0, 0}, share(-1), bad(false) {
    const int lane = threadIdx.x & 31, m = lane * p.level_step;
    if (p.batch == 1 || lane < p.batch) mine = load_sequence(p, p.batch == 1 ? 0 : lane, bad);
    if (p.cut_ctas > 0) cut = LengthCut(p, mine, 0, bad).cut;
    if (!prompt_has_levels(p.batch) || cut.shares > 0) {
#pragma unroll 1
      for (int b = lane + 32; p.cut_ctas == 0 && b < p.batch; b += 32) load_sequence(p, b, bad);
      return;
    }
#pragma unroll 1
    for (int b0 = 0; b0 < p.batch; b0 += 32) {
      PromptSequence s = mine;
      if (b0 > 0) s = b0 + lane < p.batch ? load_sequence(p, b0 + lane, bad) : PromptSequence{0, 0, 0, {0, 0}};
#pragma unroll 1
      for (int i = 0; i < min(32, p.batch - b0); ++i)
        from_level += blocks_from({__shfl_sync(0xffffffffu, s.blocks.first, i), __shfl_sync(0xffffffffu, s.blocks.count, i)}, m);
    }
  }
  // The next unit of share x.
  __device__ __forceinline__ bool next(const PromptAttnParams& p, int x, Unit& u) {
    if (x >= cut.shares) return false;
    if (x != share) {
      share = x;
      begin = at = share_begin(x, cut);
      end = share_begin(x + 1, cut);
      b0 = before = 0;
    }
    if (at >= end) return false;
#pragma unroll 1
    for (;; b0 += 32) {
      const int b = b0 + (threadIdx.x & 31);
      PromptSequence s = {0, 0, 0, {0, 0}};
      if (b < p.batch) s = p.batch <= 32 ? mine : load_sequence(p, b, bad);
      const int t = sequence_tiles(p, s), upto = before + WarpLanes{}.scan(t * p.tile_heads);
      const int src = WarpLanes{}.first(at < upto);
      if (src < 0) {
        before = __shfl_sync(0xffffffffu, upto, 31);
        if (b0 + 32 >= p.batch) return false;
        continue;
      }
      const int n = __shfl_sync(0xffffffffu, t, src), in = at - (__shfl_sync(0xffffffffu, upto, src) - n * p.tile_heads);
      const int tile = (int)((uint32_t)in / (uint32_t)n);
      u.b = b0 + src;
      u.ctx = __shfl_sync(0xffffffffu, s.ctx, src);
      u.token0 = 0;
      u.tokens = __shfl_sync(0xffffffffu, s.tokens, src);
      u.row0 = __shfl_sync(0xffffffffu, s.row0, src);
      u.head0 = tile * p.sub;
      u.kv = divide(tile, p.by_kv);
      u.tile0 = in - tile * n;
      u.tile1 = min(n, u.tile0 + end - at);
      u.whole = u.tile0 == 0 && u.tile1 == n;
      u.place = 2 * x + (at > begin ? 1 : 0);
      at += u.tile1 - u.tile0;
      return true;
    }
  }
  __device__ __forceinline__ bool more(int x) const { return x == share && at < end; }   // of share x (share -1: none)
  // Unit number x: piece x % splits of block (x / splits) / tile_heads of the batch under head tile (x / splits) %
  // tile_heads (every lane gets it).  False: there is none.
  __device__ __forceinline__ bool find(const PromptAttnParams& p, int x, Unit& u) {
    if (cut.shares > 0) return next(p, x, u);
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
