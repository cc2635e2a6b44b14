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

// Key tiles of a unit of block i of a sequence, and cells of all its blocks under one head tile.
__device__ __forceinline__ int block_tiles(const PromptAttnParams& p, const PromptSequence& s, int i) {
  return (s.ctx + min((i + 1) * p.block_tokens, s.tokens) + p.key_tile - 1) >> p.key_tile_log2;
}
__device__ __forceinline__ int sequence_cells(const PromptAttnParams& p, const PromptSequence& s) {
  int n = 0;
#pragma unroll 1
  for (int i = 0; i < s.blocks.count; ++i) n += block_tiles(p, s, i) + p.costs.unit;
  return n;
}

// The cut of the batch by its lengths (prompt_geometry.cuh); `mine` is sequence `lane`.  Warp-collective.
__device__ __forceinline__ PromptCut cut_by_lengths(const PromptAttnParams& p, const PromptSequence& mine, bool& bad) {
  int units = 0, longest = 0, shortest = kMostCutCells, cells = 0;
#pragma unroll 1
  for (int b0 = 0; b0 < p.batch; b0 += 32) {
    const int b = b0 + (threadIdx.x & 31);
    PromptSequence s = mine;
    if (b0 > 0 && b < p.batch) s = load_sequence(p, b, bad);
    if (b >= p.batch) s.blocks.count = 0;
    units += s.blocks.count;
    cells += sequence_cells(p, s);
    if (s.blocks.count > 0) {
      longest = max(longest, block_tiles(p, s, s.blocks.count - 1) + p.costs.unit);
      shortest = min(shortest, block_tiles(p, s, 0) + p.costs.unit);
    }
  }
  units = (int)__reduce_add_sync(0xffffffffu, (unsigned)units);
  cells = (int)__reduce_add_sync(0xffffffffu, (unsigned)cells);
  longest = (int)__reduce_max_sync(0xffffffffu, (unsigned)longest);
  shortest = (int)__reduce_min_sync(0xffffffffu, (unsigned)shortest);
  return prompt_cut(cells * p.tile_heads, units * p.tile_heads, longest, shortest, p.cut_ctas, p.most_shares, p.costs);
}

// The unit of a cell: sequence, block, head tile, its first cell and how many key tiles it has.
struct CutUnit {
  int b, i, head, first, tiles;
  PromptSequence s;
};
// Of cell `at`; b0 and before (0 at first): a group of 32 sequences and the cells before it, moved on.  False: there is
// none.  Warp-collective.
__device__ __forceinline__ bool find_cut_unit(const PromptAttnParams& p, const PromptSequence& mine, int at, int& b0, int& before,
                                              CutUnit& u) {
#pragma unroll 1
  for (;; b0 += 32) {
    const int b = b0 + (threadIdx.x & 31);
    bool bad = false;
    PromptSequence s = mine;
    if (b0 > 0 && b < p.batch) s = load_sequence(p, b, bad);
    if (b >= p.batch) s.blocks.count = 0;
    const int n = sequence_cells(p, s) * p.tile_heads, upto = before + WarpLanes{}.scan(n);
    const int src = WarpLanes{}.first(at < upto);
    if (src < 0) {
      if (b0 + 32 >= p.batch) return false;
      before = __shfl_sync(0xffffffffu, upto, 31);
      continue;
    }
    u.b = b0 + src;
    u.s = {__shfl_sync(0xffffffffu, s.row0, src), __shfl_sync(0xffffffffu, s.tokens, src), __shfl_sync(0xffffffffu, s.ctx, src),
           {__shfl_sync(0xffffffffu, s.blocks.first, src), __shfl_sync(0xffffffffu, s.blocks.count, src)}};
    u.first = __shfl_sync(0xffffffffu, upto - n, src);
    u.tiles = block_tiles(p, u.s, 0);
    u.i = 0;
    int cells = u.tiles + p.costs.unit;
#pragma unroll 1
    while (at >= u.first + cells * p.tile_heads) {   // (ends: the sequence has `at`)
      u.first += cells * p.tile_heads;
      u.tiles = block_tiles(p, u.s, ++u.i);
      cells = u.tiles + p.costs.unit;
    }
    u.head = (int)((uint32_t)(at - u.first) / (uint32_t)cells);
    u.first += u.head * cells;
    return true;
  }
}

// A warp's walk over the batch's units.  Batches of up to 32 sequences are in registers, one a lane (one sequence
// alone in every lane); lane l also keeps how many blocks have level l or a higher one.
struct Units {
  PromptSequence mine;
  PromptCursor cur;
  int from_level;
  PromptCut cut;                      // by the lengths
  int share, begin, at, end;          // the share last asked for: its cells, and the next of them
  int b0, before;                     // the sequence group of `at`, and the cells before it
  bool bad;   // some sequence is out of range (of those that the lane has looked at)
  __device__ __forceinline__ Units(const PromptAttnParams& p)
      : mine{0, 0, 0, {0, 0}}, cur{0, 0, 0, 0, 0}, from_level(0), cut{0, 0}, share(-1), bad(false) {
    const int lane = threadIdx.x & 31, m = lane * p.level_step;
    if (p.batch == 1 || lane < p.batch) mine = load_sequence(p, p.batch == 1 ? 0 : lane, bad);
    if (p.cut_ctas > 0) cut = cut_by_lengths(p, mine, bad);
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
    CutUnit w;
    do {
      if (at >= end || !find_cut_unit(p, mine, at, b0, before, w)) return false;
      u.tile0 = at - w.first;
      u.tile1 = min(w.tiles, u.tile0 + end - at);
      u.place = 2 * x + (at > begin ? 1 : 0);
      at = w.first + w.tiles + p.costs.unit;
    } while (u.tile1 <= u.tile0);   // the share begins behind the unit's key tiles
    u.b = w.b;
    u.ctx = w.s.ctx;
    u.token0 = w.i * p.block_tokens;
    u.tokens = min(p.block_tokens, w.s.tokens - u.token0);
    u.row0 = w.s.row0 + u.token0;
    u.head0 = w.head * p.sub;
    u.kv = divide(w.head, p.by_kv);
    u.whole = u.tile0 == 0 && u.tile1 == w.tiles;
    return true;
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
