// Geometry of packed batches of new tokens (internal; also compiled as plain C++): which sequences are
// valid, and how the attention's work units are numbered.
#pragma once

#include <cstdint>

#include "row_division.cuh"

#ifdef __CUDACC__
#define PTD_HD __host__ __device__ __forceinline__
#else
#define PTD_HD inline
#endif

namespace ptd {

struct PromptBounds {
  int n_total, max_tokens, max_ctx;
  int64_t capacity;   // positions that a sequence's cache row holds
};

// Whether sequence [off0, off1) with context `ctx` keeps within the batch's and the cache's bounds.
PTD_HD bool prompt_sequence_ok(const PromptBounds& p, int off0, int off1, int ctx) {
  return off0 >= 0 && off1 >= off0 && off1 <= p.n_total && off1 - off0 <= p.max_tokens && ctx >= 0 && ctx <= p.max_ctx &&
         (int64_t)ctx + (off1 - off0) <= p.capacity;
}

// A sequence's blocks of `width` tokens, as the attention orders them: block i of a sequence has the key
// first + i, first = ctx / width, which grows with the keys it sees.
struct PromptBlocks {
  int first, count;
};
PTD_HD PromptBlocks prompt_blocks(int ctx, int tokens, int width, IndexDivisor by_width) {
  return {divide(ctx, by_width), divide(tokens + width - 1, by_width)};
}

// Blocks of one sequence with key >= m.
PTD_HD int blocks_from(const PromptBlocks& s, int m) {
  const int c = s.first + s.count - m;
  return c < 0 ? 0 : (c > s.count ? s.count : c);
}

// A sequence of the batch: its first row and number of new tokens, context and blocks (none if out of range).
struct PromptSequence {
  int row0, tokens, ctx;
  PromptBlocks blocks;
};

// Where a sequence's first block lies among the batch's partials, counted in blocks; its others follow.  The places
// of different blocks differ (a sequence of c blocks takes more than (c - 1) * width rows, and the sequence number
// adds one), and are below prompt_places: the first row of the last sequence's last block is below n_total.
PTD_HD int block_place(int row0, int b, IndexDivisor by_width) { return divide(row0, by_width) + b; }
PTD_HD int64_t prompt_places(int n_total, int batch, int width) { return (int64_t)n_total / width + batch; }

// The blocks of a batch are numbered by level, highest first: a block's level is its key / level_step, 32 levels
// in all (the long ones first, so that what is taken last is short).  Within a level they go by sequence, and
// a sequence's by falling key.  Batches of more than kOrderedBatch sequences have one level: their many
// blocks even out, and the levels would cost a walk over the batch each.
constexpr int kLevels = 32;
constexpr int kOrderedBatch = 128;
PTD_HD int prompt_level_step(int max_ctx, int max_tokens, int width) { return (max_ctx / width + max_tokens / width + 2) / kLevels + 1; }

PTD_HD bool prompt_has_levels(int batch) { return batch > 1 && batch <= kOrderedBatch; }

// Batches of few units may be cut by the lengths on the device, so that the SMs' work evens out.  A unit takes a cell a key
// tile, and some more for its start and end; the cells of all units, sequence after sequence, block after block and head
// tile after head tile, go in equal shares, one a CTA.  A unit whose key tiles are not in one share has partials, at
// place 2 c if it begins share c, else 2 c + 1.
struct PromptCut {
  int shares, cells;   // shares 0: the units are better left whole
};
constexpr int kMostCutCtas = 255, kMostCutCells = 1 << 24;   // their product stays in 32 bits
struct CutCosts {      // in cells
  int merge, unit;     // of a CTA's partials of a unit and their merge; of a unit besides its key tiles
};

// The cut for `ctas` CTAs at a time into at most `most` shares: `cells` of `units` units (at most two rounds of them), the
// longest and the shortest of `longest` and `shortest` cells.  Whole units take the longest, or two of the mean or what is
// even and a short one.
PTD_HD PromptCut prompt_cut(int cells_, int units_, int longest_, int shortest_, int ctas_, int most, CutCosts costs) {
  const uint32_t cells = (uint32_t)cells_, units = (uint32_t)units_, ctas = (uint32_t)ctas_;
  if (cells < 2u || most < 1 || cells > (uint32_t)kMostCutCells) return {0, cells_};   // (more: sequences that overlap)
  uint32_t whole = 8u * (uint32_t)longest_;
  if (units > ctas) {
    const uint32_t two = 16u * cells / units, last = 8u * cells / ctas + 8u * (uint32_t)shortest_;
    const uint32_t less = two < last ? two : last;
    whole = whole > less ? whole : less;
  }
  const uint32_t shares = cells / 2u < (uint32_t)most ? cells / 2u : (uint32_t)most;
  const uint32_t even = 8u * ((uint32_t)(costs.merge + costs.unit)) + 8u * (cells + (uint32_t)costs.merge * units) / shares;
  return {even < whole ? (int)shares : 0, cells_};
}
PTD_HD int share_begin(int c, const PromptCut& cut) { return (int)((uint32_t)c * (uint32_t)cut.cells / (uint32_t)cut.shares); }
PTD_HD int share_of(int x, const PromptCut& cut) {   // the share that has cell x
  return (int)((((uint32_t)x + 1u) * (uint32_t)cut.shares - 1u) / (uint32_t)cut.cells);
}

// Turns of the attention's two issuers (prompt_attention_tc.cu).  M tile t's products of key tile j wait for its softmax
// and for a turn, told on one barrier; `both` is how many key tiles of the unit both M tiles have.  While both have
// products, M tile 1's of tile j come after 0's, and 0's of tile j + 1 after 1's of tile j; a turn that waits for nobody is
// the issuer's own.  Within a unit every turn passed to the other is asked for by a turn got from it, so that it cannot
// come early.  The first one of a unit is not: M tile 1 may still wait for its softmax in the unit before, whose barrier would
// count the turn in place of a softmax warp.  So issuer 1 tells that it has begun a unit with turns, and issuer 0 waits
// for that before its first product with V (it waits for M tile 0's softmax then anyway).
PTD_HD bool own_turn(int t, int j, int both) { return t == 0 ? j == 0 || j >= both : j >= both; }
PTD_HD bool passes_turn(int t, int j, int both) { return t == 0 ? j < both : j + 1 < both; }
PTD_HD bool tells_entry(int t, int both) { return t == 1 && both > 0; }
PTD_HD bool awaits_entry(int t, int both) { return t == 0 && both > 0; }

// Where the last search ended: a search for a later block goes on from there.
struct PromptCursor {
  int level, upto, above;   // a level, the blocks of it and higher ones, and of higher ones (upto 0: none known)
  int b0, before;           // a sequence, and the blocks of the level in the sequences before it
};

// Block number u: its sequence b, that sequence, and the block's place in it.  `lanes` walks the sequences: one
// lane on the host, a warp's 32 on the device, where every lane gets the answer; load(b) gives sequence b and
// is called with b = lane modulo their number; level_of(u, upto, above) gives u's level, the blocks of it and
// higher levels (upto > u where there is such a block) and of higher ones.  False: there is no such block.
template <typename Lanes, typename Load, typename LevelOf>
PTD_HD bool find_prompt_block(const Lanes& lanes, const Load& load, const LevelOf& level_of, int batch, int level_step, int u,
                              PromptCursor& cur, int& b_out, int& i_out, PromptSequence& seq_out) {
  if (u < 0) return false;
  if (batch == 1) {
    seq_out = load(0);
    b_out = 0;
    i_out = seq_out.blocks.count - 1 - u;
    return i_out >= 0;
  }
  const bool levels = prompt_has_levels(batch);
  if (levels && (u >= cur.upto || u < cur.above)) {
    cur.b0 = cur.before = 0;
    cur.level = level_of(u, cur.upto, cur.above);
  }
  const int level = cur.level, left = u - cur.above;
  if (cur.before > left) cur.b0 = cur.before = 0;
  const int m0 = level * level_step, m1 = levels && level + 1 < kLevels ? m0 + level_step : INT32_MAX;
#pragma unroll 1
  for (; cur.b0 < batch; cur.b0 += lanes.count()) {
    const int b = cur.b0 + lanes.id();
    PromptSequence s = {0, 0, 0, {0, 0}};
    if (b < batch) s = load(b);
    const int n = levels ? blocks_from(s.blocks, m0) - blocks_from(s.blocks, m1) : s.blocks.count;
    const int upto = cur.before + lanes.scan(n);
    const int src = lanes.first(left < upto);
    if (src >= 0) {
      seq_out = {lanes.get(s.row0, src), lanes.get(s.tokens, src), lanes.get(s.ctx, src),
                 {lanes.get(s.blocks.first, src), lanes.get(s.blocks.count, src)}};
      const int behind = left - (lanes.get(upto, src) - lanes.get(n, src));   // blocks of its own before u
      const int end = seq_out.blocks.first + seq_out.blocks.count;
      b_out = cur.b0 + src;
      i_out = (end < m1 ? end : m1) - 1 - seq_out.blocks.first - behind;
      return true;
    }
    cur.before = lanes.get(upto, lanes.count() - 1);
  }
  return false;
}

struct OneLane {
  PTD_HD int id() const { return 0; }
  PTD_HD int count() const { return 1; }
  PTD_HD int scan(int x) const { return x; }
  PTD_HD int first(bool p) const { return p ? 0 : -1; }
  PTD_HD int get(int x, int) const { return x; }
};

#ifdef __CUDACC__
struct WarpLanes {
  __device__ __forceinline__ int id() const { return threadIdx.x & 31; }
  __device__ __forceinline__ int count() const { return 32; }
  __device__ __forceinline__ int scan(int x) const {   // inclusive
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, o);
      if (id() >= o) x += y;
    }
    return x;
  }
  __device__ __forceinline__ int first(bool p) const { return __ffs(__ballot_sync(0xffffffffu, p)) - 1; }
  __device__ __forceinline__ int get(int x, int lane) const { return __shfl_sync(0xffffffffu, x, lane); }
};
#endif

}  // namespace ptd
