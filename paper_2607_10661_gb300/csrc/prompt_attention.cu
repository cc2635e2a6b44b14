// Prompt attention: the choice of tiles and of the cut of the keys, and the merge of the pieces.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>

#include "launch.cuh"
#include "prompt_attention.cuh"
#include "ptd_device.cuh"

namespace ptd {
namespace pa {

constexpr int kMergeThreads = 256;

// The pieces of a block: the first has its partials at place `first`, piece s at rest + s * step.
struct Pieces {
  int count;
  size_t first, rest;
  int step;
};

// Part `part` of `parts` of the merge of a block (its first row in out row0, head tile `tile`): a thread takes a row and four
// columns of kAt blocks of elements at a time, kPieces pieces of each, all of whose loads are in flight together.
template <typename T, int kAt, int kPieces>
__device__ __forceinline__ void merge_part(const PromptAttnParams& p, const Pieces& from, int row0, int tokens, int tile, int part,
                                           int parts) {
  const int rows = tokens * p.sub, groups = p.head_dim / 4, used = p.tile_tokens * p.sub;
  const int block_rows = p.block_tokens / p.tile_tokens * p.tile_rows, apart = parts * kMergeThreads;
#pragma unroll 1
  for (int e0 = part * kMergeThreads + threadIdx.x; e0 < rows * groups; e0 += kAt * apart) {
    const float2* ml[kAt];
    const float4* po[kAt];
    float M[kAt], L[kAt];
    float4 acc[kAt];
#pragma unroll
    for (int k = 0; k < kAt; ++k) {
      const int e = min(e0 + k * apart, rows * groups - 1), c = e / rows, r = e - c * rows;   // (behind the last: the last)
      const int at = r < used ? r : p.tile_rows + r - used;
      ml[k] = reinterpret_cast<const float2*>(p.part_ml) + at;
      po[k] = reinterpret_cast<const float4*>(p.part_o) + (size_t)c * block_rows + at;
      M[k] = -INFINITY, L[k] = 0.f;
      acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    for (int s0 = 0; s0 < from.count; s0 += kPieces) {
      float2 x[kAt][kPieces];
      float4 o[kAt][kPieces];
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
        const bool there = s0 + i < from.count;
        const size_t piece = s0 + i == 0 ? from.first : from.rest + (size_t)(s0 + i) * from.step;
#pragma unroll
        for (int k = 0; k < kAt; ++k) {
          x[k][i] = there ? __ldcg(ml[k] + piece * block_rows) : make_float2(-INFINITY, 0.f);
          if (there) o[k][i] = __ldcg(po[k] + piece * groups * block_rows);
        }
      }
#pragma unroll
      for (int k = 0; k < kAt; ++k) {
        float m = M[k];
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
          if (!(x[k][i].y == 0.f)) m = fmaxf(m, x[k][i].x);   // (not l > 0: a NaN among the scores has to reach the output)
        const float old = M[k] == -INFINITY ? 0.f : exp2f(M[k] - m);
        M[k] = m;
        L[k] *= old, acc[k].x *= old, acc[k].y *= old, acc[k].z *= old, acc[k].w *= old;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
          if (x[k][i].y == 0.f) continue;
          const float w = exp2f(x[k][i].x - m);
          L[k] += w * x[k][i].y;
          acc[k].x += w * o[k][i].x;
          acc[k].y += w * o[k][i].y;
          acc[k].z += w * o[k][i].z;
          acc[k].w += w * o[k][i].w;
        }
      }
    }
#pragma unroll
    for (int k = 0; k < kAt; ++k) {
      const int e = e0 + k * apart, c = e / rows, r = e - c * rows;
      if (e >= rows * groups) break;
      const float inv = 1.f / L[k];
      const int token = divide(r, p.by_sub), head = tile * p.sub + r - token * p.sub;
      T* dst = static_cast<T*>(p.out) + ((size_t)(row0 + token) * p.hq + head) * p.head_dim + c * 4;
      if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<uint2*>(dst) =
            make_uint2(pack_bf16x2(acc[k].x * inv, acc[k].y * inv), pack_bf16x2(acc[k].z * inv, acc[k].w * inv));
      } else {
        *reinterpret_cast<float4*>(dst) = make_float4(acc[k].x * inv, acc[k].y * inv, acc[k].z * inv, acc[k].w * inv);
      }
    }
  }
}

// The rows of one split block (by pieces of one length, or by the lengths on the device), from its pieces:
// O = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s, M the maximum of the m_s (a row that saw no key of a piece has l_s = 0,
// and its O_s was not written).  x of the grid is
// a block's place and head tile, or a boundary between shares of the cells, y a share of its rows and columns;
// consecutive threads take consecutive rows, as the partials lie.  Bound by the latency of the chain sequence, (m, l),
// partials; the sequence is found before the wait for the attention.
template <typename T, bool kMany>
__global__ void __launch_bounds__(kMergeThreads, kMany ? 2 : 1) prompt_merge_kernel(const PromptAttnParams p) {
  if (threadIdx.x == 0) grid_launch_dependents();
  // (the attention lets this grid be placed after its own wait, so that the batch's arrays are complete in L2, where
  // load_sequence reads them; waiting first costs 0.5 us: eight contexts of 4096 24.75 -> 25.3)
  const int lane = threadIdx.x & 31;
  int tile = 0, row0 = 0, tokens = 0, ctx = 0;
  bool bad = false, found = false;
  Pieces from = {0, 0, 0, 1};
  int part = blockIdx.y, parts = gridDim.y;
  if (p.cut_ctas > 0) {        // x: a boundary between shares; the boundaries that cut a unit share its merge
    PromptSequence mine = {0, 0, 0, {0, 0}};
    if (lane < p.batch) mine = load_sequence(p, lane, bad);
    const PromptCut cut = cut_by_lengths(p, mine, bad);
    const int c = (int)blockIdx.x, at = c + 1 < cut.shares ? share_begin(c + 1, cut) : 0;
    int b0 = 0, before = 0;
    CutUnit u;
    if (at > 0 && find_cut_unit(p, mine, at, b0, before, u) && at > u.first && at < u.first + u.tiles) {
      tile = u.head;
      row0 = u.s.row0 + u.i * p.block_tokens;
      tokens = min(p.block_tokens, u.s.tokens - u.i * p.block_tokens);
      const int c0 = share_of(u.first, cut), count = share_of(u.first + u.tiles - 1, cut) - c0 + 1;
      from = {count, 2 * (size_t)c0 + (share_begin(c0, cut) < u.first ? 1 : 0), 2 * (size_t)c0, 2};
      found = true;
      part += (c - c0) * (int)gridDim.y;
      parts *= count - 1;
    }
  } else {
    const int place = divide((int)blockIdx.x, p.by_heads);
    tile = (int)blockIdx.x - place * p.tile_heads;
    for (int b0 = 0; b0 < p.batch && !found; b0 += 32) {   // every warp looks for the sequence
      const int b = b0 + lane;
      PromptSequence s = {0, 0, 0, {0, 0}};
      if (b < p.batch) s = load_sequence(p, b, bad);
      const int i = place - block_place(s.row0, b, p.by_block);
      const int src = WarpLanes{}.first(i >= 0 && i < s.blocks.count);
      if (src < 0) continue;
      found = true;
      const int at = __shfl_sync(0xffffffffu, i, src) * p.block_tokens;
      row0 = __shfl_sync(0xffffffffu, s.row0, src) + at;
      tokens = min(p.block_tokens, __shfl_sync(0xffffffffu, s.tokens, src) - at);
      ctx = __shfl_sync(0xffffffffu, s.ctx, src) + at;
    }
  }
  grid_dependency_wait();   // the partials belong to the attention
  if (!found) return;
  if (p.cut_ctas == 0) {
    from.count = (((ctx + tokens + p.key_tile - 1) >> p.key_tile_log2) + p.piece_tiles - 1) / p.piece_tiles;
    from.first = from.rest = (size_t)blockIdx.x * p.splits;
  }
  if (from.count <= 1) return;   // written by the attention
  if (kMany && from.count == 2)
    merge_part<T, 4, 2>(p, from, row0, tokens, tile, part, parts);
  else
    merge_part<T, 1, 8>(p, from, row0, tokens, tile, part, parts);
}

// The largest divisor of `group` that is at most `most`.
int largest_divisor(int group, int most) {
  for (int d = group < most ? group : most; d > 1; --d)
    if (group % d == 0) return d;
  return 1;
}

// Key tiles per piece: all of them (uncut) where the units fill `slots` places, else as many pieces of the longest
// sequence as give every place one; one more where that is two or three and the batch may be ragged.
int choose_piece(int64_t units, int64_t key_tiles, int batch, int64_t slots) {
  if (units == 0 || units >= slots || key_tiles < 2) return (int)key_tiles;
  int64_t pieces = slots / units;
  if (batch > 1 && (pieces == 2 || pieces == 3)) ++pieces;
  return (int)((key_tiles + pieces - 1) / pieces);
}

// Tiles, blocks and the cut, for blocks of `tiles` M tiles of tile_rows rows, on `slots` places.
void plan_tiles(PromptAttnParams& p, int tile_rows, int tiles, int key_tile_log2, int64_t slots) {
  const int group = p.hq / p.hkv;
  p.tile_rows = tile_rows;
  p.key_tile_log2 = key_tile_log2;
  p.key_tile = 1 << key_tile_log2;
  p.sub = largest_divisor(group, tile_rows);
  p.tile_heads = p.hq / p.sub;
  p.tiles_per_kv = group / p.sub;
  p.tile_tokens = tile_rows / p.sub;
  p.block_tokens = tiles * p.tile_tokens;
  p.by_block = index_divisor(p.block_tokens);
  p.by_heads = index_divisor(p.tile_heads);
  p.by_kv = index_divisor(p.tiles_per_kv);
  p.by_sub = index_divisor(p.sub);
  p.level_step = prompt_level_step(p.bounds.max_ctx, p.bounds.max_tokens, p.block_tokens);
  const int64_t places = prompt_places(p.bounds.n_total, p.batch, p.block_tokens);
  const int64_t longest = (int64_t)p.batch * ((p.bounds.max_tokens + p.block_tokens - 1) / p.block_tokens);
  p.blocks = (int)(places < longest ? places : longest);
  p.places = (int)places;
  const int64_t key_tiles = ((int64_t)p.bounds.max_ctx + p.bounds.max_tokens + p.key_tile - 1) >> key_tile_log2;
  p.piece_tiles = choose_piece((int64_t)p.blocks * p.tile_heads, key_tiles, p.batch, slots);
  p.splits = (int)((key_tiles + p.piece_tiles - 1) / p.piece_tiles);
}
}  // namespace pa

size_t plan_prompt_attention(PromptAttnParams& p, bool bf16, size_t scratch, int sms) {
  p.cut_ctas = 0;
  if (bf16) {
    // A CTA an SM.  All figures here are us of a call in graph replays, 32/8 heads unless said, pages of 16.
    // One sequence of one block: pieces of one length, by the bounds (its length is not looked at: one token after
    // 4096 takes 11.8 with that bound and 50.6, uncut, with one of 131072).  By how many pieces, the rule's in brackets:
    //   one token after 4096 (8 units of 33 key tiles)   1: 49.7, 4: 19.5, 8: 14.1, [17: 11.8]
    //   one token after 32768                            10: 45.2, 14: 35.9, 17: 33.1, [19: 31.9], 20 (over a wave): 45.7
    //   60 tokens after 500                              1: 13.7, 2: 14.9, 3: 13.9, [5: 12.9]
    pa::plan_tiles(p, 128, 2, 7, sms);
    // Else by the lengths on the device, if the host's bounds allow for a gain, or uncut.  A cell is the time of a key tile
    // (~1.2 us); what a cut unit's partials and merge and any unit's start and end cost in cells (p.costs), and the
    // bound on the key tiles, are fitted to these cases.
    //   cut by the rule [uncut]: one token behind 8 ragged contexts up to 4096 23.5 [50.8], 8 equal ones 31.2 [52.0], 12 ragged
    //     31.7 [52.1], 16 ragged up to 8000 60.6 [93.7], 24 of 8000 128 [185], 32 of 4000 90.1 [99.4], 2 of 2000 12.6 [27.7]; 8
    //     tokens after 8000 beside a prompt of 512 28.6 [91.4], 4 after 16000 beside it 32.4 [177], 2 chunks of 256 after
    //     8192 67.4 [107], 61 tokens of 64/8 heads after 32707 58.8 [390], 200 tokens after 1900 25.2 [31.8].
    //   uncut by the rule [cut]: 200 tokens after 1000 21.4 [23.2], 2 of 200 after 500 16.2 [18.1], 400 after 700 20.3 [21.9],
    //     800 after 700 24.5 [26.7].
    //   what it loses: 400 tokens after 1500 32.9 [29.3], 800 after 1500 35.8 [33.5], and the merge's launch where the
    //     device leaves the units whole: 18 contexts of 2000 31.4 [30.0].
    // More than two rounds of units are never cut: 40 contexts of 4000 (320 units) 147.
    const int64_t units = (int64_t)p.blocks * p.tile_heads;
    const int64_t key_tiles = ((int64_t)p.bounds.max_ctx + p.bounds.max_tokens + p.key_tile - 1) >> p.key_tile_log2;
    if (p.batch > 1 || p.bounds.max_tokens > p.block_tokens) {
      p.piece_tiles = (int)key_tiles;
      p.splits = 1;
      p.by_splits = index_divisor(1);
      const int used = (p.bounds.max_tokens < p.block_tokens ? p.bounds.max_tokens : p.block_tokens) * p.sub;   // rows
      p.costs = {used * 6 / 256, 1 + used / 128};
      if (units > 2 * (int64_t)sms || key_tiles <= p.costs.merge + p.costs.unit + (units > sms ? 14 : 3) || sms > kMostCutCtas ||
          units * (key_tiles + p.costs.unit) > kMostCutCells)
        return 0;
      const int64_t cells = units * (key_tiles + p.costs.unit);
      p.most_shares = (int)(cells / 2 < sms ? cells / 2 : sms);
      const size_t rows = 2 * (size_t)p.most_shares * 256, bytes = rows * (p.head_dim + 2) * sizeof(float);
      if (bytes > scratch) return 0;
      p.cut_ctas = sms;
      p.part_ml = p.part_o + rows * p.head_dim;
      return bytes;
    }
  } else if ((int64_t)p.bounds.max_tokens * (p.hq / p.hkv) <= 16) {
    // Blocks of 16 rows, four CTAs an SM: one token after 2000 in four sequences of 8 heads, D = 64, 28.5 us (blocks
    // of 64 rows 32.3); pieces of 1: 30.5, [2: 28.5], 4: 37.0, 8: 52.
    pa::plan_tiles(p, 16, 1, 6, 4 * (int64_t)sms);
  } else {
    // Blocks of 64 rows, one CTA an SM for D = 128, else two; prompts see half of their keys on average, so that twice
    // the pieces are asked for.  500 tokens of 8 heads, D = 64, [1: 19], 2: 25, 4: 40; 50 tokens after 1500 of 32/8 heads,
    // D = 128, 3: 68, 6: 59, [7: 66], 10: 92.  (128 rows a block: 2048 tokens of 8 heads, D = 64, 254 us, 64 rows 236;
    // D = 128, 452 and 266.)
    const int64_t slots = (p.head_dim == 128 ? 1 : 2) * (int64_t)sms;
    pa::plan_tiles(p, 64, 1, 6, p.bounds.max_tokens > p.bounds.max_ctx ? 2 * slots : slots);
  }
  const size_t rows = (size_t)p.places * p.tile_heads * p.splits * (p.block_tokens / p.tile_tokens) * p.tile_rows;
  const size_t bytes = p.splits == 1 ? 0 : rows * (p.head_dim + 2) * sizeof(float);
  if (bytes > scratch) {
    p.piece_tiles *= p.splits;
    p.splits = 1;
  }
  p.by_splits = index_divisor(p.splits);
  if (p.splits == 1) return 0;
  p.part_ml = p.part_o + rows * p.head_dim;
  return bytes;
}

cudaError_t launch_prompt_attn_merge(const PromptAttnParams& p, bool bf16, cudaStream_t stream) {
  const int64_t rows = (int64_t)(p.bounds.max_tokens < p.block_tokens ? p.bounds.max_tokens : p.block_tokens) * p.sub;
  const unsigned shares = (unsigned)((rows * (p.head_dim / 4) + pa::kMergeThreads - 1) / pa::kMergeThreads);
  const bool many = p.cut_ctas > 0 && shares > 4;
  const auto kernel = !bf16 ? pa::prompt_merge_kernel<float, false>
                            : many ? pa::prompt_merge_kernel<__nv_bfloat16, true> : pa::prompt_merge_kernel<__nv_bfloat16, false>;
  const int blocks = p.cut_ctas > 0 ? p.most_shares : p.places * p.tile_heads;
  return launch_chained(kernel, dim3((unsigned)blocks, p.cut_ctas > 0 ? (shares + 15) / 16 : shares), dim3(pa::kMergeThreads), 0, stream, 0, p);
}

}  // namespace ptd
