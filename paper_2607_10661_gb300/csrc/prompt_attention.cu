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
constexpr int kMergeBatch = 8;   // pieces whose partials are in flight at a time

// The rows of one split block (by pieces of one length, or by the lengths on the device), from its pieces: O = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s, M the
// maximum of the m_s (a row that saw no key of a piece has l_s = 0, and its O_s was not written).  x of the grid is
// a block's place and head tile, y a share of its rows and columns: a thread takes one row and four columns,
// consecutive threads consecutive rows, as the partials lie.  Bound by the latency of the chain sequence, (m, l),
// partials; the sequence is found before the wait for the attention.
template <typename T>
__global__ void __launch_bounds__(kMergeThreads) prompt_merge_kernel(const PromptAttnParams p) {
  if (threadIdx.x == 0) grid_launch_dependents();
  // (the attention lets this grid be placed after its own wait, so that the batch's arrays are complete in L2, where
  // load_sequence reads them; waiting first costs 0.5 us: eight contexts of 4096 24.75 -> 25.3)
  const int lane = threadIdx.x & 31;
  const int place = divide((int)blockIdx.x, p.by_heads), tile = (int)blockIdx.x - place * p.tile_heads;
  int row0 = 0, tokens = 0, ctx = 0;
  bool bad = false, found = false;
  int pieces = 0;              // of the block: the first at place `first`, piece s at rest + s * step
  size_t first = 0, rest = 0;
  int step = 1;
  if (p.cut_ctas > 0) {        // (place: the sequence)
    PromptSequence s = {0, 0, 0, {0, 0}};
    if (lane < p.batch) s = load_sequence(p, lane, bad);
    const LengthCut by_lengths(p, s, place, bad);
    const PromptCut cut = by_lengths.cut;
    s = load_sequence(p, place, bad);
    row0 = s.row0, tokens = s.tokens, ctx = s.ctx;
    const int n = sequence_tiles(p, s), x = by_lengths.before + tile * n;
    if (cut.shares > 0 && n > 0) {
      const int c = share_of(x, cut);
      pieces = share_of(x + n - 1, cut) - c + 1;
      found = true;
      rest = 2 * (size_t)c, step = 2;
      first = rest + (share_begin(c, cut) < x ? 1 : 0);
    }
  } else {
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
    pieces = (((ctx + tokens + p.key_tile - 1) >> p.key_tile_log2) + p.piece_tiles - 1) / p.piece_tiles;
    first = rest = (size_t)blockIdx.x * p.splits;
  }
  if (pieces <= 1) return;   // written by the attention
  const int rows = tokens * p.sub, groups = p.head_dim / 4, used = p.tile_tokens * p.sub;
  const int block_rows = p.block_tokens / p.tile_tokens * p.tile_rows;
  for (int e = blockIdx.y * kMergeThreads + threadIdx.x; e < rows * groups; e += gridDim.y * kMergeThreads) {
    const int c = e / rows, r = e - c * rows;
    const int at = r < used ? r : p.tile_rows + r - used;
    const float2* ml = reinterpret_cast<const float2*>(p.part_ml) + at;
    const float4* po = reinterpret_cast<const float4*>(p.part_o) + (size_t)c * block_rows + at;
    float M = -INFINITY, L = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = 0; s0 < pieces; s0 += kMergeBatch) {   // the loads of a batch are in flight together
      float2 x[kMergeBatch];
      float4 o[kMergeBatch];
#pragma unroll
      for (int i = 0; i < kMergeBatch; ++i) {
        const bool there = s0 + i < pieces;
        const size_t piece = s0 + i == 0 ? first : rest + (size_t)(s0 + i) * step;
        x[i] = there ? __ldcg(ml + piece * block_rows) : make_float2(-INFINITY, 0.f);
        if (there) o[i] = __ldcg(po + piece * groups * block_rows);
      }
      float m = M;
#pragma unroll
      for (int i = 0; i < kMergeBatch; ++i)
        if (!(x[i].y == 0.f)) m = fmaxf(m, x[i].x);   // (not l > 0: a NaN among the scores has to reach the output)
      const float old = M == -INFINITY ? 0.f : exp2f(M - m);
      M = m;
      L *= old, acc.x *= old, acc.y *= old, acc.z *= old, acc.w *= old;
#pragma unroll
      for (int i = 0; i < kMergeBatch; ++i) {
        if (x[i].y == 0.f) continue;
        const float w = exp2f(x[i].x - M);
        L += w * x[i].y;
        acc.x += w * o[i].x;
        acc.y += w * o[i].y;
        acc.z += w * o[i].z;
        acc.w += w * o[i].w;
      }
    }
    const float inv = 1.f / L;
    const int token = divide(r, p.by_sub), head = tile * p.sub + r - token * p.sub;
    T* dst = static_cast<T*>(p.out) + ((size_t)(row0 + token) * p.hq + head) * p.head_dim + c * 4;
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
    } else {
      *reinterpret_cast<float4*>(dst) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
    }
  }
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

}  // namespace pa

namespace pa {
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

int prompt_most_shares(const PromptAttnParams& p) {
  const int64_t tiles = (((int64_t)p.bounds.max_ctx + p.bounds.max_tokens + p.key_tile - 1) >> p.key_tile_log2) * p.batch * p.tile_heads;
  return (int)(tiles / 2 < p.cut_ctas ? tiles / 2 : p.cut_ctas);
}

size_t plan_prompt_attention(PromptAttnParams& p, bool bf16, size_t scratch, int sms) {
  p.cut_ctas = 0;
  if (bf16) {
    // A CTA an SM.  Pieces of one length (us by their key tiles, the rule's in brackets): one token after 4096 of 32/8
    // heads, 8 units of 33 tiles, 1: 17.5, [2: 12.7], 4: 12.8, 8: 15.7, uncut 42; after 32768, 10: 42.6, [14: 34.6], 17: 33.0,
    // 20: 34.3; 61 tokens of 64/8 heads after 32707, 20: 71.6, [29: 54], 40: 62; 256 tokens after 8192, 14: 52, [17: 41], 25: 51.
    pa::plan_tiles(p, 128, 2, 7, sms);
    // Several sequences of one block each (decoding): cut by the lengths on the device, where as many units as two rounds
    // of CTAs may gain by it.  One token of 32/8 heads (us, pieces of one length or uncut in brackets): 8 ragged contexts up
    // to 4096 22.3 [24.6], equal ones 30.9 [42.0], 12 ragged 28.6 [50.5], 16 ragged up to 8000 53.4 [93.2], 24 equal ones
    // of 8000 129.6 [183.5], 32 of 4000 92.2 [99.6]; what it loses: the merge's launch where the units stay whole, 18 of
    // 2000 31.6 [30.5], and the search, 2 of 4000 15.5 [14.6], 32 ragged up to 4000 56.5 [53.1].
    const int64_t units = (int64_t)p.batch * p.tile_heads;
    const int64_t key_tiles = ((int64_t)p.bounds.max_ctx + p.bounds.max_tokens + p.key_tile - 1) >> p.key_tile_log2;
    if (p.batch > 1 && p.bounds.max_tokens <= p.block_tokens && units <= 2 * (int64_t)sms && key_tiles > (units > sms ? 15 : 4) &&
        sms <= kMostCutCtas && units * key_tiles <= kMostCutTiles) {
      p.piece_tiles = (int)key_tiles;
      p.splits = 1;
      p.by_splits = index_divisor(1);
      p.cut_ctas = sms;
      const size_t rows = 2 * (size_t)prompt_most_shares(p) * 256;
      const size_t bytes = rows * (p.head_dim + 2) * sizeof(float);
      if (bytes <= scratch) {
        p.part_ml = p.part_o + rows * p.head_dim;
        return bytes;
      }
      p.cut_ctas = 0;
      return 0;
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
  const auto kernel = bf16 ? pa::prompt_merge_kernel<__nv_bfloat16> : pa::prompt_merge_kernel<float>;
  int64_t rows = (int64_t)(p.bounds.max_tokens < p.block_tokens ? p.bounds.max_tokens : p.block_tokens) * p.sub;
  const unsigned shares = (unsigned)((rows * (p.head_dim / 4) + pa::kMergeThreads - 1) / pa::kMergeThreads);
  const int blocks = p.cut_ctas > 0 ? p.batch : p.places;
  return launch_chained(kernel, dim3((unsigned)(blocks * p.tile_heads), shares), dim3(pa::kMergeThreads), 0, stream, 0, p);
}

}  // namespace ptd
