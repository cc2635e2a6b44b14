// Log probabilities of given tokens, entropies and best alternatives from hidden states: the LM-head product with the
// softmax statistics of row_sums.cuh as its epilogue.  The logits never reach memory.
//
// Tiles of 128 rows of H by 64 to 256 rows of W, one CTA per SM:
//   warp 0     TMA producer: per 64 columns of d_model the tile's rows of H and of W, 128-byte swizzle, into a ring;
//   warp 1     allocates TMEM, one thread issues the MMAs (M 128, K 16, bf16 -> fp32) into one of two accumulators;
//   warps 2-5  epilogue: TMEM lane r holds row r's logits; thread r keeps its row's sums, its best alternatives
//              (64-bit keys: value, then the lower token) and its token's logit over the CTA's tiles of a phase.
// A second kernel merges the parts that a row's CTAs left in the workspace.
//
// What bounds it: for many rows the tensor pipe and the power cap, 4096 rows of 4096 columns by 128256 tokens 2.23 ms in graph
// replays (1.93 PFLOP/s; 2.44 - 2.59 ms, 1.66 - 1.76 PFLOP/s, among other passes); for up to a tile of rows the one read of W, 63 rows
// 158 - 163 us (6.5 TB/s; 156 of 162.6 the product at 6.75), the merge and its launch the rest.  Where d_model is short the
// epilogue, some 3.6 us a tile of 224 tokens once the lists are full, which is the product of 800 columns: 4096 rows of 151936
// tokens 757 us with d = 1024 (1.68 PFLOP/s), 512 with d = 512 (1.24; 144 tiles a CTA).  A CTA with few tiles fills its
// lists where little hides it: 20 rows of 45725 tokens, d = 1792, k = 16 52.5 us (24 of bytes), 700 rows of 50000, d = 2048,
// k = 16 122 (84 of products).
// An MMA reads its 128 rows of H from shared memory whatever the tile's width, some 68 ns: tiles narrower than 224 tokens leave
// the pipe waiting.  Steps (us, 63 rows with k = 8, 4096 with k = 4): tiles of 128 / 256 tokens, every logit of a block inserted
// where one might belong 174, 2320 (4096 rows with k = 16 4940); the block's largest taken while it belongs, only the rows of H
// there are 168, 2300 (2374); tile by cost 166, 2240; four warps a row in the merge 162.6.
#include <cuda_runtime.h>

#include <cstdint>

#include "launch.cuh"
#include "lm_logprobs.cuh"
#include "ptd_device.cuh"
#include "row_sums.cuh"
#include "topk_parts.cuh"

namespace ptd {
namespace ll {

constexpr int kThreads = 192;
constexpr uint32_t kTmemCols = 512;

// Shared memory: the ring (the plan's stages), then barriers.
constexpr int kMostStages = 12;
constexpr uint32_t kRingBytes = 222 * 1024;
constexpr uint32_t kOffBar = kRingBytes;
constexpr int kNumBars = 2 * kMostStages + 5;   // full, empty, acc_full[2], acc_empty[2], drain
constexpr uint32_t kOffTmemPtr = kOffBar + kNumBars * 8, kOffAbort = kOffTmemPtr + 4;
constexpr uint32_t kSmemBytes = kOffAbort + 16 + 1024;   // slack to align the base to 1024 B
static_assert(kSmemBytes <= 232448, "shared memory budget");
constexpr int kAccColumns = 256;   // of TMEM, of each accumulator

// H of a stage: whole groups of eight rows, the swizzle's period.  The MMA reads 128 rows from there: behind the tile's last
// one what the W of the stage (or the next stages', or the ring's last 16 KB) holds, for rows that nobody reads.
__host__ __device__ constexpr uint32_t h_bytes(const LmLogprobsPlan& plan) { return (uint32_t)plan.box_rows * 128u; }
__host__ __device__ constexpr uint32_t stage_bytes(const LmLogprobsPlan& plan) {
  return h_bytes(plan) + (uint32_t)plan.tile_tokens * 128u;
}

// The parts of rows in the workspace: part (phase, cta) has 128 rows.
struct Parts {
  RowSums* sums;
  uint64_t* keys;       // [part rows][KM]
  float* token_logit;   // [rows]
};
__device__ __forceinline__ Parts parts_of(void* workspace, const LmLogprobsPlan& plan) {
  const size_t part_rows = (size_t)((plan.row_tiles + plan.per_phase - 1) / plan.per_phase) * plan.ctas * kLmTileRows;
  Parts p;
  p.keys = static_cast<uint64_t*>(workspace);
  p.sums = reinterpret_cast<RowSums*>(p.keys + part_rows * plan.keys);
  p.token_logit = reinterpret_cast<float*>(p.sums + part_rows);
  return p;
}

// Insert key into a descending list of KM keys (0 = empty: below every real key).
template <int KM>
__device__ __forceinline__ void insert(uint64_t (&top)[KM], uint64_t key) {
  if (key <= top[KM - 1]) return;
  top[KM - 1] = key;
#pragma unroll
  for (int j = KM - 1; j > 0; --j) {
    if (top[j] > top[j - 1]) {
      const uint64_t x = top[j];
      top[j] = top[j - 1];
      top[j - 1] = x;
    }
  }
}

// The best KM logits of a row that come in the order of their tokens: an equal logit that comes later stays behind.
// Tokens of -inf (and NaN) are never taken.
template <int KM>
struct Best {
  float x[KM > 0 ? KM : 1];   // descending, -inf: none
  int token[KM > 0 ? KM : 1];

  __device__ __forceinline__ Best() {
#pragma unroll
    for (int j = 0; j < KM; ++j) x[j] = -INFINITY, token[j] = 0;
  }
  __device__ __forceinline__ void insert(float v, int t) {
#pragma unroll
    for (int j = KM - 1; j >= 0; --j) {
      const bool above = j > 0 && v > x[j > 0 ? j - 1 : 0], here = v > x[j];
      token[j] = above ? token[j > 0 ? j - 1 : 0] : (here ? t : token[j]);
      x[j] = j > 0 ? fmaxf(fminf(v, x[j > 0 ? j - 1 : 0]), x[j]) : fmaxf(v, x[j]);
    }
  }
  // Takes what belongs here of 32 logits of tokens t0 ..., whose largest is `most` (v is used up): the largest that is left,
  // its first place, again while some lane has one.  A row of n logits takes about KM ln(n / KM) of them.
  __device__ __forceinline__ void take(float (&v)[32], float most, int t0) {
    for (int i = 0; i < 32 && __any_sync(0xffffffffu, most > x[KM - 1]); ++i) {   // (each takes one)
      int at = 0;
#pragma unroll
      for (int e = 31; e >= 0; --e) at = v[e] == most ? e : at;
      if (most > x[KM - 1]) insert(most, t0 + at);
#pragma unroll
      for (int e = 0; e < 32; ++e) v[e] = e == at ? -INFINITY : v[e];
      most = largest(v);
    }
  }
  static __device__ __forceinline__ float largest(const float (&v)[32]) {
    float m[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int e = 0; e < 32; e += 8)
#pragma unroll
      for (int q = 0; q < 4; ++q) m[q] = fmax3(m[q], v[e + 2 * q], v[e + 2 * q + 1]);
    return fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
  }
};

// The CTA's units, phase by phase: f(phase, row tile, first vocabulary tile, step).
template <typename F>
__device__ __forceinline__ void for_units(const LmLogprobsPlan& plan, F&& f) {
  for (int phase = 0, t0 = 0; t0 < plan.row_tiles; ++phase, t0 += plan.per_phase) {
    const int R = min(plan.per_phase, plan.row_tiles - t0), C = plan.ctas / R;
    const int lane = (int)blockIdx.x / R;
    if (lane < C && lane < plan.vocab_tiles)
      if (!f(phase, t0 + (int)blockIdx.x % R, lane, C)) return;
  }
}

template <int KM>
__global__ void __launch_bounds__(kThreads, 1)
    lm_logprobs_kernel(const __grid_constant__ CUtensorMap map_h, const __grid_constant__ CUtensorMap map_w,
                       const __grid_constant__ LmLogprobsParams p) {
  const int stages = p.plan.stages, tile_tokens = p.plan.tile_tokens;
  const uint32_t stage = stage_bytes(p.plan), h = h_bytes(p.plan);
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint32_t base = smem_u32(smem_raw);
  const uint32_t pad = (1024u - (base & 1023u)) & 1023u;
  uint8_t* smem = smem_raw + pad;
  base += pad;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto bar = [&](int i) { return base + kOffBar + 8u * (uint32_t)i; };
  auto full_bar = [&](int s) { return bar(s); };
  auto empty_bar = [&](int s) { return bar(kMostStages + s); };
  auto accf_bar = [&](int b) { return bar(2 * kMostStages + b); };
  auto acce_bar = [&](int b) { return bar(2 * kMostStages + 2 + b); };
  const uint32_t drain_bar = bar(2 * kMostStages + 4);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + kOffAbort);

  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(accf_bar(b), 1);
      mbar_init(acce_bar(b), 4);   // one arrival per epilogue warp
    }
    mbar_init(drain_bar, 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(base + kOffTmemPtr, kTmemCols);
    tmem_relinquish();
    tc_fence_before();
  }
  grid_dependency_wait();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(smem + kOffTmemPtr);
  const int n_chunks = p.d_model / 64, vocab_tiles = p.plan.vocab_tiles;

  if (warp == 0) {
    // ================================================================ TMA producer
    if (lane == 0) {
      prefetch_tensormap(&map_h);
      prefetch_tensormap(&map_w);
      bool ok = true;
      int s = 0, g = 0;   // ring position; chunks issued
      uint32_t phase_bit = 1;
      for_units(p.plan, [&](int, int row_tile, int tile, int step) {
        for (; tile < vocab_tiles; tile += step) {
          for (int c = 0; c < n_chunks; ++c) {
            if (!(ok = mbar_wait(empty_bar(s), phase_bit, abort_flag, p.dev_status))) return false;
            const uint32_t dst = base + (uint32_t)s * stage;
            mbar_arrive_expect_tx(full_bar(s), stage);
            tma_load_2d(dst, &map_h, full_bar(s), c * 64, row_tile * kLmTileRows);
            tma_load_2d(dst + h, &map_w, full_bar(s), c * 64, tile * tile_tokens);
            ++g;
            if (++s == stages) s = 0, phase_bit ^= 1u;
          }
        }
        return true;
      });
      if (!ok) {   // let the copies already issued land before the CTA can exit
        for (int back = 1; back <= stages && g - back >= 0; ++back)
          mbar_drain(full_bar((g - back) % stages), (uint32_t)(((g - back) / stages) & 1), 100000000ull);
      }
    }
  } else if (warp == 1) {
    // ================================================================ MMA issuer
    if (lane == 0) {
      const uint32_t idesc = idesc_bf16_f32(kLmTileRows, tile_tokens, 0, 0);
      bool ok = true;
      int s = 0, it = 0;
      uint32_t phase_bit = 0;
      for_units(p.plan, [&](int, int, int tile, int step) {
        for (; tile < vocab_tiles; tile += step, ++it) {
          const int buf = it & 1;
          if (!(ok = mbar_wait(acce_bar(buf), (uint32_t)(((it >> 1) & 1) ^ 1), abort_flag, p.dev_status))) return false;
          tc_fence_after();
          const uint32_t d = tmem + (uint32_t)(buf * kAccColumns);
          for (int c = 0; c < n_chunks; ++c) {
            if (!(ok = mbar_wait(full_bar(s), phase_bit, abort_flag, p.dev_status))) return false;
            tc_fence_after();
            const uint32_t a0 = base + (uint32_t)s * stage, b0 = a0 + h;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
              mma_bf16_ss(d, smem_desc_sw128(a0 + (uint32_t)kk * 32u, 16, 1024), smem_desc_sw128(b0 + (uint32_t)kk * 32u, 16, 1024),
                          idesc, (c > 0 || kk > 0) ? 1u : 0u);
            mma_commit(empty_bar(s));   // the stage is free once these MMAs have read it
            if (++s == stages) s = 0, phase_bit ^= 1u;
          }
          mma_commit(accf_bar(buf));
        }
        return true;
      });
      if (!ok) {   // let the tensor core finish what was issued before TMEM is freed
        mma_commit(drain_bar);
        mbar_drain(drain_bar, 0, 100000000ull);
      }
    }
  } else {
    // ================================================================ epilogue
    const int wq = warp & 3;                     // TMEM lane quarter of this warp
    const uint32_t lane_base = (uint32_t)(wq * 32) << 16;
    const unsigned long long scale2 = f2_pack(p.scale, p.scale);
    const Parts parts = parts_of(p.workspace, p.plan);
    int it = 0;
    for_units(p.plan, [&](int phase, int row_tile, int tile, int step) {
      const int r = wq * 32 + lane, row = row_tile * kLmTileRows + r;
      const int token = row < p.rows ? p.tokens[row] : -1;
      ThreadSums sums;
      Best<KM> best;
      const bool any_row = row - lane < p.rows;   // of the warp's rows
      for (; tile < vocab_tiles; tile += step, ++it) {
        const int buf = it & 1;
        if (!mbar_wait_warp(accf_bar(buf), (uint32_t)((it >> 1) & 1), abort_flag, p.dev_status)) return false;
        tc_fence_after();
        const int t0 = tile * tile_tokens;
#pragma unroll 1
        for (int c0 = 0; c0 < tile_tokens && any_row; c0 += 32) {
          uint32_t v[32];
          tmem_ld32(tmem + lane_base + (uint32_t)(buf * kAccColumns + c0), v);
          tmem_ld_wait();
          const int tb = t0 + c0;
          float x[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) x[e] = __uint_as_float(v[e]);
          if (tb + 32 > p.vocab) {   // rows of W past the last one were read as zeros
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (tb + e >= p.vocab) x[e] = -INFINITY;
          }
          const float most = Best<KM>::largest(x);
          sums.raise(most, p.scale);
          sums.add(x, scale2);
          if ((unsigned)(token - tb) < 32u) {
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (token == tb + e && token < p.vocab) parts.token_logit[row] = x[e];
          }
          if constexpr (KM > 0) best.take(x, most, tb);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(acce_bar(buf));
      }
      if (row < p.rows) {
        const size_t at = ((size_t)phase * p.plan.ctas + blockIdx.x) * kLmTileRows + r;
        parts.sums[at] = sums.sums();
#pragma unroll
        for (int j = 0; j < KM; ++j)
          parts.keys[at * KM + j] =
              best.x[j] == -INFINITY ? 0ull : topk::make_key(topk::ordered_bits(best.x[j]), (uint32_t)best.token[j]);
      }
      return true;
    });
  }
  __syncthreads();
  if (threadIdx.x == 0) grid_launch_dependents();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

// Latency: the parts' reads, insertions and rounds of maxima; four warps a row where the parts are many (63 rows, 152 parts:
// the whole call 162.6 us, 166 with one warp a row).
// kWarps warps per row: each lane merges some of the row's parts, a warp its lanes' by KM rounds of a warp-wide maximum (the owning
// lane pops its head), the first warp the warps'.
constexpr int kMergeThreads = 128;

template <int KM>
__device__ __forceinline__ void warp_top(uint64_t (&top)[KM > 0 ? KM : 1], uint64_t (&out)[KM > 0 ? KM : 1]) {
#pragma unroll
  for (int j = 0; j < KM; ++j) {
    const uint64_t best = topk::warp_max_u64(top[0]);
    out[j] = best;
    if (best != 0ull && top[0] == best) {   // keys are distinct
#pragma unroll
      for (int q = 0; q < KM - 1; ++q) top[q] = top[q + 1];
      top[KM - 1] = 0ull;
    }
  }
}

template <int KM, int kWarps>
__global__ void __launch_bounds__(kMergeThreads) lm_logprobs_merge_kernel(const __grid_constant__ LmLogprobsParams p) {
  constexpr int kList = KM > 0 ? KM : 1, kRowWarps = kMergeThreads / 32 / kWarps;   // rows of a CTA
  __shared__ RowSums sums_s[kWarps];
  __shared__ uint64_t keys_s[kWarps * kList];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int row = kWarps > 1 ? (int)blockIdx.x : (int)blockIdx.x * kRowWarps + warp;
  if (threadIdx.x == 0) grid_launch_dependents();
  grid_dependency_wait();
  if (row >= p.rows) return;   // (a whole CTA where its warps share a row)
  const Parts parts = parts_of(p.workspace, p.plan);
  const int row_tile = row / kLmTileRows, phase = row_tile / p.plan.per_phase, t0 = phase * p.plan.per_phase;
  const int R = min(p.plan.per_phase, p.plan.row_tiles - t0), C = min(p.plan.ctas / R, p.plan.vocab_tiles);
  const int token = p.tokens[row];
  const bool inside = token >= 0 && token < p.vocab;
  const float token_logit = inside ? parts.token_logit[row] : 0.f;
  RowSums sums = {-INFINITY, 0.f, 0.f};
  uint64_t top[kList];
#pragma unroll
  for (int j = 0; j < KM; ++j) top[j] = 0ull;
  for (int c = (kWarps > 1 ? warp * 32 : 0) + lane; c < C; c += 32 * kWarps) {
    const size_t at = ((size_t)phase * p.plan.ctas + c * R + (row_tile - t0)) * kLmTileRows + row % kLmTileRows;
    uint64_t list[kList];   // read together: an insertion may end early, and the next load would wait for it
#pragma unroll
    for (int j = 0; j < KM; ++j) list[j] = parts.keys[at * KM + j];
    sums = merge_sums(sums, parts.sums[at], p.scale);
#pragma unroll
    for (int j = 0; j < KM; ++j) insert(top, list[j]);
  }
  sums = merge_lanes<32>(sums, p.scale);
  uint64_t best[kList];
  warp_top<KM>(top, best);
  if constexpr (kWarps > 1) {
    if (lane == 0) {
      sums_s[warp] = sums;
#pragma unroll
      for (int j = 0; j < KM; ++j) keys_s[warp * kList + j] = best[j];
    }
    __syncthreads();
    if (warp != 0) return;
    sums = merge_lanes<kWarps>(sums_s[lane & (kWarps - 1)], p.scale);
#pragma unroll
    for (int j = 0; j < KM; ++j) top[j] = lane < kWarps ? keys_s[lane * kList + j] : 0ull;
    warp_top<KM>(top, best);
  }
  const RowResult result(sums);
  if (lane == 0) {
    p.logprob[row] = inside ? result.logprob(token_logit, p.inv_temperature) : -INFINITY;
    if (p.entropy != nullptr) p.entropy[row] = result.entropy;
  }
#pragma unroll
  for (int j = 0; j < KM; ++j)
    if (lane == j && j < p.k) {
      p.top_idx[(size_t)row * p.k + j] = best[j] != 0ull ? (int32_t)(~(uint32_t)best[j]) : -1;
      p.top_val[(size_t)row * p.k + j] =
          result.logprob(best[j] != 0ull ? topk::from_ordered((uint32_t)(best[j] >> 32)) : -INFINITY, p.inv_temperature);
    }
}

template <int KM>
cudaError_t launch(const CUtensorMap& map_h, const CUtensorMap& map_w, const LmLogprobsParams& p, cudaStream_t stream) {
  cudaError_t e = cudaFuncSetAttribute(lm_logprobs_kernel<KM>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBytes);
  if (e != cudaSuccess) return e;
  e = launch_chained(lm_logprobs_kernel<KM>, dim3(p.plan.ctas), dim3(kThreads), kSmemBytes, stream, 0, map_h, map_w, p);
  if (e != cudaSuccess) return e;
  // a CTA per row where a row has many parts, which is where the rows are few
  constexpr int kWarps = kMergeThreads / 32;
  if (p.plan.row_tiles < 4)
    return launch_chained(lm_logprobs_merge_kernel<KM, kWarps>, dim3(p.rows), dim3(kMergeThreads), 0, stream, 0, p);
  return launch_chained(lm_logprobs_merge_kernel<KM, 1>, dim3((p.rows + kWarps - 1) / kWarps), dim3(kMergeThreads), 0, stream, 0, p);
}

}  // namespace ll

// Tokens of a tile, by what the phases would take.  Per 64 columns of d_model (ns, all SMs busy): the four MMAs 270 up to 192
// tokens (the rows of H are read from shared memory anew for each), 291 with 224 and 340 with 256; W 128 bytes a token from
// HBM, at 44.6 a ns and SM, once for the phase's row tiles; the lesser of the two hides but for some 15 %.  After a phase's last
// tile its epilogue, some 35 ns a token (those of the tiles before are taken as hidden, which they are from d = 800 on).  GB300, d = 4096, 128256 tokens, us with 128 / 192 / 224 / 256 tokens: 63 rows 169 / 169 /
// 166 / 171, 200 rows 254 / 189 / 184 / 196, 500 rows 477 / 330 / 305 / 322, 4096 rows 3678 / 2548 / 2251 / 2300; 5707 rows of
// 10605 tokens, d = 2752 348 / 223 / 227 / 242; 2000 rows of 1000, d = 512 25.1 / 30.0 / 32.2 / 34.2 (with 64 19.7).
constexpr int kLeastTile = 64;
static int choose_tile_tokens(int row_tiles, int per_phase, int vocab, int d_model, int sms) {
  int best = 0;
  double least = 0.;
  for (int tile = kLeastTile; tile <= 256; tile += 32) {
    const int64_t vocab_tiles = ((int64_t)vocab + tile - 1) / tile;
    const double mma = tile <= 192 ? 270. : (tile == 224 ? 291. : 340.);
    double total = 0.;
    const auto add = [&](int64_t phases, int R) {
      const int64_t C = sms / R, rounds = (vocab_tiles + C - 1) / C;
      const double load = tile * 128. / (44.6 * R), chunk = (mma > load ? mma : load) + 0.15 * (mma > load ? load : mma);
      total += (double)phases * ((double)rounds * (d_model / 64) * chunk + 35. * tile);
    };
    add(row_tiles / per_phase, per_phase);
    if (row_tiles % per_phase != 0) add(1, row_tiles % per_phase);
    if (best == 0 || total < least) best = tile, least = total;
  }
  return best;
}

static LmLogprobsPlan make_plan(int rows, int vocab, int tile_tokens, int k, int sms) {
  LmLogprobsPlan plan;
  plan.row_tiles = (rows + kLmTileRows - 1) / kLmTileRows;
  plan.per_phase = sms < 8 ? sms : 8;
  plan.box_rows = rows < kLmTileRows ? (rows + 7) / 8 * 8 : kLmTileRows;
  plan.tile_tokens = tile_tokens;
  plan.vocab_tiles = (vocab + tile_tokens - 1) / tile_tokens;
  // the MMA reads 128 rows from the last stage's H too
  const uint32_t stages = (ll::kRingBytes - (kLmTileRows - plan.box_rows) * 128u) / ll::stage_bytes(plan);
  plan.stages = stages < (uint32_t)ll::kMostStages ? (int)stages : ll::kMostStages;
  plan.keys = k == 0 ? 0 : (k <= 4 ? 4 : (k <= 8 ? 8 : 16));
  const int64_t most = (int64_t)(plan.row_tiles < plan.per_phase ? plan.row_tiles : plan.per_phase) * plan.vocab_tiles;
  plan.ctas = most < sms ? (int)most : sms;
  return plan;
}

LmLogprobsPlan plan_lm_logprobs(int rows, int vocab, int d_model, int k, int sms) {
  const int row_tiles = (rows + kLmTileRows - 1) / kLmTileRows;
  return make_plan(rows, vocab, choose_tile_tokens(row_tiles, sms < 8 ? sms : 8, vocab, d_model, sms), k, sms);
}

size_t lm_logprobs_workspace_bytes(int rows, int vocab, int k, int sms) {
  // (of the plan with the most CTAs: the tile goes by d_model too)
  const LmLogprobsPlan plan = make_plan(rows, vocab, kLeastTile, k, sms);
  const size_t part_rows = (size_t)((plan.row_tiles + plan.per_phase - 1) / plan.per_phase) * plan.ctas * kLmTileRows;
  return part_rows * (plan.keys * sizeof(uint64_t) + sizeof(RowSums)) + (size_t)rows * sizeof(float);
}

cudaError_t launch_lm_logprobs(const CUtensorMap& map_h, const CUtensorMap& map_w, const LmLogprobsParams& p, cudaStream_t stream) {
  switch (p.plan.keys) {
    case 0: return ll::launch<0>(map_h, map_w, p, stream);
    case 4: return ll::launch<4>(map_h, map_w, p, stream);
    case 8: return ll::launch<8>(map_h, map_w, p, stream);
    default: return ll::launch<16>(map_h, map_w, p, stream);
  }
}

}  // namespace ptd
