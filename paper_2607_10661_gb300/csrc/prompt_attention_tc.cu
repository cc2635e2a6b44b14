// Causal attention of packed new tokens over the cache on the 5th-generation tensor cores (tcgen05 + TMEM +
// TMA), bf16, D = 128.
//
// Work.  `sub` query heads of one KV head and `tile_tokens` tokens form the rows r = token * sub + head of an
// M tile (128 rows), two M tiles a block, so that 2 * 128 rows share every K and V tile of 128 keys; a block
// meets only the tiles that its last token sees, each M tile only those that its own does.  A work unit is a
// (block, head tile), or a piece of its keys (partials, merged by prompt_merge_kernel).  Units are numbered
// longest first over the whole batch (prompt_geometry.cuh); the grid has one CTA per unit, and a resident CTA
// takes the numbers of CTAs that have not started yet (cluster launch control), so that the SMs' shares
// even out whatever the lengths, and a unit's first loads and its set-up run beside the unit before it.  Few units
// go by equal shares of their key tiles instead where that is shorter (PromptCut).
//
// Warps (384 threads; the first four give registers to the others):
//   0       scheduler and TMA producer: claims the next unit before the last tiles of this one are asked for;
//           K and V tiles into a ring of five, Q.
//   1, 2    MMA issuers of M tile 0 and 1: S_t = Q_t K^T, then PV_t, S_t' | PV_t', S_t'' | .., in turns, so that
//           one M tile's softmax runs beside the other's products (without turns 2047 tokens of 32 MHA heads
//           take 36.0 us instead of 31.3).
//   3       V check: of key tiles that some row sees in part, infinities and NaN of V are set to 0 (a
//           weight of 0 must not meet them) and noted; the rows that see such a key add it at the end.
//   4 - 11  softmax of M tile 0 (4 - 7) and 1 (8 - 11), a thread a row: running maximum, moved only when
//           exceeded by 2^8, exp2, bf16 weights over S in TMEM (told in two halves), fp32 row sum; O / l at the end.
// TMEM: S_0 | S_1 | O_0 | O_1, 128 fp32 columns each; P_t lies over the first 64 columns of S_t.
//
// Bound by the tensor pipe and the power cap for long prompts: 8192 tokens of 32/8 heads 337 us among other passes (1.63
// PFLOP/s of the seen pairs, 0.95 of cuBLAS' sustained rate), 300 after a pause (1.83); 16384 of 64/8 heads 2.60 ms (1.69
// PFLOP/s) and 2.29.  Ragged prompts of some hundred tokens (31 us for 18.5 GFLOP) are bound by changes of unit, ~4.5 us
// each: the V check, masked tiles, outputs, and code that has left the instruction caches (so it is kept short).
// Decoding: by HBM, ~6 us from the start to the first output, and the merge: 8 contexts of up to 4096 22.4 us for 73 MB,
// 24 of 8000 128 us for 787 MB (6.1 TB/s).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <climits>
#include <cmath>
#include <cstdint>

#include "attention_tc.cuh"
#include "launch.cuh"
#include "prompt_attention.cuh"
#include "ptd_device.cuh"

namespace ptd {
namespace pt {

using pa::Unit;
using tc::kHalfBytes;
using tc::kTileBytes;

constexpr int kThreads = 384;
constexpr int kTiles = 5;    // of the ring of K and V tiles
constexpr int kSteps = 8;    // barriers for steps whose tiles have been read: more than steps that tiles are held for
// Registers a thread: 168 at launch (384 threads), then 104 for warps 0 - 3 and 200 for the softmax warps,
// which hold a row's 128 scores: 128 * 104 + 256 * 200 = 384 * 168.
constexpr int kRegsLaunch = 168, kRegsFew = 104, kRegsMany = 200;
static_assert(128 * kRegsFew + 256 * kRegsMany <= kThreads * kRegsLaunch, "register split");
constexpr uint32_t kOffQ = 0;
constexpr uint32_t kOffRing = 2 * kTileBytes;
constexpr uint32_t kOffBar = kOffRing + kTiles * kTileBytes;
// The ring takes a unit's tiles as K_0 | V_0, K_1 | V_1, K_2 | .. | V_n-1; a step is what lies between two bars:
// its tiles are free when its products are done, which one commit tells.
enum Bar {
  kFull = 0,
  kLoadV = kFull + kTiles,    // a V tile that is checked before it counts as full
  kDone = kLoadV + kTiles,    // steps, in turn, by both issuers
  kSFull = kDone + kSteps,
  kPHalf = kSFull + 2,        // P of a tile's first 64 keys, by its four warps, and the issuer's turn, by the other issuer
  kPFull = kPHalf + 2,        // of the others, by the four warps
  kOFull = kPFull + 2,
  kQFull = kOFull + 2,
  kQEmpty = kQFull + 2,
  kSegFull = kQEmpty + 2,
  kSegEmpty = kSegFull + 2,
  kClaim = kSegEmpty + 2,
  kEntry,                     // issuer 1 has begun a unit with turns
  kDrain,
  kBars = kDrain + 2
};
constexpr uint32_t kOffTmemPtr = kOffBar + kBars * 8;
constexpr uint32_t kOffAbort = kOffTmemPtr + 4;
constexpr uint32_t kOffClaim = (kOffAbort + 4 + 15) / 16 * 16;   // the scheduler's answer, 16 bytes

// A bounded wait of a warp for the barrier's phase: false when it, or another role, has given up.  A try_wait that
// finds the phase open sleeps until it ends, for 1.95 us at most (measured), so that 2^20 tries are 2 s.  (The roles'
// code is larger than the near instruction caches: a short loop in place of mbar_wait_warp's clock.)  A wait that lasts
// while other roles work on a whole unit (kUnitTries: 128 s) is as long as the unit's keys make it, ~1 us a key tile, and ends
// at once where one of them has given up.
constexpr int kTries = 1 << 20, kUnitTries = 1 << 26;
template <int kMost = kTries>
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* dev_status) {
#pragma unroll 1
  for (int tries = 0; tries < kMost; ++tries) {
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    if (__any_sync(0xffffffffu, *abort_flag != 0)) return false;
  }
  *abort_flag = 1;
  atomicMax(dev_status, (int)PTD_ERR_TIMEOUT);
  return false;
}

// One lane of the warp, always the same; the compiler knows such a branch to be one thread's, and its copies then
// cost 17 cycles to issue instead of 60.
__device__ __forceinline__ bool elect_lane() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0;
}

// A unit as the roles need it.
struct Seg {
  int valid;
  int b, row0, ctx, token0, tokens, head0, kv;
  int piece;             // place of its partials, -1: it is a whole block
  int kt0;               // first key tile
  int n[2];              // key tiles of either M tile (0: not there, or no keys in this piece)
  int edge;              // first key tile that some row sees in part
  int bad;               // the V check found infinities or NaN
};
constexpr uint32_t kOffSeg = kOffClaim + 16;
constexpr uint32_t kSmemUsed = kOffSeg + 2 * sizeof(Seg);
constexpr uint32_t kSmemBytes = kSmemUsed + 1024;   // slack to align the base to 1024 B
static_assert(kSmemBytes <= 232448, "shared memory budget");

// Ask for the number of a CTA of this grid that has not started (16 bytes to `dst`, counted on `bar`).
__device__ __forceinline__ void claim_cta(uint32_t dst, uint32_t bar) {
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(dst),
               "r"(bar)
               : "memory");
}
// Its blockIdx.x, or -1 if there was none.
__device__ __forceinline__ int claimed_cta(uint32_t src) {
  int x;
  asm volatile(
      "{\n\t.reg .b128 answer;\n\t.reg .pred got;\n\t.reg .b32 y, z, w;\n\tld.shared.b128 answer, [%1];\n\t"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 got, answer;\n\tmov.b32 %0, -1;\n\t"
      "@got clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%0, y, z, w}, answer;\n\t}"
      : "=r"(x)
      : "r"(src)
      : "memory");
  return x;
}

// O (TMEM at tO) times alpha, kept out of the hot loop.  Warp-collective.
static __device__ __noinline__ void rescale_o(uint32_t tO, float alpha) {
#pragma unroll 1
  for (int q = 0; q < 8; ++q) {
    uint32_t o[16];
    tmem_ld16(tO + (uint32_t)q * 16u, o);
    tmem_ld_wait();
#pragma unroll
    for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
    tmem_st16(tO + (uint32_t)q * 16u, o);
  }
  tmem_st_wait();
}

// Softmax of one key tile of this thread's row: S (TMEM at tS) becomes the bf16 P over its first 64 columns,
// against the reference maximum m_run (log2 units), which only moves up, and only when exceeded by more than
// 2^8; then the row sum and O (TMEM at tO, if `has_o`) are rescaled.  The weights are rounded to bf16, as the tensor cores
// take them beside V (the row sum adds them before that): the error against 64 bits is 1.2 to 1.4 times that of 32-bit
// weights, whose outputs are rounded to bf16 too (2.0e-3 of the outputs' size for 1.5e-3, decoding 2.3e-3 for 1.6e-3).
// With need_mask (warp-uniform) the row sees the tile's keys 0 .. last.  The whole row is in registers: one maximum and
// one vote a tile, and then exponentials and packing without a dependence between chunks.  Warp-collective.
__device__ __forceinline__ void softmax_tile(uint32_t tS, uint32_t tO, bool has_o, bool need_mask, int last, float sl2,
                                             float& m_run, float& l_run, uint32_t half_bar) {
  uint32_t r[4][32];
#pragma unroll
  for (int c = 0; c < 4; ++c) tmem_ld32(tS + (uint32_t)c * 32u, r[c]);
  tmem_ld_wait();
  if (need_mask) {
    const int all = (int)__reduce_min_sync(0xffffffffu, (unsigned)max(last, 0));   // what every row of the warp sees
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      if (all < c * 32 + 31) {
#pragma unroll
        for (int e = 0; e < 32; ++e) r[c][e] = c * 32 + e <= last ? r[c][e] : __float_as_uint(-INFINITY);
      }
    }
  }
  float a[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    a[c] = -INFINITY;
#pragma unroll
    for (int e = 0; e < 32; e += 2) a[c] = fmax3(a[c], __uint_as_float(r[c][e]), __uint_as_float(r[c][e + 1]));
  }
  const float cm = fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3])) * sl2;
  const bool raise = cm > m_run + tc::kRescaleLog2;
  if (__any_sync(0xffffffffu, raise)) {   // (a rescale's TMEM accesses are warp-collective)
    float alpha = 1.f;
    if (raise) {
      alpha = m_run == -INFINITY ? 0.f : ptx_exp2(m_run - cm);
      m_run = cm;
    }
    l_run *= alpha;
    if (has_o) rescale_o(tO, alpha);
  }
  const float m_use = m_run == -INFINITY ? 0.f : m_run;   // -inf only while nothing is visible
  const unsigned long long negm = f2_pack(-m_use, -m_use), sl2x2 = f2_pack(sl2, sl2);
  unsigned long long sum[2] = {f2_pack(0.f, 0.f), f2_pack(0.f, 0.f)};
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    uint32_t pk[16];
#pragma unroll
    for (int e = 0; e < 32; e += 2) {
      float x0, x1;
      f2_unpack(f2_fma(f2_pack(__uint_as_float(r[c][e]), __uint_as_float(r[c][e + 1])), sl2x2, negm), x0, x1);
      const float p0 = ptx_exp2(x0), p1 = ptx_exp2(x1);
      sum[(e >> 1) & 1] = f2_add(sum[(e >> 1) & 1], f2_pack(p0, p1));
      pk[e >> 1] = pack_bf16x2(p0, p1);
    }
    tmem_st16(tS + (uint32_t)c * 16u, pk);   // P chunk c: columns [16c, 16c+16) of S
    if (c == 1) {   // the products of the first 64 keys may start
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if ((threadIdx.x & 31) == 0) mbar_arrive(half_bar);
    }
  }
  float s0, s1;
  f2_unpack(f2_add(sum[0], sum[1]), s0, s1);
  l_run += s0 + s1;
  tmem_st_wait();
  tc_fence_before();
}

// The eight instructions of S_t = Q_t K^T, and [kBegin, kEnd) of those of O_t (+)= P_t V (see tc::issue_s, issue_pv), from
// one elected lane: against a lane chosen by a predicate on each instruction 16384 tokens of 64/8 heads take 2472 us
// instead of 2653, 8192 of 32/8 heads 300 instead of 330 (graph replays).
__device__ __forceinline__ void issue_s(uint32_t s_tmem, uint32_t q_desc, uint32_t k_desc) {
  if (elect_lane()) {
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      const uint32_t o = (uint32_t)(kk >> 2) * (kHalfBytes >> 4) + (uint32_t)(kk & 3) * 2u;
      mma_ss_if(1u, s_tmem, q_desc + o, k_desc + o, tc::kDescHi, tc::kIdescS, kk > 0 ? 1u : 0u);
    }
  }
  __syncwarp();
}
template <int kBegin, int kEnd>
__device__ __forceinline__ void issue_pv(uint32_t s_tmem, uint32_t v_desc, bool acc) {
  if (elect_lane()) {
#pragma unroll
    for (int kk = kBegin; kk < kEnd; ++kk)
      mma_ts_if(1u, s_tmem + 256u, s_tmem + (uint32_t)kk * 8u, v_desc + (uint32_t)kk * 128u, tc::kDescHi, tc::kIdescPV,
                (acc || kk > 0) ? 1u : 0u);
  }
  __syncwarp();
}

// 32 bytes of a row.  A warp's rows lie apart, so a store costs a pass a row whatever its width: 32 bytes at a
// time where the output allows (16 at a time: ragged prompts 33.7 us instead of 30.5, 4096 tokens 87.8 instead of 84.4).
__device__ __forceinline__ void store_row(uint4* dst, const uint32_t (&w)[8], bool wide) {
  if (wide) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst), "r"(w[0]), "r"(w[1]), "r"(w[2]),
                 "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
  } else {
    dst[0] = make_uint4(w[0], w[1], w[2], w[3]);
    dst[1] = make_uint4(w[4], w[5], w[6], w[7]);
  }
}

// Bit 15 of either half: the bf16 there is an infinity or NaN.
__device__ __forceinline__ uint32_t exponent_full(uint32_t w) { return (w & 0x7F807F80u) + 0x00800080u; }
__device__ __forceinline__ uint32_t finite_or_zero(uint32_t w) {
  if ((w & 0x7F80u) == 0x7F80u) w &= 0xFFFF0000u;
  if ((w & 0x7F800000u) == 0x7F800000u) w &= 0xFFFFu;
  return w;
}

// 16 outputs of a row (columns c ..) plus the infinities and NaN of V at keys [key0, key1], which the V check
// took out of the products.
template <bool kPaged>
__device__ __forceinline__ void add_bad(const PromptAttnParams& p, float* o, int b, int kv, int c, int key0, int key1) {
  for (int key = key0; key <= key1; ++key) {
    size_t r;
    if (kPaged) {
      const int pg = p.block_table[(size_t)b * p.max_pages + (key >> p.page_log2)];
      if (pg < 0 || pg >= p.num_pages) continue;
      r = ((size_t)p.layer * p.num_pages + pg) * p.page_size + (key & (p.page_size - 1));
    } else {
      r = ((size_t)p.layer * p.batch + b) * p.seq_capacity + key;
    }
    const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(p.v) + (r * p.hkv + kv) * 128 + c;
#pragma unroll 1
    for (int e = 0; e < 16; ++e) {
      const float x = __bfloat162float(v[e]);
      if (!isfinite(x)) o[e] += x;
    }
  }
}

// kPages: 0 for a contiguous cache, else the most pages that a key tile has (2: pages of 64 and 128, 8: of 16 and 32;
// 4096 tokens of 32/8 heads in pages of 128 take 84.4 us with 2 and 90.2 with 8).
template <int kPages>
__global__ void __launch_bounds__(kThreads, 1)
    prompt_tc_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                     const __grid_constant__ CUtensorMap map_q, const PromptAttnParams p) {
  constexpr bool kPaged = kPages > 0;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  uint32_t base = smem_u32(smem_raw);
  const uint32_t pad = (1024u - (base & 1023u)) & 1023u;
  uint8_t* smem = smem_raw + pad;
  base += pad;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  auto bar = [&](int i) { return base + kOffBar + 8u * (uint32_t)i; };
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + kOffAbort);
  Seg* segs = reinterpret_cast<Seg*>(smem + kOffSeg);
  const int used = p.tile_tokens * p.sub;   // rows of an M tile

  // set-up that reads no global memory: it may overlap the stream's previous grid
  if (threadIdx.x == 0) {
    for (int i = 0; i < kBars; ++i) {
      const int count = i >= kDone && i < kDone + kSteps ? 2 : i >= kPHalf && i < kPHalf + 2 ? 5
                        : i >= kPFull && i < kPFull + 2 ? 4 : i >= kSegEmpty && i < kSegEmpty + 2 ? 11 : 1;
      mbar_init(bar(i), count);
    }
    *abort_flag = 0;
    fence_mbar_init();
    prefetch_tensormap(&map_k);
    prefetch_tensormap(&map_v);
    prefetch_tensormap(&map_q);
  }
  if (warp == 1) {
    tmem_alloc(base + kOffTmemPtr, tc::kTmemCols);
    tmem_relinquish();
    tc_fence_before();
  }
  if (used < 128) {   // rows that no load writes: finite, so that they cost no rescaling
    for (int i = threadIdx.x; i < 2 * 2 * (128 - used) * 8; i += kThreads) {
      const int c = i & 7, r = (i >> 3) % (128 - used), h = (i >> 3) / (128 - used);
      st_shared_v4(base + kOffQ + (uint32_t)h * kHalfBytes + (uint32_t)(used + r) * 128u + (uint32_t)c * 16u, 0, 0, 0, 0);
    }
    fence_proxy_async_smem();
  }
  grid_dependency_wait();   // every input and output belongs to the stream's previous work
  __syncthreads();
  tc_fence_after();
  if (threadIdx.x == 0) grid_launch_dependents();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(smem + kOffTmemPtr);

  // The unit of a role's turn `it` (two slots), as long as there is one.
  auto wait_seg = [&](int it) -> const volatile Seg* {
    if (!wait_warp<kUnitTries>(bar(kSegFull + (it & 1)), (uint32_t)(it >> 1) & 1u, abort_flag, p.dev_status)) return nullptr;
    const volatile Seg* s = segs + (it & 1);
    return s->valid ? s : nullptr;
  };
  auto free_seg = [&](int it) {
    __syncwarp();
    if (lane == 0) mbar_arrive(bar(kSegEmpty + (it & 1)));
  };

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsFew));
    if (warp == 1 || warp == 2) {
      // ================================================================ MMA issuer of M tile t
      const int t = warp - 1;
      const uint32_t dq = (uint32_t)smem_desc_sw128(base + kOffQ + (uint32_t)t * kTileBytes, 16, 1024);
      const uint32_t dk = (uint32_t)smem_desc_sw128(base + kOffRing, 16, 1024);
      const uint32_t dv = (uint32_t)smem_desc_sw128(base + kOffRing, kHalfBytes, 1024);
      const uint32_t s_tmem = tmem + (uint32_t)t * 128u;
      auto commit = [&](int b) {
        if (elect_lane()) mma_commit(bar(b));
        __syncwarp();
      };
      auto arrive = [&](int b) {
        if (elect_lane()) mbar_arrive(bar(b));
        __syncwarp();
      };
      auto wait = [&](int b, int uses) { return wait_warp(bar(b), (uint32_t)uses & 1u, abort_flag, p.dev_status); };
      bool ok = true;
      int steps = 0, ps = 0, qs = 0;   // steps, P and Q taken
      int entries = 0;                 // units with turns that issuer 1 was waited for in
      int at = 0;                      // ring place of the next tile
      uint32_t phase = 0;              // the ring's turn
      auto take = [&](uint32_t& tile) {   // waits for the next tile; its descriptor offset
        if (!wait(kFull + at, (int)phase)) return false;
        tile = (uint32_t)at * (kTileBytes >> 4);
        if (++at == kTiles) at = 0, phase ^= 1u;
        return true;
      };
      auto step_done = [&](bool issued) {   // the step's tiles are free when its products are done
        if (issued) commit(kDone + steps % kSteps); else arrive(kDone + steps % kSteps);
        ++steps;
      };
      for (int it = 0; ok; ++it) {
        const volatile Seg* sg = wait_seg(it);
        if (sg == nullptr) break;
        const int n = max(sg->n[0], sg->n[1]), mine = sg->n[t], both = min(sg->n[0], sg->n[1]);
        free_seg(it);
        uint32_t k_tile = 0, v_tile = 0;
        if (tells_entry(t, both)) arrive(kEntry);
        if (!(ok = take(k_tile))) break;
        if (mine > 0) {
          if (!(ok = wait(kQFull + t, qs++))) break;
          tc_fence_after();
          issue_s(s_tmem, dq, dk + k_tile);
          commit(kSFull + t);
          if (mine == 1) commit(kQEmpty + t);
        }
        step_done(mine > 0);
        if (awaits_entry(t, both) && !(ok = wait(kEntry, entries++))) break;
        for (int j = 0; j < n; ++j) {
          if (j < mine && own_turn(t, j, both)) arrive(kPHalf + t);
          if (!(ok = take(v_tile))) break;
          if (j + 1 < n && !(ok = take(k_tile))) break;
          if (j < mine) {
            if (!(ok = wait(kPHalf + t, ps))) break;
            tc_fence_after();
            issue_pv<0, 4>(s_tmem, dv + v_tile, j > 0);
            if (!(ok = wait(kPFull + t, ps++))) break;
            tc_fence_after();
            issue_pv<4, 8>(s_tmem, dv + v_tile, j > 0);
            if (j + 1 < mine) issue_s(s_tmem, dq, dk + k_tile);
            if (passes_turn(t, j, both)) arrive(kPHalf + (t ^ 1));
            if (j + 1 < mine) {
              commit(kSFull + t);
              if (j + 2 == mine) commit(kQEmpty + t);
            } else {
              commit(kOFull + t);
            }
          }
          step_done(j < mine);
        }
      }
      if (elect_lane() && *abort_flag) {
        // error path: let the tensor core finish what was issued before TMEM is freed
        mma_commit(bar(kDrain + t));
        mbar_drain(bar(kDrain + t), 0, 100000000ull);
      }
    } else if (warp == 0) {
      // ================================================================ scheduler and TMA producer
      bool ok = true;
      int at = 0, qc[2] = {0, 0};   // ring place of the next tile, Q tiles copied
      uint32_t armed = 0, checked = 0;   // a bit per ring place: its barrier's turn (full; loaded, for the check)
      int steps = 0, done = 0;      // steps begun, and known to be done
      int step_of = -1;             // lane i: the step of the tile in ring place i
      const int per_tile = kPaged ? 128 >> p.page_log2 : 1;
      const uint32_t page_bytes = kPaged ? (uint32_t)p.page_size * 128u : 0u;   // of half the columns
      // waits until the next ring place is free
      auto place = [&]() {
        const int last = __shfl_sync(0xffffffffu, step_of, at);
        for (; done <= last; ++done)
          if (!wait_warp(bar(kDone + done % kSteps), (uint32_t)(done / kSteps) & 1u, abort_flag, p.dev_status)) return false;
        return true;
      };
      pa::Units units(p);
      if (units.bad) atomicMax(p.dev_status, (int)PTD_ERR_INVALID_BATCH);
      __syncwarp();
      constexpr int kNoUnit = INT_MAX;
      int x = (int)blockIdx.x, claims = 0;   // the next unit's number, if it is known; claims made
      bool claimed = false;                  // the last one has not been read yet
      auto claim = [&]() {
        if (lane == 0) {
          mbar_arrive_expect_tx(bar(kClaim), 16);
          claim_cta(base + kOffClaim, bar(kClaim));
        }
        claimed = true;
        ++claims;
      };
      // The walk: steps of a unit (V of tile j and K of tile j + 1, j = -1 .. n - 1), and before its last ones
      // the claim and the search of the next, so that its first copies follow at once.
      Unit u;                      // the next unit, once it is known
      bool search = true, found = false;
      int it = 0, j = 0, n = 0, search_at = 0, b = 0, kv = 0, kt0 = 0, edge = 0, head0 = 0, row0 = 0, end_page = 0;
      int nq[2] = {0, 0}, next_page = -1, row_v = 0;
      const int* bt = nullptr;
      // this lane's page of key tile i (read a step ahead, so that no copy waits for it)
      auto page_of = [&](int i) {
        const int g = (kt0 + i) * per_tile + lane;
        return kPaged && i < n && lane < per_tile && g < end_page ? bt[g] : -1;
      };
      auto pages_in = [&](int i) { return kPaged ? min(per_tile, end_page - (kt0 + i) * per_tile) : 1; };
      // first row of this lane's page of tile i, or of the tile
      auto row_of = [&](int i, int page) {
        if (!kPaged) return (p.layer * p.batch + b) * p.seq_capacity + (kt0 + i) * 128;
        const bool there = page >= 0 && page < p.num_pages;
        if (!there && lane < pages_in(i)) atomicMax(p.dev_status, (int)PTD_ERR_INVALID_BATCH);
        return there ? (p.layer * p.num_pages + page) * p.page_size : -128;   // (-128: TMA fills zeros)
      };
      auto copy = [&](const CUtensorMap* map, bool check, int i, int row) {   // tile i into the next ring place
        const uint32_t full = bar((check ? kLoadV : kFull) + at), dst = base + kOffRing + (uint32_t)at * kTileBytes;
        if constexpr (kPaged) {
          const int pages = pages_in(i);
          int rows[kPages > 0 ? kPages : 1];
#pragma unroll
          for (int g = 0; g < kPages; ++g) rows[g] = __shfl_sync(0xffffffffu, row, g);
          if (elect_lane()) {
            mbar_arrive_expect_tx(full, (uint32_t)pages * page_bytes * 2u);
#pragma unroll
            for (int g = 0; g < kPages; ++g) {
              if (g < pages) {
                tma_load_3d(dst + (uint32_t)g * page_bytes, map, full, 0, kv, rows[g]);
                tma_load_3d(dst + (uint32_t)g * page_bytes + kHalfBytes, map, full, 64, kv, rows[g]);
              }
            }
          }
        } else {
          if (elect_lane()) {
            mbar_arrive_expect_tx(full, kTileBytes);
            tma_load_3d(dst, map, full, 0, kv, row);
            tma_load_3d(dst + kHalfBytes, map, full, 64, kv, row);
          }
        }
        __syncwarp();
        if (lane == at) step_of = steps;
        armed ^= 1u << at;
        if (check) checked ^= 1u << at;
        if (++at == kTiles) at = 0;
      };
      while (ok) {
        if (search) {   // a unit with keys, or the end of the grid
          search = found = false;
#pragma unroll 1
          while (!found) {
            if (x == kNoUnit) {   // (the first unit is the CTA's own)
              if (!claimed) claim();
              if (!(ok = wait_warp(bar(kClaim), (uint32_t)(claims - 1) & 1u, abort_flag, p.dev_status))) break;
              claimed = false;
              x = claimed_cta(base + kOffClaim);
              fence_proxy_async_smem();
              __syncwarp();
              if (x < 0) break;
            }
            found = units.find(p, x, u);
            if (!found || !units.more(x)) x = kNoUnit;
          }
          if (!ok) break;
        }
        if (j == n) {   // the unit's tiles are all asked for
          if (!(ok = wait_warp(bar(kSegEmpty + (it & 1)), ((uint32_t)(it >> 1) & 1u) ^ 1u, abort_flag, p.dev_status))) break;
          b = u.b, kv = u.kv, kt0 = u.tile0, head0 = u.head0, row0 = u.row0;
          edge = (u.ctx + u.token0 + 1) / 128;
          // M tile 0's last token may see fewer tiles than the block's
          const int tiles0 = (u.ctx + u.token0 + min(u.tokens, p.tile_tokens) + 127) / 128;
          nq[0] = max(0, min(tiles0, u.tile1) - kt0), nq[1] = u.tokens > p.tile_tokens ? u.tile1 - kt0 : 0;
          n = max(nq[0], nq[1]);
          if (lane == 0) {
            Seg s = {};
            s.valid = found;
            if (found) {
              s.b = b;
              s.row0 = row0;
              s.ctx = u.ctx;
              s.token0 = u.token0;
              s.tokens = u.tokens;
              s.head0 = head0;
              s.kv = kv;
              s.piece = u.whole ? -1 : u.place;
              s.kt0 = kt0;
              s.edge = edge;
              s.n[0] = nq[0];
              s.n[1] = nq[1];
            }
            segs[it & 1] = s;
            mbar_arrive(bar(kSegFull + (it & 1)));
          }
          __syncwarp();
          if (!found) break;
          ++it;
          j = -1;
          search_at = n > 2 ? n - 2 : n - 1;
          end_page = kPaged ? (u.ctx + u.token0 + u.tokens + p.page_size - 1) >> p.page_log2 : 0;
          bt = kPaged ? p.block_table + (size_t)b * p.max_pages : nullptr;
          next_page = page_of(0);
        }
        const int row_k = j + 1 < n ? row_of(j + 1, next_page) : 0;
        next_page = page_of(j + 2);
#pragma unroll 1
        for (int k = 0; k < 2 && ok; ++k) {   // V of tile j, then K of tile j + 1
          const int i = j + k;
          if (i < 0 || i >= n) continue;
          if ((ok = place())) copy(k ? &map_k : &map_v, k == 0 && kt0 + j >= edge, i, k ? row_k : row_v);
        }
        if (!ok) break;
        row_v = row_k;
        if (j == -1) {
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            if (!ok || nq[t] == 0 ||
                !(ok = wait_warp(bar(kQEmpty + t), ((uint32_t)qc[t] & 1u) ^ 1u, abort_flag, p.dev_status)))
              continue;
            ++qc[t];
            if (elect_lane()) {
              const uint32_t dst = base + kOffQ + (uint32_t)t * kTileBytes;
              mbar_arrive_expect_tx(bar(kQFull + t), (uint32_t)used * 256u);
              tma_load_3d(dst, &map_q, bar(kQFull + t), 0, head0, row0 + t * p.tile_tokens);
              tma_load_3d(dst + kHalfBytes, &map_q, bar(kQFull + t), 64, head0, row0 + t * p.tile_tokens);
            }
            __syncwarp();
          }
        }
        if (j == search_at - 1 && x == kNoUnit) claim();
        search = j == search_at;
        ++steps;
        ++j;
      }
      if (lane == 0 && *abort_flag) {
        // drain the copies already issued (bounded) before the CTA can exit
        for (int s = 0; s < kTiles; ++s) {
          mbar_drain(bar(kFull + s), ((armed >> s) & 1u) ^ 1u, 100000000ull);
          mbar_drain(bar(kLoadV + s), ((checked >> s) & 1u) ^ 1u, 100000000ull);
        }
        for (int t = 0; t < 2; ++t)
          if (qc[t] > 0) mbar_drain(bar(kQFull + t), (uint32_t)(qc[t] - 1) & 1u, 100000000ull);
        if (claims > 0) mbar_drain(bar(kClaim), (uint32_t)(claims - 1) & 1u, 100000000ull);
      }
    } else {
      // ================================================================ V check
      bool ok = true;
      int tiles = 0;            // of the ring before this unit's
      uint32_t checked = 0;     // a bit per ring place: its barrier's turn
      for (int it = 0; ok; ++it) {
        const volatile Seg* sg = wait_seg(it);
        if (sg == nullptr) break;
        const int n = max(sg->n[0], sg->n[1]), kt0 = sg->kt0, edge = sg->edge;
        const int first = sg->ctx + sg->token0 + 1, end = first - 1 + sg->tokens;   // keys that only some see
        for (int j = max(0, edge - kt0); j < n; ++j) {
          int vs = tiles + 2 * j + 1;   // (the tiles go K_0, V_0, K_1, V_1, ..)
          vs -= vs / kTiles * kTiles;
          if (!(ok = wait_warp<kUnitTries>(bar(kLoadV + vs), (checked >> vs) & 1u, abort_flag, p.dev_status))) break;
          checked ^= 1u << vs;
          // 16-byte chunks: rows of the first half (64 columns), then of the second.  Rows that all of the block's
          // tokens see stay as they are, rows behind the block's last token become 0.
          uint4* tile = reinterpret_cast<uint4*>(smem + kOffRing + (size_t)vs * kTileBytes);
          const int r0 = max(0, first - (kt0 + j) * 128), r1 = min(128, end - (kt0 + j) * 128);
          const int half = ((lane >> 3) & 1) * 1024;   // two rows a turn, sixteen lanes each
#pragma unroll 8
          for (int r = r1 + (lane >> 4); r < 128; r += 2) tile[half + r * 8 + (lane & 7)] = make_uint4(0, 0, 0, 0);
          uint32_t bad = 0u;
#pragma unroll 8
          for (int r = r0 + (lane >> 4); r < r1; r += 2) {
            const uint4 v = tile[half + r * 8 + (lane & 7)];
            bad |= exponent_full(v.x) | exponent_full(v.y) | exponent_full(v.z) | exponent_full(v.w);
          }
          if (__any_sync(0xffffffffu, (bad & 0x80008000u) != 0u)) {
            for (int r = r0 + (lane >> 4); r < r1; r += 2) {
              uint4 v = tile[half + r * 8 + (lane & 7)];
              v.x = finite_or_zero(v.x), v.y = finite_or_zero(v.y), v.z = finite_or_zero(v.z), v.w = finite_or_zero(v.w);
              tile[half + r * 8 + (lane & 7)] = v;
            }
            if (lane == 0) segs[it & 1].bad = 1;
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(kFull + vs));
        }
        tiles = (tiles + 2 * n) % kTiles;
        free_seg(it);
      }
    }
  } else {
    // ================================================================ softmax / epilogue
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsMany));
    const int t = (warp - 4) >> 2;
    const int row = (warp & 3) * 32 + lane;   // = TMEM lane this warp may access
    const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t tS = tmem + lane_base + (uint32_t)t * 128u, tO = tS + 256u;
    const int my_token = t * p.tile_tokens + divide(row, p.by_sub), my_head = row - divide(row, p.by_sub) * p.sub;
    const bool in_tile = row < used;
    int tiles = 0, outs = 0;
    for (int it = 0;; ++it) {
      const volatile Seg* sg = wait_seg(it);
      if (sg == nullptr) break;
      const int n = sg->n[t], kt0 = sg->kt0, tokens = sg->tokens, q0 = sg->ctx + sg->token0;
      const int pos = q0 + min(my_token, tokens - 1);   // the last key that this row sees
      const bool row_valid = in_tile && my_token < tokens;
      const int whole = (q0 + t * p.tile_tokens + 1) / 128;   // first key tile that some row sees in part
      // a warp without rows leaves what it finds: its rows of O are not read
      const bool any_row = (warp & 3) * 32 < min(used, (tokens - t * p.tile_tokens) * p.sub);
      float m_run = -INFINITY, l_run = 0.f;
      bool ok = true;
      for (int j = 0; j < n; ++j, ++tiles) {
        if (!(ok = wait_warp(bar(kSFull + t), (uint32_t)tiles & 1u, abort_flag, p.dev_status))) break;
        tc_fence_after();
        if (any_row)
          softmax_tile(tS, tO, j > 0, kt0 + j >= whole, pos - (kt0 + j) * 128, p.scale_log2, m_run, l_run, bar(kPHalf + t));
        else if (lane == 0)
          mbar_arrive(bar(kPHalf + t));
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(kPFull + t));
      }
      if (!ok) break;
      if (n > 0) {
        if (!wait_warp(bar(kOFull + t), (uint32_t)outs & 1u, abort_flag, p.dev_status)) break;
        ++outs;
        tc_fence_after();
      }
      const bool bad = sg->bad != 0;
      const int piece = sg->piece;
      const float inv = piece < 0 ? 1.f / l_run : 1.f;   // a piece stays unnormalised
      float4* po = reinterpret_cast<float4*>(p.part_o) + (size_t)max(piece, 0) * 32 * 256 + t * 128 + row;
      if (piece >= 0 && row_valid)
        reinterpret_cast<float2*>(p.part_ml)[(size_t)piece * 256 + t * 128 + row] =
            n > 0 ? make_float2(m_run, l_run) : make_float2(-INFINITY, 0.f);
      if (n > 0 && any_row) {
        const bool wide = (reinterpret_cast<uintptr_t>(p.out) & 31u) == 0;
        uint4* dst = reinterpret_cast<uint4*>(p.out) + (((size_t)sg->row0 + my_token) * p.hq + sg->head0 + my_head) * 16;
#pragma unroll 1
        for (int c = 0; c < 8; ++c) {
          uint32_t r[16];
          tmem_ld16(tO + (uint32_t)c * 16u, r);
          tmem_ld_wait();
          if (bad && row_valid) {
            float ob[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) ob[e] = __uint_as_float(r[e]) * inv;
            add_bad<kPaged>(p, ob, sg->b, sg->kv, c * 16, max(kt0, sg->edge) * 128, min(pos, (kt0 + n) * 128 - 1));
#pragma unroll
            for (int e = 0; e < 16; ++e) r[e] = __float_as_uint(ob[e]);
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) r[e] = __float_as_uint(__uint_as_float(r[e]) * inv);
          }
          if (row_valid) {
            if (piece < 0) {
              uint32_t w[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) w[e] = pack_bf16x2(__uint_as_float(r[2 * e]), __uint_as_float(r[2 * e + 1]));
              store_row(dst + c * 2, w, wide);
            } else {
#pragma unroll
              for (int g = 0; g < 4; ++g)
                po[(size_t)(c * 4 + g) * 256] = make_float4(__uint_as_float(r[4 * g]), __uint_as_float(r[4 * g + 1]),
                                                            __uint_as_float(r[4 * g + 2]), __uint_as_float(r[4 * g + 3]));
            }
          }
          __syncwarp();
        }
      }
      tc_fence_before();
      free_seg(it);
    }
  }

  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, tc::kTmemCols);
  }
}

}  // namespace pt

cudaError_t launch_prompt_attn_tc(const CUtensorMap& map_k, const CUtensorMap& map_v, const CUtensorMap& map_q,
                                  const PromptAttnParams& p, cudaStream_t stream) {
  const auto kernel = p.page_size == 0 ? pt::prompt_tc_kernel<0> : (p.page_size >= 64 ? pt::prompt_tc_kernel<2> : pt::prompt_tc_kernel<8>);
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)pt::kSmemBytes);
  if (e != cudaSuccess) return e;
  const int units = p.blocks * p.tile_heads * p.splits, shares = p.cut_ctas > 0 ? p.most_shares : 0;
  return launch_chained(kernel, dim3((unsigned)(units > shares ? units : shares)), dim3(pt::kThreads), pt::kSmemBytes,
                        stream, 0, map_k, map_v, map_q, p);
}

}  // namespace ptd
