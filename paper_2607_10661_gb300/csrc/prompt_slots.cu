// Pages, block tables, cache slots and positions of a packed batch of new tokens.
//
// Sequence b, with C_b positions in the cache and n_b new ones, needs ceil((C_b + n_b) / P) pages of P
// positions and holds held_b.  With g_b = max(0, held_b - need_b) and t_b = max(0, need_b - held_b), their
// exclusive sums G_b and T_b over the sequences, G and T in all, and a stack of f free pages:
//   the page given back with rank r (sequence b with G_b <= r < G_b + g_b) is block_table[b][need_b + r - G_b];
//   the page taken with rank r comes from the top: given page G - 1 - r while r < G, else free_pages[f - 1 - (r - G)];
//   the given pages of rank r < G - T stay on the stack, at free_pages[f + r].
// So every moved page, and every token's page, is a function of the two sums alone.  Each CTA forms the
// sums of the whole batch in shared memory (a few loads a thread) and takes its share of the tokens and of the
// moved pages: no CTA waits for another, and one launch does it all.  The new counts go to buffers of their
// own, as other CTAs still read the old ones; the block-table entries written lie behind those read.
//
// What bounds it: latency (a launch, two dependent reads, a scan, a search, the page, the write): 256 requests of
// up to 4096 positions, one token each, some finished and some new, 3.3 us, 1024 of them 4.4 us, one 2.4 us, 96 prompts
// of up to 4096 tokens 4.0 us.  Bytes matter from some 10^6 tokens on.
#include <cuda_runtime.h>

#include <cstdint>

#include "launch.cuh"
#include "prompt.cuh"
#include "ptd_device.cuh"

namespace ptd {
namespace ps {

constexpr int kThreads = 512;
// Dynamic shared memory of the largest batch.  The limit belongs to the kernel, not to a launch: a call that set its own
// batch's size could lower it between another thread's call and its launch.
constexpr size_t kMostSmem = (5 * (size_t)PTD_MAX_PROMPT_BATCH + 1) * sizeof(int);

// The last i in [0, n) with a[i] <= x (a[0] <= x; a non-decreasing).
__device__ __forceinline__ int last_at_most(const int* a, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

template <bool kPool>
__global__ void __launch_bounds__(kThreads) prompt_slots_kernel(const PromptSlotsParams p, int tokens_per_cta) {
  extern __shared__ int smem[];
  __shared__ unsigned long long warp_sum[kThreads / 32];
  __shared__ unsigned long long total_s;
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5, B = p.batch;
  int* off = smem;              // [B + 1]
  int* ctx = off + B + 1;       // [B]
  int* held = ctx + B;          // [B], with a pool, as the next two
  int* gives = held + B;        // exclusive sums
  int* takes = gives + B;
  if (t == 0) grid_launch_dependents();
  grid_dependency_wait();
  for (int b = t; b <= B; b += kThreads) {
    off[b] = p.token_offsets[b];
    if (b < B) {
      ctx[b] = p.ctx_lens[b];
      if (kPool) held[b] = p.held[b];
    }
  }
  const int f = kPool ? *p.free_count : 0;
  __syncthreads();
  // a thread's run of sequences
  const int per = (B + kThreads - 1) / kThreads, b0 = min(B, t * per), b1 = min(B, b0 + per);
  bool bad = kPool && (f < 0 || f > p.num_pages);
  unsigned long long sum = 0ull;   // pages taken << 32 | given
  // (a valid sequence's positions fit its table row, and so an int)
  auto need_of = [&](int b) { return (ctx[b] + (off[b + 1] - off[b]) + p.page_size - 1) >> p.page_log2; };
  for (int b = b0; b < b1; ++b) {
    const bool ok = prompt_sequence_ok(p.bounds, off[b], off[b + 1], ctx[b]) &&
                    (!kPool || (held[b] >= 0 && held[b] <= p.max_pages));
    bad = bad || !ok;
    if (kPool && ok) {
      const int d = need_of(b) - held[b];
      sum += d > 0 ? (unsigned long long)d << 32 : (unsigned long long)(unsigned)(-d);
    }
  }
  bool refused = false;
  int G = 0, T = 0;
  if (kPool) {
    unsigned long long incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned long long y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    if (lane == 31) warp_sum[warp] = incl;
    bad = __syncthreads_or(bad) != 0;
    if (warp == 0) {
      unsigned long long w = lane < kThreads / 32 ? warp_sum[lane] : 0ull;
#pragma unroll
      for (int o = 1; o < kThreads / 32; o <<= 1) {
        const unsigned long long y = __shfl_up_sync(0xffffffffu, w, o);
        if (lane >= o) w += y;
      }
      if (lane < kThreads / 32) warp_sum[lane] = w;
      if (lane == kThreads / 32 - 1) total_s = w;
    }
    __syncthreads();
    unsigned long long at = (warp > 0 ? warp_sum[warp - 1] : 0ull) + incl - sum;
    G = (int)(unsigned)total_s;
    T = (int)(total_s >> 32);
    bad = bad || (int64_t)f + G - T > p.num_pages;   // more pages than there are: some page is held twice
    refused = bad || (int64_t)T > (int64_t)f + G;
    if (!bad) {
      for (int b = b0; b < b1; ++b) {
        gives[b] = (int)(unsigned)at;
        takes[b] = (int)(at >> 32);
        const int d = need_of(b) - held[b];
        at += d > 0 ? (unsigned long long)d << 32 : (unsigned long long)(unsigned)(-d);
      }
    }
    if (blockIdx.x == 0) {
      for (int b = b0; b < b1; ++b) p.new_held[b] = refused ? held[b] : need_of(b);
      if (t == 0) {
        *p.new_free_count = refused ? f : f + G - T;
        if (refused) atomicMax(p.dev_status, bad ? (int)PTD_ERR_INVALID_BATCH : (int)PTD_ERR_NO_PAGES);
      }
    }
    __syncthreads();
  } else {
    bad = __syncthreads_or(bad) != 0;
    if (bad && blockIdx.x == 0 && t == 0) atomicMax(p.dev_status, (int)PTD_ERR_INVALID_BATCH);
  }
  auto given = [&](int r) {   // the page given back with rank r
    const int b = last_at_most(gives, B, r);
    return p.block_table[(size_t)b * p.max_pages + need_of(b) + (r - gives[b])];
  };
  auto taken = [&](int r) { return r < G ? given(G - 1 - r) : p.free_pages[f - 1 - (r - G)]; };
  if (kPool && !refused) {
    // the last CTAs first: the first ones have the tokens
    const int step = gridDim.x * kThreads, r0 = ((int)gridDim.x - 1 - (int)blockIdx.x) * kThreads + t;
    for (int r = r0; r < T; r += step) {
      const int b = last_at_most(takes, B, r);
      p.table_out[(size_t)b * p.max_pages + held[b] + (r - takes[b])] = taken(r);
    }
    for (int r = r0; r < G - T; r += step) p.free_pages[f + r] = given(r);
  }
  const int n0 = (int)min((int64_t)p.bounds.n_total, (int64_t)blockIdx.x * tokens_per_cta);
  const int n1 = min(p.bounds.n_total, n0 + tokens_per_cta);
  for (int n = n0 + t; n < n1; n += kThreads) {
    int slot = -1, pos = -1;
    if (!refused && n >= off[0] && n < off[B]) {
      const int b = last_at_most(off, B, n);
      if (n < off[b + 1] && (!bad || prompt_sequence_ok(p.bounds, off[b], off[b + 1], ctx[b]))) {
        pos = ctx[b] + (n - off[b]);
        if (p.page_size == 0) {
          slot = b * p.seq_capacity + pos;
        } else {
          const int i = pos >> p.page_log2;
          const int page = !kPool || i < held[b] ? p.block_table[(size_t)b * p.max_pages + i] : taken(takes[b] + i - held[b]);
          if (page >= 0 && page < p.num_pages) {
            slot = (page << p.page_log2) + (pos & (p.page_size - 1));
          } else {
            pos = -1;
            atomicMax(p.dev_status, (int)PTD_ERR_INVALID_BATCH);
          }
        }
      }
    }
    p.slots[n] = slot;
    p.positions[n] = pos;
  }
}

}  // namespace ps

cudaError_t launch_prompt_slots(const PromptSlotsParams& p, int sms, cudaStream_t stream) {
  const bool pool = p.free_pages != nullptr;
  const size_t smem = ((pool ? 5 : 2) * (size_t)p.batch + 1) * sizeof(int);
  int ctas = (p.bounds.n_total + ps::kThreads - 1) / ps::kThreads;
  if (ctas > sms) ctas = sms;
  const int per = (p.bounds.n_total + ctas - 1) / ctas;
  // Pages move beside the tokens, not before them, and a finished request has many: by CTAs, 4: 256 requests 4.4 us,
  // 1024 10.6; 16: 3.3 and 5.6; 48: 3.3 and 4.4; 152: 3.5 and 4.4.
  if (pool && ctas < 48) ctas = 48;
  const auto kernel = pool ? ps::prompt_slots_kernel<true> : ps::prompt_slots_kernel<false>;
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)ps::kMostSmem);
    if (e != cudaSuccess) return e;
  }
  return launch_chained(kernel, dim3(ctas), dim3(ps::kThreads), smem, stream, 0, p, per);
}

}  // namespace ptd
