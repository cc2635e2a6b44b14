// Forks of paged sequences: every target sequence goes on from the first n tokens of a source sequence.
//
// With P positions a page, target b takes the first floor(n_b / P) pages of its parent's row as they are (shared, full pages
// are not written again) and, where n_b % P positions are left, the page behind them: for itself alone.  Let u[x] be -1 if
// some target has page x as a full one, else the lowest target that has it as its last, partial one, else none:
//   target b keeps its partial page x if u[x] = b, otherwise it takes a free page and the x's first n_b % P rows are copied;
//   a page of the source rows with no u is given back, by the lowest source row that holds it.
// The free page taken with rank r (by target) is free[f - 1 - r], the given page of rank r (by source row, index) goes to
// free[f - T + r] of the new stack: everything is a function of u, of each page's first holder and of two sums, and the
// result does not depend on the order in which threads run (minima alone are made by atomics).
//
// The plan reads every source entry once: with m the most full pages that a target has of the row, entry i < m is full
// somewhere (u = -1), and only what lies behind can be given or kept.  Between its parts (sizes and m; u and the holders; counts;
// sums, stack and list of copies) all threads wait for one another: one CTA does it with u and the holders in its shared memory
// where they fit and the rows are few enough, else a cluster of eight with both in the scratch.  Then a grid copies: table
// rows, the rest of the stack, and K/V rows of all layers in chunks.
//
// What bounds it: the plan's latency (a chain of small reads, barriers and code that runs once: entries eight or sixteen at a
// time, or the two sums one after the other, were slower for their longer code), then the copies' writes.  GB300, graph replays:
// one prompt of 2043 positions continued 64 times, 32 layers of 8 KV heads, 20.1 - 22.4 us (91 MB written, the source comes from L2);
// 128 beams of some 60 pages, 8 layers, 12.5 - 13.4; 2048 beams of 140 pages in one layer 56.  At first, with target entries marked
// one by one, every row's entries ranked and the tables written by the plan, 36.3, 20.2 and 90.
// The pool counts too (u and the holders are cleared, the stack is looked over and copied): that prompt in 4 layers with 300 pages
// 8.9 us, with 20000 10.5, with 30000, which the cluster plans, 12.4, with 100000 14.0.
// (A CTA that keeps a source chunk in registers for the next copy of the same page, or the table prefetched while the sizes
// are looked at: 0.5 - 1 us more.)
#include <cuda_runtime.h>

#include <climits>
#include <cstdint>

#include "launch.cuh"
#include "page_fork.cuh"
#include "ptd_device.cuh"
#include "row_division.cuh"

namespace ptd {
namespace pf {

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int kCtas = 8;           // of the planning cluster
constexpr int kNone = INT_MAX;
constexpr int kCopyThreads = 256, kCopyLoads = 4;
constexpr int kChunk = kCopyThreads * kCopyLoads * 16;   // bytes of one CTA's turn

constexpr int kRefused = -1;
struct Scratch {
  int32_t* bad;       // [1] a page number out of range
  int32_t* copies;    // [1] T, or kRefused
  int32_t* fresh;     // [to_batch] the page taken, or -1
  int32_t* copy;      // [to_batch][3] from page, to page, rows
  int32_t* gives;     // the cluster's: [from_batch] pages given back
  int32_t* lead;      // [from_batch] the index of the first of them
  int32_t* takes;     // [to_batch] 0 or 1
  int32_t* first;     // [num_pages] lowest source row that could give the page
  int32_t* user;      // [num_pages] u
  __host__ __device__ Scratch(int32_t* at, int num_pages, int from_batch, int to_batch)
      : bad(at), copies(at + 1), fresh(at + 4), copy(fresh + to_batch), gives(copy + 3 * (size_t)to_batch),
        lead(gives + from_batch), takes(lead + from_batch), first(takes + to_batch), user(first + num_pages) {}
};

// Exclusive sums of n pairs (two counts in one word), by the whole CTA: load(i) is a pair, store(i, sums) takes what comes before
// it (after every load of the thread's own run); the totals to every thread.
template <typename Load, typename Store>
__device__ __forceinline__ unsigned long long exclusive_sums(int n, unsigned long long* warp_s, Load load, Store store) {
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int per = (n + kThreads - 1) / kThreads, i0 = min(n, t * per), i1 = min(n, i0 + per);
  unsigned long long sum = 0ull;
#pragma unroll 1
  for (int i = i0; i < i1; ++i) sum += load(i);
  unsigned long long incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long y = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += y;
  }
  if (lane == 31) warp_s[warp] = incl;
  __syncthreads();
  const unsigned long long w = warp_s[lane], b = lane < warp ? w : 0ull;   // as many warps as lanes
  const auto add = [](unsigned long long x) {
    return (unsigned long long)__reduce_add_sync(0xffffffffu, (unsigned)(x >> 32)) << 32 | __reduce_add_sync(0xffffffffu, (unsigned)x);
  };
  unsigned long long at = add(b) + incl - sum;
#pragma unroll 1
  for (int i = i0; i < i1; ++i) {
    const unsigned long long x = load(i);
    store(i, at);
    at += x;
  }
  const unsigned long long total = add(w);
  __syncthreads();
  return total;
}

// Rows' entries to threads: each row by a group of 2^k neighbouring threads of the plan (8 at least), as many as there are
// for a row, kUnroll entries of a thread in flight: f(row, index, entry) for every index of [begin(row), end(row)).
constexpr int kUnroll = 4;
__device__ __forceinline__ int group_of(int rows, int all) {
  int group = 8;
  while (group < all && (int64_t)rows * group * 2 <= all) group *= 2;
  return group;
}
template <typename Begin, typename End, typename Row, typename F>
__device__ __forceinline__ void for_entries(int rows, int me, int all, Begin begin, End end, Row row_of, F f) {
  const int group = group_of(rows, all);
  for (int b = me / group; b < rows; b += all / group) {
    const int n = end(b);
    const int32_t* row = row_of(b);
    for (int i0 = begin(b) + (me & (group - 1)); i0 < n; i0 += kUnroll * group) {
      int x[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) x[u] = i0 + u * group < n ? __ldg(row + i0 + u * group) : -1;
#pragma unroll
      for (int u = 0; u < kUnroll; ++u)
        if (i0 + u * group < n) f(b, i0 + u * group, x[u]);
    }
  }
}

// f(i, a[i]) for i = me, me + all, ... < n, kUnroll of them in flight.
template <typename F>
__device__ __forceinline__ void for_stack(const int32_t* a, int n, int me, int all, F f) {
  for (int i0 = me; i0 < n; i0 += kUnroll * all) {
    int x[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) x[u] = i0 + u * all < n ? __ldg(a + i0 + u * all) : 0;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (i0 + u * all < n) f(i0 + u * all, x[u]);
  }
}

template <bool kOne>   // one CTA, else a cluster of kCtas
__global__ void __launch_bounds__(kThreads, 1) page_fork_plan_kernel(const __grid_constant__ PageForkParams p) {
  extern __shared__ int smem[];
  __shared__ unsigned long long warp_s[kWarps];
  __shared__ int bad_s;
  const int F = p.from_batch, B = p.to_batch, W = p.max_pages, log2p = p.page_log2, below = (1 << log2p) - 1;
  int* held = smem;             // [F]
  int* most = held + F;         // [F] m
  int* gives_s = most + F;      // [F] counts (one CTA), then exclusive sums
  int* parent = gives_s + F;    // [B]
  int* tokens = parent + B;     // [B] 0 without a parent
  int* takes_s = tokens + B;    // [B]
  const Scratch sc(p.scratch, p.num_pages, F, B);
  int* lead = kOne ? takes_s + B : sc.lead;
  int* first = kOne ? lead + F : sc.first;
  int* user = kOne ? first + p.num_pages : sc.user;
  int* bad_page = kOne ? &bad_s : sc.bad;
  const int t = threadIdx.x, lane = t & 31, cta = kOne ? 0 : blockIdx.x;
  constexpr int all = (kOne ? 1 : kCtas) * kThreads, warps = all / 32;   // of the plan
  const int me = cta * kThreads + t, my_warp = cta * kWarps + (t >> 5);
  auto barrier = [&] {
    if constexpr (kOne) {
      __syncthreads();
    } else {
      asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
      asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
  };
  auto seen = [&](const int* x) { return kOne ? *(volatile const int*)x : __ldcg(x); };   // what other threads wrote
  if (t == 0) grid_launch_dependents();
  grid_dependency_wait();

  // the sizes and m, by every CTA; nothing is known of any page
  const int f = *p.free_count;
  bool bad = f < 0 || f > p.num_pages;
  for (int b = t; b < F; b += kThreads) {
    const int n = p.held[b];
    held[b] = n;
    most[b] = 0;
    if (kOne) gives_s[b] = 0; else if (cta == 0) sc.gives[b] = 0;
    if (cta == 0) lead[b] = kNone;
    bad = bad || n < 0 || n > W;
  }
  for (int b = t; b < B; b += kThreads) {
    const int from = p.parents[b], n = p.lens[b];
    parent[b] = from;
    tokens[b] = from == -1 ? 0 : n;
    bad = bad || from < -1 || from >= F;
  }
  for (int x = me; x < p.num_pages; x += all) first[x] = user[x] = kNone;
  if (me == 0) *bad_page = 0;
  bad = __syncthreads_or(bad) != 0;   // the same in every CTA
  if (!bad) {
    bool out = false;
    for (int b = t; b < B; b += kThreads) {
      const int from = parent[b], n = tokens[b];
      if (from < 0) continue;
      out = out || n < 0 || (n + (int64_t)below) >> log2p > held[from];
      if (n >> log2p > most[from]) atomicMax(most + from, n >> log2p);
    }
    bad = out;
  }
  bad = __syncthreads_or(bad) != 0;
  barrier();

  auto zero = [](int) { return 0; };
  auto held_of = [&](int b) { return held[b]; };
  auto source_row = [&](int b) { return p.table + (size_t)b * W; };
  auto last_page = [&](int b) { return __ldg(source_row(parent[b]) + (tokens[b] >> log2p)); };   // of a target with a partial one
  if (!bad) {
    bool out = false;
    for_entries(F, me, all, zero, held_of, source_row, [&](int b, int i, int x) {
      if (x < 0 || x >= p.num_pages) {
        out = true;
      } else if (i >= most[b]) {
        atomicMin(first + x, b);
      } else {
        atomicMin(user + x, -1);
      }
    });
    for (int b = me; b < B; b += all)
      if ((tokens[b] & below) != 0) {
        const int x = last_page(b);
        if (x >= 0 && x < p.num_pages) atomicMin(user + x, b);
      }
    for_stack(p.free_pages, f, me, all, [&](int, int x) { out = out || x < 0 || x >= p.num_pages; });
    if (out) atomicOr(bad_page, 1);
  }
  barrier();
  bad = bad || seen(bad_page) != 0;

  // what each row gives and takes
  auto given = [&](int b, int x) { return seen(first + x) == b && seen(user + x) == kNone; };
  if (!bad) {
    const int group = group_of(F, all);
    for (int b = me / group; b < F; b += all / group) {   // (uniform in a warp where the group is one or more)
      int count = 0, least = kNone;
      const int n = held[b];
      for (int i0 = most[b] + (me & (group - 1)); i0 < n; i0 += kUnroll * group) {
        int x[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) x[u] = i0 + u * group < n ? __ldg(source_row(b) + i0 + u * group) : -1;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
          if (x[u] >= 0 && given(b, x[u])) ++count, least = min(least, i0 + u * group);
      }
      if (group >= 32) {
        const int sum = __reduce_add_sync(0xffffffffu, count);
        least = __reduce_min_sync(0xffffffffu, least);
        count = lane == 0 ? sum : 0;
      }
      if (count > 0) {
        atomicAdd(kOne ? gives_s + b : sc.gives + b, count);
        atomicMin(lead + b, least);
      }
    }
    for (int b = me; b < B; b += all) {
      const int takes = (tokens[b] & below) != 0 && seen(user + last_page(b)) != b ? 1 : 0;
      if (kOne) takes_s[b] = takes; else sc.takes[b] = takes;
    }
  }
  barrier();

  int G = 0, T = 0;
  if (!bad) {
    const unsigned long long total = exclusive_sums(
        max(F, B), warp_s,
        [&](int i) {
          const unsigned gives = i < F ? (unsigned)(kOne ? gives_s[i] : __ldcg(sc.gives + i)) : 0u;
          const unsigned takes = i < B ? (unsigned)(kOne ? takes_s[i] : __ldcg(sc.takes + i)) : 0u;
          return (unsigned long long)takes << 32 | gives;
        },
        [&](int i, unsigned long long before) {
          if (i < F) gives_s[i] = (int)(unsigned)before;
          if (i < B) takes_s[i] = (int)(before >> 32);
        });
    G = (int)(unsigned)total;
    T = (int)(total >> 32);
  }
  bad = bad || (int64_t)f - T + G > p.num_pages;   // more pages than there are: some page is held and free
  const bool refused = bad || T > f;
  if (me == 0) {
    *p.new_free_count = refused ? 0 : f - T + G;
    *sc.copies = refused ? kRefused : T;
    if (refused) atomicMax(p.dev_status, bad ? (int)PTD_ERR_INVALID_BATCH : (int)PTD_ERR_NO_PAGES);
  }
  for (int b = me; b < B; b += all) {
    p.new_held[b] = refused ? 0 : (int)(((unsigned)tokens[b] + (unsigned)below) >> log2p);
    if (refused) continue;
    const int rank = takes_s[b];
    int fresh = -1;
    if ((b + 1 < B ? takes_s[b + 1] : T) != rank) {
      fresh = p.free_pages[f - 1 - rank];
      sc.copy[3 * rank] = last_page(b);
      sc.copy[3 * rank + 1] = fresh;
      sc.copy[3 * rank + 2] = tokens[b] & below;
    }
    sc.fresh[b] = fresh;
  }
  if (refused) return;
  for (int b = my_warp; b < F; b += warps) {
    if ((b + 1 < F ? gives_s[b + 1] : G) == gives_s[b]) continue;
    int at = f - T + gives_s[b];
    for (int i0 = seen(lead + b); i0 < held[b]; i0 += 32 * kUnroll) {
      int x[kUnroll];
      bool mine[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) x[u] = i0 + 32 * u + lane < held[b] ? __ldg(source_row(b) + i0 + 32 * u + lane) : -1;
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) mine[u] = x[u] >= 0 && given(b, x[u]);
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const uint32_t mask = __ballot_sync(0xffffffffu, mine[u]);
        const int place = at + __popc(mask & ((1u << lane) - 1u));
        if (mine[u] && place < p.num_pages) p.new_free_pages[place] = x[u];
        at += __popc(mask);
      }
    }
  }
}

// K and V rows: a CTA's turn is one chunk of a copy's bytes in one layer's K or V (the grid's y); then table rows by warps and what
// stays of the stack by threads.
__global__ void __launch_bounds__(kCopyThreads)
    page_copy_kernel(const __grid_constant__ PageForkParams p, int chunks, IndexDivisor by_chunks) {
  const Scratch sc(p.scratch, p.num_pages, p.from_batch, p.to_batch);
  if (threadIdx.x == 0) grid_launch_dependents();
  grid_dependency_wait();
  const int copies = *sc.copies;
  if (copies == kRefused) return;
  const int64_t page_bytes = p.row_bytes << p.page_log2, layer_bytes = p.num_pages * page_bytes;
  for (int turn = blockIdx.x; turn < copies * chunks; turn += gridDim.x) {
    const int c = divide(turn, by_chunks);
    const int from = sc.copy[3 * c], to = sc.copy[3 * c + 1];
    const int64_t at = (int64_t)(turn - c * chunks) * kChunk, left = (sc.copy[3 * c + 2] * p.row_bytes - at) / 16;
    if (left <= 0) continue;
    const int n = (int)min(left, (int64_t)(kChunk / 16)) - (int)threadIdx.x;   // vectors from this thread's first on
    const int64_t src_at = from * page_bytes + at, dst_at = to * page_bytes + at;
    for (int plane = blockIdx.y; plane < 2 * p.num_layers; plane += gridDim.y) {
      uint8_t* base = static_cast<uint8_t*>((plane & 1) != 0 ? p.v : p.k) + (plane >> 1) * layer_bytes;
      const uint4* src = reinterpret_cast<const uint4*>(base + src_at) + threadIdx.x;
      uint4* dst = reinterpret_cast<uint4*>(base + dst_at) + threadIdx.x;
      uint4 x[kCopyLoads];
#pragma unroll
      for (int u = 0; u < kCopyLoads; ++u)
        if (u * kCopyThreads < n) x[u] = src[u * kCopyThreads];
#pragma unroll
      for (int u = 0; u < kCopyLoads; ++u)
        if (u * kCopyThreads < n) dst[u * kCopyThreads] = x[u];
    }
  }
  // the last CTAs first: the first ones have the copies
  const int ctas = (int)(gridDim.x * gridDim.y), cta = ctas - 1 - (int)(blockIdx.y * gridDim.x + blockIdx.x);
  const int all = ctas * kCopyThreads, me = cta * kCopyThreads + (int)threadIdx.x;
  for (int b = me >> 5; b < p.to_batch; b += all >> 5) {
    const int need = p.new_held[b], fresh = sc.fresh[b];
    const int32_t* row = p.table + (size_t)max(p.parents[b], 0) * p.max_pages;
    int32_t* to = p.new_table + (size_t)b * p.max_pages;
    for_stack(row, need, threadIdx.x & 31, 32, [&](int i, int x) { to[i] = i == need - 1 && fresh >= 0 ? fresh : x; });
  }
  for_stack(p.free_pages, *p.free_count - copies, me, all, [&](int i, int x) { p.new_free_pages[i] = x; });
}

}  // namespace pf

int page_copy_chunks(int64_t page_bytes) {
  const int64_t n = (page_bytes + pf::kChunk - 1) / pf::kChunk;
  return n < INT_MAX ? (int)n : INT_MAX;
}

size_t page_fork_scratch_ints(int num_pages, int from_batch, int to_batch) {
  return 4 + 2 * (size_t)num_pages + 2 * (size_t)from_batch + 5 * (size_t)to_batch;
}

cudaError_t launch_page_fork(const PageForkParams& p, int sms, cudaStream_t stream) {
  constexpr size_t kMostSmem = 6 * (size_t)PTD_MAX_PROMPT_BATCH * sizeof(int), kMostOneSmem = 200 * 1024;
  const size_t sizes = 3 * ((size_t)p.from_batch + p.to_batch) * sizeof(int);
  const size_t with_pages = sizes + ((size_t)p.from_batch + 2 * (size_t)p.num_pages) * sizeof(int);
  // (us, one CTA and the cluster: 32 source rows of 71 entries 7.5 and 10.9, 1 of 1000 9.1 and 11.2, 128 of 71 12.5 and 13.0,
  // [the rule's bound] 256 of 140 19.7 and 14.4, 512 of 140 33 and 21.6)
  const bool one = with_pages <= kMostOneSmem && (int64_t)p.from_batch * p.max_pages <= 12288;
  const size_t smem = one ? with_pages : sizes;
  cudaError_t e = cudaSuccess;
  if (smem > 47 * 1024) {   // the limits are the kernels', the same for every call
    if (one)
      e = cudaFuncSetAttribute(pf::page_fork_plan_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostOneSmem);
    else
      e = cudaFuncSetAttribute(pf::page_fork_plan_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostSmem);
    if (e != cudaSuccess) return e;
  }
  e = launch_chained(one ? pf::page_fork_plan_kernel<true> : pf::page_fork_plan_kernel<false>,
                                       dim3(one ? 1 : pf::kCtas), dim3(pf::kThreads), smem, stream, one ? 0 : pf::kCtas, p);
  if (e != cudaSuccess) return e;
  const int chunks = page_copy_chunks(p.row_bytes << p.page_log2);
  // eight CTAs an SM, but no more than there may be turns
  const int64_t planes = 2 * (int64_t)p.num_layers < 64 ? 2 * (int64_t)p.num_layers : 64, turns = (int64_t)p.to_batch * chunks;
  const int64_t places = (8 * (int64_t)sms + planes - 1) / planes;
  return launch_chained(pf::page_copy_kernel, dim3((unsigned)(turns < places ? turns : places), (unsigned)planes),
                        dim3(pf::kCopyThreads), 0, stream, 0, p, chunks, index_divisor(chunks));
}

}  // namespace ptd
