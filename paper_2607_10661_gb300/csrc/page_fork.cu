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
// One cluster plans (u and the holders; counts of each row; sums, the new tables and stack, the list of copies), with three
// cluster barriers between these; then a grid copies rows, all layers of K and V, in chunks.
#include <cuda_runtime.h>

#include <climits>
#include <cstdint>

#include "launch.cuh"
#include "page_fork.cuh"
#include "ptd_device.cuh"

namespace ptd {
namespace pf {

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int kCtas = 8;           // of the planning cluster
constexpr int kNone = INT_MAX;
constexpr int kCopyThreads = 256, kCopyLoads = 4;
constexpr int kChunk = kCopyThreads * kCopyLoads * 16;   // bytes of one CTA's turn

struct Scratch {
  int32_t* bad;       // [1] a page number out of range
  int32_t* copies;    // [1]
  int32_t* first;     // [num_pages] lowest source row that holds the page
  int32_t* user;      // [num_pages] u
  int32_t* gives;     // [from_batch] pages given back
  int32_t* takes;     // [to_batch] 0 or 1
  int32_t* copy;      // [to_batch][3] from page, to page, rows
  __host__ __device__ Scratch(int32_t* at, int num_pages, int from_batch, int to_batch)
      : bad(at), copies(at + 1), first(at + 4), user(first + num_pages), gives(user + num_pages), takes(gives + from_batch),
        copy(takes + to_batch) {}
};

__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Exclusive sums of in[0 .. n) (written by other CTAs) into out, by the whole CTA; the total to every thread.
__device__ __forceinline__ int exclusive_sums(const int32_t* in, int n, int* out, int* warp_s) {
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int per = (n + kThreads - 1) / kThreads, i0 = min(n, t * per), i1 = min(n, i0 + per);
  int sum = 0;
  for (int i = i0; i < i1; ++i) sum += __ldcg(in + i);
  int incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += y;
  }
  if (lane == 31) warp_s[warp] = incl;
  __syncthreads();
  int before = 0, total = 0;
  for (int w = 0; w < kWarps; ++w) {
    const int x = warp_s[w];
    before += w < warp ? x : 0;
    total += x;
  }
  int at = before + incl - sum;
  for (int i = i0; i < i1; ++i) {
    out[i] = at;
    at += __ldcg(in + i);
  }
  __syncthreads();   // warp_s is read, out is there
  return total;
}

__global__ void __launch_bounds__(kThreads, 1) page_fork_plan_kernel(const __grid_constant__ PageForkParams p) {
  extern __shared__ int smem[];
  __shared__ int warp_s[kWarps];
  int* gives_s = smem;                  // [from_batch] exclusive sums
  int* takes_s = smem + p.from_batch;   // [to_batch]
  const Scratch sc(p.scratch, p.num_pages, p.from_batch, p.to_batch);
  const int t = threadIdx.x, lane = t & 31, cta = blockIdx.x;
  const int all = kCtas * kThreads, me = cta * kThreads + t;            // threads of the cluster
  const int warps = kCtas * kWarps, my_warp = cta * kWarps + (t >> 5);
  const int W = p.max_pages, log2p = p.page_log2, below = (1 << log2p) - 1;
  if (t == 0) grid_launch_dependents();
  grid_dependency_wait();

  // the sizes, checked by every CTA; nothing is known of any page
  const int f = *p.free_count;
  bool bad = f < 0 || f > p.num_pages;
  for (int b = t; b < p.from_batch; b += kThreads) bad = bad || p.held[b] < 0 || p.held[b] > W;
  for (int b = t; b < p.to_batch; b += kThreads) {
    const int from = p.parents[b], n = p.lens[b];
    bad = bad || from < -1 || from >= p.from_batch || (from >= 0 && (n < 0 || (n + (int64_t)below) >> log2p > p.held[from]));
  }
  for (int x = me; x < p.num_pages; x += all) sc.first[x] = sc.user[x] = kNone;
  if (me == 0) *sc.bad = 0;
  bad = __syncthreads_or(bad) != 0;   // the same in every CTA
  auto tokens_of = [&](int b) { return p.parents[b] < 0 ? 0 : p.lens[b]; };
  cluster_barrier();

  // every page's first holder and u
  if (!bad) {
    bool out = false;
    for (int b = my_warp; b < p.from_batch; b += warps) {
      const int n = p.held[b];
      for (int i = lane; i < n; i += 32) {
        const int x = p.table[(size_t)b * W + i];
        if (x >= 0 && x < p.num_pages) {
          if (__ldcg(sc.first + x) > b) atomicMin(sc.first + x, b);
        } else {
          out = true;
        }
      }
    }
    for (int b = my_warp; b < p.to_batch; b += warps) {
      const int n = tokens_of(b), full = n >> log2p;
      const int32_t* row = p.table + (size_t)max(p.parents[b], 0) * W;
      for (int i = lane; i < full; i += 32) {
        const int x = row[i];
        if (x >= 0 && x < p.num_pages && __ldcg(sc.user + x) != -1) atomicMin(sc.user + x, -1);
      }
      if (lane == 0 && (n & below) != 0) {
        const int x = row[full];
        if (x >= 0 && x < p.num_pages) atomicMin(sc.user + x, b);
      }
    }
    for (int i = me; i < f; i += all) {
      const int x = p.free_pages[i];
      out = out || x < 0 || x >= p.num_pages;
    }
    if (out) atomicOr(sc.bad, 1);
  }
  cluster_barrier();
  bad = bad || __ldcg(sc.bad) != 0;

  // what each row gives and takes
  if (!bad) {
    for (int b = my_warp; b < p.from_batch; b += warps) {
      const int n = p.held[b];
      int count = 0;
      for (int i = lane; i < n; i += 32) {
        const int x = p.table[(size_t)b * W + i];
        count += __ldcg(sc.first + x) == b && __ldcg(sc.user + x) == kNone ? 1 : 0;
      }
      count = __reduce_add_sync(0xffffffffu, count);
      if (lane == 0) sc.gives[b] = count;
    }
    for (int b = me; b < p.to_batch; b += all) {
      const int n = tokens_of(b);
      sc.takes[b] = (n & below) != 0 && __ldcg(sc.user + p.table[(size_t)p.parents[b] * W + (n >> log2p)]) != b ? 1 : 0;
    }
  }
  cluster_barrier();

  int G = 0, T = 0;
  if (!bad) {
    G = exclusive_sums(sc.gives, p.from_batch, gives_s, warp_s);
    T = exclusive_sums(sc.takes, p.to_batch, takes_s, warp_s);
  }
  bad = bad || (int64_t)f - T + G > p.num_pages;   // more pages than there are: some page is held and free
  const bool refused = bad || T > f;
  if (me == 0) {
    *p.new_free_count = refused ? 0 : f - T + G;
    *sc.copies = refused ? 0 : T;
    if (refused) atomicMax(p.dev_status, bad ? (int)PTD_ERR_INVALID_BATCH : (int)PTD_ERR_NO_PAGES);
  }
  if (refused) {
    for (int b = me; b < p.to_batch; b += all) p.new_held[b] = 0;
    return;
  }
  for (int b = my_warp; b < p.to_batch; b += warps) {
    const int n = tokens_of(b), full = n >> log2p;
    const int32_t* row = p.table + (size_t)max(p.parents[b], 0) * W;
    int32_t* to = p.new_table + (size_t)b * W;
    for (int i = lane; i < full; i += 32) to[i] = row[i];
    if (lane == 0) {
      p.new_held[b] = full + ((n & below) != 0 ? 1 : 0);
      if ((n & below) != 0) {
        int x = row[full];
        if (__ldcg(sc.takes + b) != 0) {
          const int rank = takes_s[b], fresh = p.free_pages[f - 1 - rank];
          sc.copy[3 * rank] = x;
          sc.copy[3 * rank + 1] = fresh;
          sc.copy[3 * rank + 2] = n & below;
          x = fresh;
        }
        to[full] = x;
      }
    }
  }
  for (int i = me; i < f - T; i += all) p.new_free_pages[i] = p.free_pages[i];
  for (int b = my_warp; b < p.from_batch; b += warps) {
    if (__ldcg(sc.gives + b) == 0) continue;
    const int n = p.held[b];
    int at = f - T + gives_s[b];
    for (int i0 = 0; i0 < n; i0 += 32) {
      const int x = i0 + lane < n ? p.table[(size_t)b * W + i0 + lane] : -1;
      const bool given = x >= 0 && __ldcg(sc.first + x) == b && __ldcg(sc.user + x) == kNone;
      const uint32_t mask = __ballot_sync(0xffffffffu, given);
      const int place = at + __popc(mask & ((1u << lane) - 1u));
      if (given && place < p.num_pages) p.new_free_pages[place] = x;
      at += __popc(mask);
    }
  }
}

// Item: (copy, layer, K or V, chunk of a page's bytes).
__global__ void __launch_bounds__(kCopyThreads) page_copy_kernel(const __grid_constant__ PageForkParams p, int chunks) {
  const Scratch sc(p.scratch, p.num_pages, p.from_batch, p.to_batch);
  if (threadIdx.x == 0) grid_launch_dependents();
  grid_dependency_wait();
  const int64_t per_copy = (int64_t)p.num_layers * 2 * chunks, items = (int64_t)*sc.copies * per_copy;
  const int64_t page_bytes = p.row_bytes << p.page_log2;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int c = (int)(item / per_copy);
    int rest = (int)(item - c * per_copy);
    const int chunk = rest % chunks;
    rest /= chunks;
    const int layer = rest >> 1;
    const int from = sc.copy[3 * c], to = sc.copy[3 * c + 1];
    const int64_t bytes = sc.copy[3 * c + 2] * p.row_bytes, at = (int64_t)chunk * kChunk;
    uint8_t* base = static_cast<uint8_t*>((rest & 1) != 0 ? p.v : p.k) + (int64_t)layer * p.num_pages * page_bytes + at;
    const uint4* src = reinterpret_cast<const uint4*>(base + from * page_bytes);
    uint4* dst = reinterpret_cast<uint4*>(base + to * page_bytes);
    const int64_t left = (bytes - at) / 16;
    uint4 x[kCopyLoads];
#pragma unroll
    for (int u = 0; u < kCopyLoads; ++u)
      if (threadIdx.x + u * kCopyThreads < left) x[u] = __ldcs(src + threadIdx.x + u * kCopyThreads);
#pragma unroll
    for (int u = 0; u < kCopyLoads; ++u)
      if (threadIdx.x + u * kCopyThreads < left) dst[threadIdx.x + u * kCopyThreads] = x[u];
  }
}

}  // namespace pf

size_t page_fork_scratch_ints(int num_pages, int from_batch, int to_batch) {
  return 4 + 2 * (size_t)num_pages + (size_t)from_batch + 4 * (size_t)to_batch;
}

cudaError_t launch_page_fork(const PageForkParams& p, int sms, cudaStream_t stream) {
  constexpr size_t kMostSmem = 2 * (size_t)PTD_MAX_PROMPT_BATCH * sizeof(int);
  const size_t smem = ((size_t)p.from_batch + p.to_batch) * sizeof(int);
  if (smem > 47 * 1024) {   // the limit is the kernel's, the same for every call
    const cudaError_t e =
        cudaFuncSetAttribute(pf::page_fork_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostSmem);
    if (e != cudaSuccess) return e;
  }
  const cudaError_t e =
      launch_chained(pf::page_fork_plan_kernel, dim3(pf::kCtas), dim3(pf::kThreads), smem, stream, pf::kCtas, p);
  if (e != cudaSuccess) return e;
  const int64_t page_bytes = p.row_bytes << p.page_log2;
  const int chunks = (int)((page_bytes + pf::kChunk - 1) / pf::kChunk);
  const int64_t most = (int64_t)p.to_batch * p.num_layers * 2 * chunks, places = 8 * (int64_t)sms;
  return launch_chained(pf::page_copy_kernel, dim3((unsigned)(most < places ? most : places)), dim3(pf::kCopyThreads), 0, stream, 0,
                        p, chunks);
}

}  // namespace ptd
