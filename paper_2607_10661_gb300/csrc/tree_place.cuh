// The tree, position and cache row of a node (internal; shared by the kernels that append a tree's rows).
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "ptd_device.cuh"

namespace ptd {
namespace tr {

constexpr int kThreads = 256;

// What every thread of a CTA works out for its node: the tree, the position and the cache row.
struct Place {
  int pos;      // C + |pi(i)| - 1
  size_t row;   // cache row of its slot, within a layer
  bool fits;
};

// Node n's place (block-wide: one barrier).  Every thread finds the tree, walks the ancestors and
// reads the block table itself: the reads are broadcasts, and no further barrier is needed.
// False (status set) when the tree is not one.
__device__ __forceinline__ bool find_place(const int32_t* node_offsets, const int32_t* parents, const int32_t* ctx_lens,
                                           int batch, int n, int page_size, int seq_capacity, int num_pages,
                                           const int32_t* block_table, int max_pages, bool first, int* par_s,
                                           int32_t* positions_out, int32_t* dev_status, Place& out) {
  const int t = threadIdx.x, lane = t & 31;
  int b = batch - 1;   // the first tree that ends after node n
  for (int b0 = 0; b0 < batch - 1; b0 += 32) {
    const int q = b0 + lane;
    const uint32_t hit = __ballot_sync(0xffffffffu, q < batch - 1 && node_offsets[q + 1] > n);
    if (hit != 0u) {
      b = b0 + __ffs(hit) - 1;
      break;
    }
  }
  const int node0 = node_offsets[b];
  const int T = node_offsets[b + 1] - node0;
  const int C = ctx_lens[b];
  const int i = n - node0;
  bool bad = T < 1 || T > kThreads || i < 0 || i >= T;
  if (!bad && t < T) {
    const int p = parents[node0 + t];
    par_s[t] = p;
    bad = t == 0 ? p != -1 : (p < 0 || p >= t);
  }
  if (__syncthreads_or(bad)) {
    if (t == 0) atomicMax(dev_status, (int)PTD_ERR_INVALID_TREE);
    return false;
  }
  const int slot = C + i;
  const int cap = page_size > 0 ? max_pages * page_size : seq_capacity;
  out.fits = C >= 0 && slot < cap;
  out.row = (size_t)b * seq_capacity + slot;
  if (out.fits && page_size > 0) {
    const int pg = block_table[(size_t)b * max_pages + slot / page_size];
    out.fits = pg >= 0 && pg < num_pages;
    out.row = (size_t)page_size * pg + slot % page_size;
  }
  int depth = 0;
  for (int a = i; a != -1; a = par_s[a]) ++depth;
  out.pos = C + depth - 1;
  if (t == 0 && first) {
    if (positions_out) positions_out[n] = out.pos;
    if (!out.fits) atomicMax(dev_status, (int)PTD_ERR_INVALID_TREE);
  }
  return true;
}

}  // namespace tr
}  // namespace ptd
