// Geometry of packed batches of new tokens (internal; also compiled as plain C++): which sequences are
// valid, and how the attention's work units are numbered.
#pragma once

#include <cstdint>

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

// Pages for `len` positions.
PTD_HD int pages_for(int64_t len, int page_size) { return (int)((len + page_size - 1) / page_size); }

// A sequence's blocks of `width` tokens, as the attention orders them: block i of a sequence has the key
// first + i, first = ctx / width, which grows with the keys it sees.
struct PromptBlocks {
  int first, count;
};
PTD_HD PromptBlocks prompt_blocks(int ctx, int tokens, int width) { return {ctx / width, (tokens + width - 1) / width}; }

// Blocks of one sequence with key >= m.
PTD_HD int blocks_from(const PromptBlocks& s, int m) {
  const int c = s.first + s.count - m;
  return c < 0 ? 0 : (c > s.count ? s.count : c);
}

// Block number u of a batch in descending order of key (longest first, equal keys by sequence): its sequence
// and place in it.  With F(m) the number of blocks of key >= m, its key is the largest m with F(m) > u.
// `lanes` walks the sequences: one lane on the host, a warp's 32 on the device, where every lane gets the
// answer; seq(b) gives sequence b's blocks; max_key is above every key.  False: no such block.
template <typename Lanes, typename Seq>
PTD_HD bool find_prompt_block(const Lanes& lanes, const Seq& seq, int batch, int max_key, int u, int* b_out, int* i_out) {
  if (batch == 1) {
    const PromptBlocks s = seq(0);
    *b_out = 0;
    *i_out = s.count - 1 - u;
    return u >= 0 && u < s.count;
  }
  auto from = [&](int m) {
    int c = 0;
    for (int b = lanes.id(); b < batch; b += lanes.count()) c += blocks_from(seq(b), m);
    return lanes.sum(c);
  };
  if (u < 0 || from(0) <= u) return false;
  int lo = 0, hi = max_key;   // F(lo) > u >= F(hi)
  while (hi - lo > 1) {
    const int mid = lo + (hi - lo) / 2;
    if (from(mid) > u) lo = mid; else hi = mid;
  }
  int left = u - from(lo + 1);   // its place among the sequences that have a block of key lo
  for (int b0 = 0; b0 < batch; b0 += lanes.count()) {
    const int b = b0 + lanes.id();
    bool has = false;
    if (b < batch) {
      const PromptBlocks s = seq(b);
      has = s.first <= lo && lo < s.first + s.count;
    }
    const uint32_t hit = lanes.ballot(has);
    const int n = lanes.popcount(hit);
    if (left < n) {
      const int q = b0 + lanes.nth(hit, left);
      *b_out = q;
      *i_out = lo - seq(q).first;
      return true;
    }
    left -= n;
  }
  return false;
}

struct OneLane {
  PTD_HD int id() const { return 0; }
  PTD_HD int count() const { return 1; }
  PTD_HD int sum(int x) const { return x; }
  PTD_HD uint32_t ballot(bool p) const { return p ? 1u : 0u; }
  PTD_HD int popcount(uint32_t x) const { return (int)x; }
  PTD_HD int nth(uint32_t, int) const { return 0; }
};

#ifdef __CUDACC__
struct WarpLanes {
  __device__ __forceinline__ int id() const { return threadIdx.x & 31; }
  __device__ __forceinline__ int count() const { return 32; }
  __device__ __forceinline__ int sum(int x) const { return (int)__reduce_add_sync(0xffffffffu, (unsigned)x); }
  __device__ __forceinline__ uint32_t ballot(bool p) const { return __ballot_sync(0xffffffffu, p); }
  __device__ __forceinline__ int popcount(uint32_t x) const { return __popc(x); }
  __device__ __forceinline__ int nth(uint32_t x, int k) const { return __fns(x, 0, k + 1); }
};
#endif

}  // namespace ptd
