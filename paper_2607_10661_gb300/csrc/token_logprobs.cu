// Log probabilities of given tokens, entropies and the k best alternatives of rows of logits: one read of them
// all, and a second one of the few vectors that the alternatives may lie in.
//
// A row belongs to one CTA, or, where there are few long rows, is cut into contiguous parts, one CTA of a cluster each.
// Every thread keeps the sums of row_sums.cuh over its vectors, against the largest logit that it has seen: a batch of vectors
// in registers gives a maximum, then the exponentials, while the next batch is on its way.  The alternatives: with T the k-th
// largest of the maxima of 32 groups of lanes, k elements at least reach T, and few more; the vectors of the lanes whose maximum
// does are read again (L2) by all threads, what reaches T goes to a buffer, and an element's place is the number of larger
// ones in it.  A cluster's CTAs send their sums and keys to its first one, which writes the row.
//
// Where fewer than k groups hold a number above -inf (rows that a mask leaves few tokens, next to none in a part of a row) T is
// -inf and every masked element reaches it, and where long runs are equal to T: the buffer is lost and k rounds follow, a read of
// the part each.
//
// What bounds it: the one read, 1021 fp32 rows of 32000, k = 16 25.7 - 26.7 us in graph replays (4.9 - 5.1 TB/s; some 22
// with k = 0: a CTA's selection takes some 1.5 us that its own reads do not overlap), 512 bf16 rows of 128256 29.6 (4.4
// TB/s); for few rows the chain of reads, exponentials, selection and merge: one row of 128256, k = 8 6.0 us, 63 rows, k = 4
// 8.7.  At first (no batch in flight, the owners of candidates reading alone) 37.3, -, 7.2 and 11.1.  Where the rounds follow,
// they: with one to seven tokens of a row allowed, k = 8, one row 33 us, 63 rows 158 (fp32 36 and 190).
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "launch.cuh"
#include "ptd_device.cuh"
#include "row_sums.cuh"
#include "token_logprobs.cuh"
#include "topk_parts.cuh"

namespace cg = cooperative_groups;

namespace ptd {
namespace tl {

using namespace topk;

constexpr int kMaxParts = 8, kMaxK = 16;
constexpr int kCand = 256;         // candidate buffer (keys)
constexpr int kLoads = 4;          // vectors of a thread in flight
constexpr int kSmThreads = 1024;   // that an SM holds

template <typename T, int kThreads, bool kCluster>
__global__ void __launch_bounds__(kThreads, kSmThreads / kThreads)
    token_logprobs_kernel(const __grid_constant__ TokenLogprobsParams p) {
  constexpr int VN = Vec<T>::kN, kWarps = kThreads / 32, kGroup = kThreads / 32;   // lanes of one of the 32 groups
  __shared__ __align__(16) uint64_t cand_s[kCand];
  __shared__ __align__(16) uint64_t all_keys[kMaxParts * kMaxK];   // the parts' keys, in the cluster's first CTA
  __shared__ RowSums all_sums[kMaxParts];                          // and their sums
  __shared__ __align__(16) uint32_t group_max_s[32];
  __shared__ __align__(8) uint64_t parts_bar_s;
  __shared__ uint64_t round_s[kWarps];
  __shared__ RowSums warp_sums[kWarps];
  __shared__ uint16_t owners_s[kThreads];
  __shared__ int n_cand_s, n_owners_s, abort_s;

  cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)blockIdx.x, parts = (int)gridDim.x;   // the grid's x is one row's parts
  const int64_t r = (int64_t)blockIdx.z * gridDim.y + blockIdx.y;
  if (r >= p.rows) return;   // the whole cluster
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, k = p.k;
  const uint32_t parts_bar = smem_u32(&parts_bar_s);
  if (tid == 0) {
    if (kCluster) {
      mbar_init(parts_bar, (uint32_t)(parts * (k + 1)));   // an arrival per key and one per part's sums (the first CTA's is used)
      fence_mbar_init();
    }
    abort_s = 0;
    n_cand_s = 0;
    n_owners_s = 0;
  }
  if (kCluster && rank == 0 && tid < kMaxParts * kMaxK) all_keys[tid] = 0ull;
  __syncthreads();
  if (kCluster) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  grid_dependency_wait();   // the logits and the outputs belong to the stream's previous work

  // this CTA's part: the vector body starts at the row's first 16-byte boundary (head and tail
  // elements outside it go to the first and last CTA one by one)
  const T* row = static_cast<const T*>(p.logits) + r * p.row_stride;
  int a0 = (int)(((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / sizeof(T));
  if (a0 > p.vocab) a0 = p.vocab;
  const int nvec = (p.vocab - a0) / VN;
  const int a1 = a0 + nvec * VN;
  const int v_begin = min(nvec, rank * p.per), nv = min(nvec, v_begin + p.per) - v_begin;
  const uint4* vrow = reinterpret_cast<const uint4*>(row + a0) + v_begin;
  const bool own_head = rank == 0 && tid == 0, own_tail = rank == parts - 1 && tid == kThreads - 1;

  // the token's logit, asked for before the row (two dependent reads)
  float token_logit = 0.f;
  bool inside = false;
  if (own_head) {
    const int token = p.tokens[r];
    inside = token >= 0 && token < p.vocab;
    if (inside) token_logit = Vec<T>::scalar(row + token);
  }

  // 1. the sums; lane maxima, then of a group's lanes
  ThreadSums sums;
  float vmax = -INFINITY;   // of the vectors alone
  {
    constexpr uint32_t kNone = VN == 8 ? kBf16x2NegInf : 0xFF800000u;   // -inf
    const unsigned long long scale2 = f2_pack(p.scale, p.scale);
    uint4 next[kLoads];
    auto load = [&](int v0) {
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        const int v = v0 + u * kThreads;
        next[u] = v < nv ? __ldg(vrow + v) : make_uint4(kNone, kNone, kNone, kNone);
      }
    };
    load(tid);
#pragma unroll 1
    for (int v0 = tid; v0 < nv; v0 += kLoads * kThreads) {
      uint4 x[kLoads];
#pragma unroll
      for (int u = 0; u < kLoads; ++u) x[u] = next[u];
      load(v0 + kLoads * kThreads);   // the next batch is on its way while this one is added
      float m = vec_max<T>(x[0]);
#pragma unroll
      for (int u = 1; u < kLoads; ++u) m = fmaxf(m, vec_max<T>(x[u]));
      vmax = fmaxf(vmax, m);
      sums.raise(m, p.scale);
      float f[kLoads * VN];
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        float g[8];
        Vec<T>::unpack(x[u], g);
#pragma unroll
        for (int e = 0; e < VN; ++e) f[u * VN + e] = g[e];
      }
      sums.add(f, scale2);
    }
    auto add1 = [&](float f) {
      sums.raise(f, p.scale);
      const float pair[2] = {f, -INFINITY};
      sums.add(pair, scale2);
    };
    if (own_head)
      for (int i = 0; i < a0; ++i) add1(Vec<T>::scalar(row + i));
    if (own_tail)
      for (int i = a1; i < p.vocab; ++i) add1(Vec<T>::scalar(row + i));
  }
  {
    const bool has_elems = tid < nv || (own_head && a0 > 0) || (own_tail && a1 < p.vocab);
    uint32_t o = has_elems ? ordered_bits(sums.most) : 0u;
#pragma unroll
    for (int d = 1; d < kGroup; d <<= 1) o = max(o, __shfl_xor_sync(0xffffffffu, o, d));
    if ((lane & (kGroup - 1)) == 0) group_max_s[tid / kGroup] = o;
    const RowSums w = merge_lanes<32>(sums.sums(), p.scale);
    if (lane == 0) warp_sums[warp] = w;
  }
  __syncthreads();

  // 2. the threshold (0: fewer than k groups hold elements, so every element is a candidate)
  float thr = INFINITY;
  if (k > 0) {
    const uint32_t kth = k <= 8 ? kth_largest_ord(group_max_s[lane], k) : kth_of_32(group_max_s, k);
    thr = kth != 0u ? from_ordered(kth) : -INFINITY;
  }

  // 3. the candidates
  auto push = [&](float f, uint32_t idx) {
    const int at = atomicAdd(&n_cand_s, 1);
    if (at < kCand) cand_s[at] = make_key(ordered_bits(f), idx);
  };
  if (k > 0) {
    if (own_head)
      for (int i = 0; i < a0; ++i) {
        const float f = Vec<T>::scalar(row + i);
        if (f >= thr) push(f, (uint32_t)i);
      }
    if (own_tail)
      for (int i = a1; i < p.vocab; ++i) {
        const float f = Vec<T>::scalar(row + i);
        if (f >= thr) push(f, (uint32_t)i);
      }
    // the vectors of the lanes whose maximum reaches the threshold (about k), by all threads
    if (vmax >= thr && tid < nv) owners_s[atomicAdd(&n_owners_s, 1)] = (uint16_t)tid;
    __syncthreads();
    const int owners = n_owners_s, each = (nv + kThreads - 1) / kThreads, items = owners * each;
    for (int i0 = tid; i0 < items; i0 += kLoads * kThreads) {
      uint4 x[kLoads];
      int v[kLoads];
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        const int i = i0 + u * kThreads, round = i / owners;
        v[u] = i < items ? owners_s[i - round * owners] + round * kThreads : nv;
        x[u] = __ldg(vrow + min(v[u], nv - 1));
      }
      if (*(volatile int*)&n_cand_s > kCand) break;   // the buffer is already lost
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        if (v[u] < nv && vec_max<T>(x[u]) >= thr) {
          float f[8];
          Vec<T>::unpack(x[u], f);
          const uint32_t at = (uint32_t)(a0 + (v_begin + v[u]) * VN);
#pragma unroll
          for (int e = 0; e < VN; ++e)
            if (f[e] >= thr) push(f[e], at + e);
        }
      }
    }
  }
  // meanwhile every warp merges the warps' sums (none is written before the next barrier)
  const RowSums part = merge_lanes<kWarps>(warp_sums[lane & (kWarps - 1)], p.scale);
  __syncthreads();
  uint64_t* dst_keys = nullptr;
  uint32_t dst_bar = 0;
  auto arrive = [&](int count) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0], %1;" ::"r"(dst_bar), "r"(count) : "memory");
  };
  if constexpr (kCluster) {
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");   // the first CTA's keys and barrier are set up
    dst_keys = cluster.map_shared_rank(all_keys, 0) + rank * kMaxK;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(dst_bar) : "r"(parts_bar));
    if (tid == 0) {
      cluster.map_shared_rank(all_sums, 0)[rank] = part;
      arrive(1);
    }
  }
  // The next grid may be placed from here on: where its CTAs had waited from the start, 63 rows took 14.4 us a call, not 8.7.
  if (tid == 0) grid_launch_dependents();
  const RowResult whole(part);   // of a row in one part
  auto write_entry = [&](int at, uint64_t key, const RowResult& result) {   // alternative `at` of the row
    p.top_idx[r * k + at] = (int32_t)(~(uint32_t)(key & 0xFFFFFFFFull));
    const uint32_t ord = (uint32_t)(key >> 32);
    p.top_val[r * k + at] = result.logprob(ord != 0u ? from_ordered(ord) : __int_as_float(0x7fffffff), p.inv_temperature);   // 0: NaN
  };
  auto write_row = [&](const RowResult& result) {
    p.logprob[r] = inside ? result.logprob(token_logit, p.inv_temperature) : -INFINITY;
    if (p.entropy != nullptr) p.entropy[r] = result.entropy;
  };
  if (k > 0) {
    const int n = n_cand_s;
    const int n_elems = nv * VN + (rank == 0 ? a0 : 0) + (rank == parts - 1 ? p.vocab - a1 : 0);
    if (n <= kCand && n >= min(k, n_elems)) {
      for (int i = tid; i < n; i += kThreads) {
        const uint64_t key = cand_s[i];
        int before = 0;
        for (int j = 0; j < n; ++j) before += cand_s[j] > key ? 1 : 0;
        if (before < k) {
          if constexpr (kCluster) {
            dst_keys[before] = key;
            arrive(1);
          } else {
            write_entry(before, key, whole);
          }
        }
      }
      if (kCluster && n < k && tid == 0) arrive(k - n);   // fewer elements than k in this part
    } else {
      // k rounds over the part (long runs of equal values, or NaN; every thread takes part); 0 is below every number's order
      uint64_t last = ~0ull;
      for (int q = 0; q < k; ++q) {
        uint64_t best = 0ull;
        auto take = [&](float f, uint32_t idx) {
          const uint64_t key = make_key(f == f ? ordered_bits(f) : 0u, idx);
          if (key < last && key > best) best = key;
        };
        if (own_head)
          for (int i = 0; i < a0; ++i) take(Vec<T>::scalar(row + i), (uint32_t)i);
        if (own_tail)
          for (int i = a1; i < p.vocab; ++i) take(Vec<T>::scalar(row + i), (uint32_t)i);
        for (int v = tid; v < nv; v += kThreads) {
          float f[8];
          Vec<T>::unpack(__ldg(vrow + v), f);
#pragma unroll
          for (int e = 0; e < VN; ++e) take(f[e], (uint32_t)(a0 + (v_begin + v) * VN + e));
        }
        best = warp_max_u64(best);
        if (lane == 0) round_s[warp] = best;
        __syncthreads();
        best = round_s[0];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) best = best > round_s[w] ? best : round_s[w];
        if (tid == 0) {
          if constexpr (kCluster) {
            dst_keys[q] = best;
            arrive(1);
          } else {
            write_entry(q, best, whole);
          }
        }
        last = best;
        __syncthreads();   // round_s is read
      }
    }
  }
  if constexpr (!kCluster) {
    if (tid == 0) write_row(whole);
  } else if (rank == 0 && tid < kMaxParts * kMaxK) {   // four warps
    mbar_wait_cluster(parts_bar, 0u, &abort_s, p.dev_status);
    __syncwarp();
    const int at_part = lane & (kMaxParts - 1);
    const RowResult result(merge_lanes<kMaxParts>(at_part < parts ? all_sums[at_part] : RowSums{-INFINITY, 0.f, 0.f}, p.scale));
    if (tid == 0) write_row(result);
    const uint64_t key = all_keys[tid];
    if (key != 0ull) {
      int before = 0;
      for (int c = 0; c < parts; ++c)
        for (int j = 0; j < k; ++j) before += all_keys[c * kMaxK + j] > key ? 1 : 0;
      if (before < k) write_entry(before, key, result);
    }
  }
}

template <typename T, int kThreads, bool kCluster>
cudaError_t launch_as(TokenLogprobsParams p, int parts, cudaStream_t stream) {
  p.per = (p.vocab / Vec<T>::kN + parts - 1) / parts;   // (rows off 16 bytes have one vector fewer)
  const unsigned gy = (unsigned)(p.rows < 32768 ? p.rows : 32768), gz = (unsigned)((p.rows + gy - 1) / gy);
  return launch_chained(token_logprobs_kernel<T, kThreads, kCluster>, dim3((unsigned)parts, gy, gz), dim3(kThreads), 0, stream,
                        kCluster ? (unsigned)parts : 0u, p);
}

template <typename T>
cudaError_t launch(const TokenLogprobsParams& p, int sms, cudaStream_t stream) {
  // Long rows that are few: a cluster each, while every CTA has an SM.  Measured (us in 8, in 4 parts of 256 threads, in one of
  // 512; bf16 rows of 128256, k = 4): 1 row 5.8 / 6.2 / 8.6, 19 rows 6.6 / 6.4 / 8.8, 32 rows 7.5 / 7.2 / 8.8, 63 rows 9.0 /
  // 8.8 / 8.8; rows of 32000: 1 row 5.3 / 5.1 / 4.8, 19 rows 5.9 / 5.4 / 4.9.
  const int64_t vectors = (int64_t)p.vocab / Vec<T>::kN;
  for (int parts = kMaxParts; vectors >= 8192 && parts >= 4; parts /= 2)
    if (p.rows * parts <= sms) return launch_as<T, 256, true>(p, parts, stream);
  // One CTA per row: the most threads with which the rows are less than two waves of CTAs (four where a row is 384 KB or more and
  // its reads outweigh a CTA's fixed part), at most 512 and no more than its vectors, so that every group of lanes has some.  Measured (us with
  // 1024 / 512 / 256 / 128 threads): 100 bf16 rows of 32000, k = 4 5.9 / 6.0 / 5.6 / 5.9; 300 of 50257 15.2 / 10.1 / 11.1 / 11.4;
  // 512 of 128256, k = 8 40.2 / 30.2 / 30.4 / 50.0; 700 of 32000 25.7 / 15.4 / 11.9 / 15.2; 4096 of 32000 148 / 81.8 / 57.9 / 51.5;
  // fp32, 1021 rows of 32000, k = 16 48.5 / 34.1 / 27.3 / 31.4; 894 of 128256 86.6 / 77.1 / 90.7 / 99.9; 2000 of 1000
  // 54.7 / 26.1 / 14.6 / 8.4.  Clusters for more rows were slower: 1021 rows in two parts 36.9, in four 51.9.
  const int64_t threads = 1792 * (int64_t)sms / p.rows * (vectors >= 24000 ? 2 : 1);
  if (threads >= 512 && vectors >= 512) return launch_as<T, 512, false>(p, 1, stream);
  if (threads >= 256 && vectors >= 256) return launch_as<T, 256, false>(p, 1, stream);
  return launch_as<T, 128, false>(p, 1, stream);
}

}  // namespace tl

cudaError_t launch_token_logprobs(TokenLogprobsParams p, bool bf16, int sms, cudaStream_t stream) {
  return bf16 ? tl::launch<__nv_bfloat16>(p, sms, stream) : tl::launch<float>(p, sms, stream);
}

}  // namespace ptd
