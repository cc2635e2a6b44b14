// Causal attention of packed new tokens over an fp32 cache, on the CUDA cores.
//
// Rows r = token * sub + head of one block of tokens under `sub` query heads of one KV head (64 rows, or 16 for
// batches of few) meet the block's keys in tiles of 64: S = Q K^T, softmax with a running maximum
// and sum in fp32, O += P V.  256 threads as 16 x 16: thread (y, x) takes the rows y + 16 a, of S the keys x + 16 c, of
// O D / 16 columns.  Q, K, V and P are in shared memory, O and the statistics in registers; the products are
// packed in pairs (of S over two columns of the head, of O over two outputs), fp32 throughout.  K of the next
// tile is copied beside the softmax and P V, V beside the next S.  Key tiles that some row does not see in full
// and that hold an infinity or a NaN of V take a path that leaves hidden products out, so that these never meet a
// weight of 0.
//
// Bound by shared-memory reads and the FMA pipe for many rows (2048 tokens of 32/8 heads, D = 64, 37 TFLOP/s), by
// latency for few.
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>

#include "launch.cuh"
#include "prompt_attention.cuh"
#include "ptd_device.cuh"

namespace ptd {
namespace pa {

constexpr int kThreads = 256;
constexpr int kKeys = 64;
constexpr int kPitchP = kKeys + 16;   // the two rows that a warp writes meet different banks

template <int D, int RT>
struct Simt {
  static constexpr int kRows = 16 * RT;
  static constexpr int kPitch = D + 4;   // of Q and K rows: 16-byte reads of eight rows meet every bank once
  static constexpr size_t kSmem = (size_t)((kRows + kKeys) * kPitch + kKeys * D + kRows * kPitchP) * sizeof(float);
};

// 16 bytes from global to shared memory, or zeros.
__device__ __forceinline__ void copy16(float* dst, const float* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_issued() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// All but the newest group have landed (this thread's).
__device__ __forceinline__ void copies_but_one() { asm volatile("cp.async.wait_group 1;" ::: "memory"); }

template <int D, int RT>
__global__ void __launch_bounds__(kThreads) prompt_simt_kernel(const PromptAttnParams p) {
  using L = Simt<D, RT>;
  extern __shared__ __align__(16) float smem_f[];
  constexpr int kPitch = L::kPitch, kRows = L::kRows, kChunks = kKeys * (D / 4) / kThreads;
  constexpr int VC = D / 16 < 4 ? D / 16 : 4, NB = D / (16 * VC);   // O columns: nb * 16 VC + x VC + i
  float* Qs = smem_f;
  float* Ks = Qs + kRows * kPitch;
  float* Vs = Ks + kKeys * kPitch;
  float* Ps = Vs + kKeys * D;
  __shared__ Unit unit_s;
  __shared__ int found_s;
  __shared__ int64_t key_row[2][kKeys];   // cache rows of a tile's keys, -1: none
  const int t = threadIdx.x, x = t & 15, y = t >> 4;
  grid_dependency_wait();
  if (t == 0) grid_launch_dependents();   // (after the wait: the merge reads the batch's arrays before its own)
  if (t < 32) {
    Units units(p);
    if (units.bad) atomicMax(p.dev_status, (int)PTD_ERR_INVALID_BATCH);
    Unit u;
    const bool found = units.find(p, blockIdx.x, u);
    if (t == 0) {
      if (found) unit_s = u;
      found_s = found;
    }
  }
  __syncthreads();
  if (!found_s) return;
  const Unit u = unit_s;
  const int rows = u.tokens * p.sub, end = u.ctx + u.token0 + u.tokens;
  auto find_rows = [&](int kt) {   // the cache rows of tile kt's keys
    const int key = kt * kKeys + t;
    if (t >= kKeys) return;
    int64_t row = -1;
    if (key < end) {
      if (p.page_size > 0) {
        const int page = p.block_table[(size_t)u.b * p.max_pages + (key >> p.page_log2)];
        if (page >= 0 && page < p.num_pages)
          row = ((int64_t)p.layer * p.num_pages + page) * p.page_size + (key & (p.page_size - 1));
        else
          atomicMax(p.dev_status, (int)PTD_ERR_INVALID_BATCH);
      } else {
        row = ((int64_t)p.layer * p.batch + u.b) * p.seq_capacity + key;
      }
    }
    key_row[kt & 1][t] = row;
  };
  auto copy_tile = [&](float* dst, int pitch, const void* from, int kt) {   // 16-byte chunks of tile kt's rows
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      const int e = t + i * kThreads, j = e / (D / 4), c = (e - j * (D / 4)) * 4;
      const int64_t row = kt < u.tile1 ? key_row[kt & 1][j] : -1;
      copy16(dst + j * pitch + c, static_cast<const float*>(from) + ((row < 0 ? 0 : row) * p.hkv + u.kv) * D + c, row >= 0);
    }
    copies_issued();
  };
  find_rows(u.tile0);
  __syncthreads();
  copy_tile(Ks, kPitch, p.k, u.tile0);
  copy_tile(Vs, D, p.v, u.tile0);
  for (int e = t; e < kRows * (D / 4); e += kThreads) {
    const int r = e / (D / 4), c = (e - r * (D / 4)) * 4, token = divide(r, p.by_sub);
    float4 q = make_float4(0.f, 0.f, 0.f, 0.f);
    if (r < rows)
      q = *reinterpret_cast<const float4*>(static_cast<const float*>(p.q) + (size_t)(u.row0 + token) * p.q_stride +
                                           (size_t)(u.head0 + r - token * p.sub) * D + c);
    *reinterpret_cast<float4*>(Qs + r * kPitch + c) = q;
  }
  int last[RT];   // the last key that each of this thread's rows sees
#pragma unroll
  for (int a = 0; a < RT; ++a) last[a] = u.ctx + u.token0 + divide(min(y + 16 * a, rows - 1), p.by_sub);
  float m[RT], l[RT];
  unsigned long long o[RT][NB][VC / 2];
#pragma unroll
  for (int a = 0; a < RT; ++a) {
    m[a] = -INFINITY;
    l[a] = 0.f;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < VC / 2; ++i) o[a][b][i] = f2_pack(0.f, 0.f);
  }
  for (int kt = u.tile0; kt < u.tile1; ++kt) {
    const int key0 = kt * kKeys;
    if (kt + 1 < u.tile1) find_rows(kt + 1);
    copies_but_one();
    __syncthreads();   // K of this tile (and, the first time, Q) is there
    float s[RT][4];
    {
      unsigned long long s2[RT][4];
#pragma unroll
      for (int a = 0; a < RT; ++a)
#pragma unroll
        for (int c = 0; c < 4; ++c) s2[a][c] = f2_pack(0.f, 0.f);
#pragma unroll 4
      for (int d = 0; d < D; d += 4) {
        ulonglong2 q[RT], k[4];
#pragma unroll
        for (int a = 0; a < RT; ++a) q[a] = *reinterpret_cast<const ulonglong2*>(Qs + (y + 16 * a) * kPitch + d);
#pragma unroll
        for (int c = 0; c < 4; ++c) k[c] = *reinterpret_cast<const ulonglong2*>(Ks + (x + 16 * c) * kPitch + d);
#pragma unroll
        for (int a = 0; a < RT; ++a)
#pragma unroll
          for (int c = 0; c < 4; ++c) s2[a][c] = f2_fma(q[a].y, k[c].y, f2_fma(q[a].x, k[c].x, s2[a][c]));
      }
#pragma unroll
      for (int a = 0; a < RT; ++a)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          float lo, hi;
          f2_unpack(s2[a][c], lo, hi);
          s[a][c] = lo + hi;
        }
    }
    __syncthreads();   // K has been read, the next tile's rows are known
    copy_tile(Ks, kPitch, p.k, kt + 1);
    const bool edge = key0 + kKeys - 1 > u.ctx + u.token0;   // some row does not see the whole tile
#pragma unroll
    for (int a = 0; a < RT; ++a) {
      float mx = -INFINITY;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        s[a][c] = edge && key0 + x + 16 * c > last[a] ? -INFINITY : s[a][c] * p.scale_log2;
        mx = fmaxf(mx, s[a][c]);
      }
#pragma unroll
      for (int w = 1; w < 16; w <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
      const float m_new = fmaxf(m[a], mx), ref = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = exp2f(m[a] - ref);
      m[a] = m_new;
      float sum = 0.f;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const float w = exp2f(s[a][c] - ref);
        sum += w;
        Ps[(y + 16 * a) * kPitchP + x + 16 * c] = w;
      }
      l[a] = l[a] * alpha + sum;
      const unsigned long long alpha2 = f2_pack(alpha, alpha);
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < VC / 2; ++i) o[a][b][i] = f2_mul(o[a][b][i], alpha2);
    }
    copies_but_one();
    // V of this tile is there (a row's weights are its own warp's).  Hidden products are left out one by one only
    // where the tile holds an infinity or a NaN: 0 times any other value adds nothing.
    float odd = 0.f;
    if (edge) {
#pragma unroll
      for (int i = 0; i < kChunks; ++i) {   // the chunks that this thread has copied
        const float4 v = *reinterpret_cast<const float4*>(Vs + (t + i * kThreads) * 4);
        odd += v.x * 0.f + v.y * 0.f + v.z * 0.f + v.w * 0.f;
      }
    }
    const bool one_by_one = __syncthreads_or(odd != 0.f) != 0;   // (NaN differs from 0)
    auto value = [&](int j, unsigned long long (&v)[NB][VC / 2]) {
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const float* at = Vs + j * D + b * 16 * VC + x * VC;
        if constexpr (VC == 4) {
          const ulonglong2 w = *reinterpret_cast<const ulonglong2*>(at);
          v[b][0] = w.x, v[b][1] = w.y;
        } else {
          v[b][0] = *reinterpret_cast<const unsigned long long*>(at);
        }
      }
    };
    if (!one_by_one) {
#pragma unroll 1
      for (int j = 0; j < kKeys; j += 4) {
        float4 w[RT];
#pragma unroll
        for (int a = 0; a < RT; ++a) w[a] = *reinterpret_cast<const float4*>(Ps + (y + 16 * a) * kPitchP + j);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          unsigned long long v[NB][VC / 2];
          value(j + q, v);
#pragma unroll
          for (int a = 0; a < RT; ++a) {
            const float wq = q == 0 ? w[a].x : q == 1 ? w[a].y : q == 2 ? w[a].z : w[a].w;
            const unsigned long long w2 = f2_pack(wq, wq);
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
              for (int i = 0; i < VC / 2; ++i) o[a][b][i] = f2_fma(w2, v[b][i], o[a][b][i]);
          }
        }
      }
    } else {
#pragma unroll 1
      for (int j = 0; j < kKeys && key0 + j < end; ++j) {
        unsigned long long v[NB][VC / 2];
        value(j, v);
#pragma unroll
        for (int a = 0; a < RT; ++a) {
          const float wq = Ps[(y + 16 * a) * kPitchP + j];
          const unsigned long long w2 = f2_pack(wq, wq);
          const bool seen = key0 + j <= last[a];
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < VC / 2; ++i) o[a][b][i] = seen ? f2_fma(w2, v[b][i], o[a][b][i]) : o[a][b][i];
        }
      }
    }
    __syncthreads();   // V has been read
    copy_tile(Vs, D, p.v, kt + 1);
  }
#pragma unroll
  for (int a = 0; a < RT; ++a) {
    const int r = y + 16 * a, token = divide(r, p.by_sub);
#pragma unroll
    for (int w = 1; w < 16; w <<= 1) l[a] += __shfl_xor_sync(0xffffffffu, l[a], w);
    if (r >= rows) continue;
    const float inv = u.whole ? 1.f / l[a] : 1.f;   // a piece stays unnormalised
    if (!u.whole && x == 0) reinterpret_cast<float2*>(p.part_ml)[(size_t)u.place * kRows + r] = make_float2(m[a], l[a]);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int d = b * 16 * VC + x * VC;
      float* dst = u.whole ? static_cast<float*>(p.out) + ((size_t)(u.row0 + token) * p.hq + u.head0 + r - token * p.sub) * D + d
                           : p.part_o + (((size_t)u.place * (D / 4) + d / 4) * kRows + r) * 4 + d % 4;
#pragma unroll
      for (int i = 0; i < VC / 2; ++i) {
        float lo, hi;
        f2_unpack(o[a][b][i], lo, hi);
        *reinterpret_cast<float2*>(dst + 2 * i) = make_float2(lo * inv, hi * inv);
      }
    }
  }
}

}  // namespace pa

cudaError_t launch_prompt_attn_simt(const PromptAttnParams& p, cudaStream_t stream) {
  const dim3 grid((unsigned)(p.blocks * p.tile_heads * p.splits));
#define PTD_SIMT_LAUNCH(D, RT)                                                                                         \
  do {                                                                                                                 \
    const auto kernel = pa::prompt_simt_kernel<D, RT>;                                                                 \
    const cudaError_t e =                                                                                              \
        cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)pa::Simt<D, RT>::kSmem);        \
    if (e != cudaSuccess) return e;                                                                                    \
    return launch_chained(kernel, grid, dim3(pa::kThreads), pa::Simt<D, RT>::kSmem, stream, 0, p);                     \
  } while (0)
  if (p.tile_rows == 64) {
    if (p.head_dim == 32) PTD_SIMT_LAUNCH(32, 4);
    if (p.head_dim == 64) PTD_SIMT_LAUNCH(64, 4);
    PTD_SIMT_LAUNCH(128, 4);
  }
  if (p.head_dim == 32) PTD_SIMT_LAUNCH(32, 1);
  if (p.head_dim == 64) PTD_SIMT_LAUNCH(64, 1);
  PTD_SIMT_LAUNCH(128, 1);
#undef PTD_SIMT_LAUNCH
}

}  // namespace ptd
