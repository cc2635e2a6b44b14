// Causal attention of packed new tokens over an fp32 cache, on the CUDA cores.
//
// Rows r = token * sub + head of one block of tokens under `sub` query heads of one KV head (64 rows) meet
// the block's keys in tiles of 64: S = Q K^T, softmax with a running maximum and sum in fp32, O += P V.
// 256 threads as 16 x 16: thread (y, x) takes rows 4 y .. 4 y + 3, of S the keys x + 16 c, of O D / 16 columns.
// Q, K, V and P are in shared memory, O and the statistics in registers.  Key tiles that some row does not
// see in full take a path that leaves hidden products out, so that what lies in hidden slots (not even an
// infinity or a NaN of V) never meets a weight of 0.
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>

#include "launch.cuh"
#include "prompt_attention.cuh"
#include "ptd_device.cuh"

namespace ptd {
namespace pa {

constexpr int kThreads = 256;
constexpr int kRows = 64;
constexpr int kKeys = 64;
constexpr int kPitchP = kKeys + 4;

template <int D>
struct Simt {
  static constexpr int kPitch = D + 4;   // of Q and K rows: 16-byte reads of eight rows meet every bank once
  static constexpr size_t kSmem = (size_t)((kRows + kKeys) * kPitch + kKeys * D + kRows * kPitchP) * sizeof(float);
};

template <int D>
__global__ void __launch_bounds__(kThreads) prompt_simt_kernel(const PromptAttnParams p) {
  extern __shared__ __align__(16) float smem_f[];
  constexpr int kPitch = Simt<D>::kPitch;
  constexpr int VC = D / 16 < 4 ? D / 16 : 4, NB = D / (16 * VC);   // O columns: nb * 16 VC + x VC + i
  float* Qs = smem_f;
  float* Ks = Qs + kRows * kPitch;
  float* Vs = Ks + kKeys * kPitch;
  float* Ps = Vs + kKeys * D;
  __shared__ Unit unit_s;
  __shared__ int found_s;
  const int t = threadIdx.x, x = t & 15, y = t >> 4;
  if (t == 0) grid_launch_dependents();
  grid_dependency_wait();
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
  // 16-byte chunks of a row: Q
  for (int e = t; e < kRows * (D / 4); e += kThreads) {
    const int r = e / (D / 4), c = (e - r * (D / 4)) * 4;
    float4 q = make_float4(0.f, 0.f, 0.f, 0.f);
    if (r < rows)
      q = *reinterpret_cast<const float4*>(static_cast<const float*>(p.q) + (size_t)(u.row0 + r / p.sub) * p.q_stride +
                                           (size_t)(u.head0 + r % p.sub) * D + c);
    *reinterpret_cast<float4*>(Qs + r * kPitch + c) = q;
  }
  int last[4];   // the last key that each of this thread's rows sees
#pragma unroll
  for (int a = 0; a < 4; ++a) last[a] = u.ctx + u.token0 + min(y * 4 + a, rows - 1) / p.sub;
  float m[4], l[4], o[4][NB][VC];
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    m[a] = -INFINITY;
    l[a] = 0.f;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < VC; ++i) o[a][b][i] = 0.f;
  }
  for (int kt = u.tile0; kt < u.tile1; ++kt) {
    const int key0 = kt * kKeys;
    __syncthreads();   // the tile before has been read
    for (int e = t; e < kKeys * (D / 4); e += kThreads) {
      const int j = e / (D / 4), c = (e - j * (D / 4)) * 4, key = key0 + j;
      float4 k = make_float4(0.f, 0.f, 0.f, 0.f), v = k;
      if (key < end) {
        size_t row;
        bool there = true;
        if (p.page_size > 0) {
          const int page = p.block_table[(size_t)u.b * p.max_pages + key / p.page_size];
          there = page >= 0 && page < p.num_pages;
          row = ((size_t)p.layer * p.num_pages + page) * p.page_size + key % p.page_size;
        } else {
          row = ((size_t)p.layer * p.batch + u.b) * p.seq_capacity + key;
        }
        if (there) {
          const size_t at = (row * p.hkv + u.kv) * D + c;
          k = *reinterpret_cast<const float4*>(static_cast<const float*>(p.k) + at);
          v = *reinterpret_cast<const float4*>(static_cast<const float*>(p.v) + at);
        } else {
          atomicMax(p.dev_status, (int)PTD_ERR_INVALID_BATCH);
        }
      }
      *reinterpret_cast<float4*>(Ks + j * kPitch + c) = k;
      *reinterpret_cast<float4*>(Vs + j * D + c) = v;
    }
    __syncthreads();
    float s[4][4];
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
      for (int c = 0; c < 4; ++c) s[a][c] = 0.f;
#pragma unroll 4
    for (int d = 0; d < D; d += 4) {
      float4 q[4], k[4];
#pragma unroll
      for (int a = 0; a < 4; ++a) q[a] = *reinterpret_cast<const float4*>(Qs + (y * 4 + a) * kPitch + d);
#pragma unroll
      for (int c = 0; c < 4; ++c) k[c] = *reinterpret_cast<const float4*>(Ks + (x + 16 * c) * kPitch + d);
#pragma unroll
      for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          s[a][c] = fmaf(q[a].x, k[c].x, s[a][c]);
          s[a][c] = fmaf(q[a].y, k[c].y, s[a][c]);
          s[a][c] = fmaf(q[a].z, k[c].z, s[a][c]);
          s[a][c] = fmaf(q[a].w, k[c].w, s[a][c]);
        }
    }
    const bool edge = key0 + kKeys - 1 > u.ctx + u.token0;   // some row does not see the whole tile
#pragma unroll
    for (int a = 0; a < 4; ++a) {
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
        Ps[(y * 4 + a) * kPitchP + x + 16 * c] = w;
      }
      l[a] = l[a] * alpha + sum;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < VC; ++i) o[a][b][i] *= alpha;
    }
    __syncwarp();   // a row's 16 threads are in one warp
    if (!edge) {
#pragma unroll 4
      for (int j = 0; j < kKeys; ++j) {
        float w[4];
#pragma unroll
        for (int a = 0; a < 4; ++a) w[a] = Ps[(y * 4 + a) * kPitchP + j];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int i = 0; i < VC; ++i) {
            const float v = Vs[j * D + b * 16 * VC + x * VC + i];
#pragma unroll
            for (int a = 0; a < 4; ++a) o[a][b][i] = fmaf(w[a], v, o[a][b][i]);
          }
      }
    } else {
      for (int j = 0; j < kKeys && key0 + j < end; ++j) {
        float w[4];
#pragma unroll
        for (int a = 0; a < 4; ++a) w[a] = Ps[(y * 4 + a) * kPitchP + j];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int i = 0; i < VC; ++i) {
            const float v = Vs[j * D + b * 16 * VC + x * VC + i];
#pragma unroll
            for (int a = 0; a < 4; ++a) o[a][b][i] = key0 + j <= last[a] ? fmaf(w[a], v, o[a][b][i]) : o[a][b][i];
          }
      }
    }
  }
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    const int r = y * 4 + a;
#pragma unroll
    for (int w = 1; w < 16; w <<= 1) l[a] += __shfl_xor_sync(0xffffffffu, l[a], w);
    if (r >= rows) continue;
    if (!u.whole) {
      const size_t piece = u.place;
      if (x == 0) reinterpret_cast<float2*>(p.part_ml)[piece * kRows + r] = make_float2(m[a], l[a]);
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < VC; ++i) {
          const int d = b * 16 * VC + x * VC + i;
          p.part_o[((piece * (D / 4) + d / 4) * kRows + r) * 4 + d % 4] = o[a][b][i];
        }
    } else {
      const float inv = 1.f / l[a];
      float* dst = static_cast<float*>(p.out) + ((size_t)(u.row0 + r / p.sub) * p.hq + u.head0 + r % p.sub) * D;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < VC; ++i) dst[b * 16 * VC + x * VC + i] = o[a][b][i] * inv;
    }
  }
}

}  // namespace pa

cudaError_t launch_prompt_attn_simt(const PromptAttnParams& p, cudaStream_t stream) {
  const dim3 grid((unsigned)(p.blocks * p.tile_heads * p.splits));
#define PTD_SIMT_LAUNCH(D)                                                                                          \
  do {                                                                                                                 \
    const auto kernel = pa::prompt_simt_kernel<D>;                                                                  \
    const cudaError_t e =                                                                                              \
        cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)pa::Simt<D>::kSmem);         \
    if (e != cudaSuccess) return e;                                                                                    \
    return launch_chained(kernel, grid, dim3(pa::kThreads), pa::Simt<D>::kSmem, stream, 0, p);                      \
  } while (0)
  if (p.head_dim == 32) PTD_SIMT_LAUNCH(32);
  if (p.head_dim == 64) PTD_SIMT_LAUNCH(64);
  PTD_SIMT_LAUNCH(128);
#undef PTD_SIMT_LAUNCH
}

}  // namespace ptd
