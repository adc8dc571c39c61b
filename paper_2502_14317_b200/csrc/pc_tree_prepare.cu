// The rotated queries of pc_tree_attn as rows in memory, for kernels whose CTAs do not make them, and who sees whom.
#include "pc_kernels.h"
#include "pc_tree_rows.cuh"

namespace pc {

// Blocks of a token and 32 of its heads, a warp for every eighth.  What a token has for all heads is computed once: whom it sees by the first warp, a pair's
// angle by a thread.  (By every warp for itself: 640 tokens of 32 heads 14 us.)
template <int D>
__global__ void __launch_bounds__(256) tree_rows_kernel(const __grid_constant__ CacheRows p, const __grid_constant__ TreePhase t) {
  constexpr int E = D / 32;
  __shared__ float2 angle[D / 2];
  __shared__ long long pos;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, G = p.Hq / p.Hkv;
  const int seq = blockIdx.x / p.w, i = blockIdx.x - seq * p.w;
  const double part = threadIdx.x < D / 2 ? part_of_turn(t.turns, threadIdx.x) : 0.0;
  chain();
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) {
    if (p.clear != nullptr) p.clear[0] = p.clear[1] = 0;
    if (p.clear_too != nullptr) *p.clear_too = 0;
  }
  uint32_t x[4][E / 2];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int h = blockIdx.y * 32 + u * 8 + warp;
    if (h >= p.Hq) break;
    const uint16_t* const at = static_cast<const uint16_t*>(p.q) + seq * p.stride[0] + i * p.stride[1] + h * p.stride[2];
    if constexpr (E == 4) {
      const uint2 y = __ldg(reinterpret_cast<const uint2*>(at) + lane);
      x[u][0] = y.x; x[u][1] = y.y;
    } else {
      x[u][0] = __ldg(reinterpret_cast<const uint32_t*>(at) + lane);
    }
  }
  if (warp == 0) {
    const int entries = __ldg(t.lens + seq);
    const unsigned long long sees = tree_seen(t.parents == nullptr ? nullptr : t.parents + seq * t.parent_stride, p.w, lane).of(i);
    if (lane == 0) {
      if (blockIdx.y == 0) t.sees[blockIdx.x] = sees;
      pos = (long long)p.pos0 + (p.pos ? __ldg(p.pos + seq) : entries) + (sees ? __popcll(sees) - 1 : 0);
    }
  }
  if (t.turn) {
    __syncthreads();
    if (threadIdx.x < D / 2) angle[threadIdx.x] = turned(part, pos);
    __syncthreads();
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int h = blockIdx.y * 32 + u * 8 + warp;
    if (h >= p.Hq) break;
    if (t.turn) {
      float c[E], s[E];
#pragma unroll
      for (int e = 0; e < E; ++e) { const float2 a = angle[E * (lane & 15) + e]; c[e] = a.x; s[e] = a.y; }
      turn_row<D>(x[u], c, s, lane);
    }
    const int hkv = h / G;
    const size_t at = (size_t)hkv * p.B * p.w * G + (size_t)blockIdx.x * G + h % G;
    TreeTurner<D>::store(p.rows, at, lane, x[u]);
    leave_beside<D>(p, at, lane, x[u]);
  }
}

cudaError_t launch_tree_rows(const CacheRows& p, const TreePhase& t, int d, cudaStream_t st) {
  const dim3 grid((unsigned)(p.B * p.w), (unsigned)((p.Hq + 31) / 32));
  return d == 128 ? launch_chained(tree_rows_kernel<128>, grid, dim3(256), 0, st, 1, p, t) : launch_chained(tree_rows_kernel<64>, grid, dim3(256), 0, st, 1, p, t);
}

}  // namespace pc
