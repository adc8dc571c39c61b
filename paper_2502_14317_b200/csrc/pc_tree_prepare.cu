// What stands before and behind the attention kernels of pc_tree_attn: the rotated queries as rows in memory, for kernels whose CTAs do not make them, with
// who sees whom; and the join of a row's partial results.
#include "pc_kernels.h"
#include "pc_cache_finish.cuh"
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
  // as chain(), but what is cleared is so before the next kernel starts: that looks at lengths and pages before it waits for this one, and may have a code to leave
  cudaGridDependencySynchronize();
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) {
    if (p.clear != nullptr) p.clear[0] = p.clear[1] = 0;
    if (p.clear_too != nullptr) *p.clear_too = 0;
    __threadfence();
  }
  __syncthreads();
  cudaTriggerProgrammaticLaunchCompletion();
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

// Results of a row's pieces joined, a warp for ROWS rows, whose statistics and then results are on their way together: of 20480 rows of 3 slots both are two waits.
template <int D, int ROWS>
__global__ void __launch_bounds__(128) tree_merge_kernel(const CacheMerge p) {
  constexpr int E = D / 32;
  const int lane = threadIdx.x & 31, G = p.q.Hq / p.q.Hkv;
  chain();
  const long long first = ((long long)blockIdx.x * 4 + (threadIdx.x >> 5)) * ROWS, all = (long long)p.q.Hkv * p.total_rows;
  if (first >= all) return;
  float2 ml[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r)
    ml[r] = first + r < all && lane < p.n_slots ? p.part_ml[(first + r) * p.n_slots + lane] : make_float2(-INFINITY, 0.0f);
  RowSum<D> x[ROWS];
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const long long row = first + r;
    const float* const po = p.part_o + row * p.n_slots * D + lane * E;
    x[r].join(ml[r], p.n_slots < 32 ? p.n_slots : 32, [&](int s, float (&y)[E]) {
      if constexpr (E == 4) { const float4 z = *reinterpret_cast<const float4*>(po + s * D); y[0] = z.x; y[1] = z.y; y[2] = z.z; y[3] = z.w; }
      else { const float2 z = *reinterpret_cast<const float2*>(po + s * D); y[0] = z.x; y[1] = z.y; }
    });
    if (p.n_slots > 32 && row < all) x[r].join_slots(p.part_ml + row * p.n_slots, p.part_o + row * p.n_slots * D, p.n_slots, 32, 1, lane);
  }
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    const long long row = first + r;
    if (row >= all) break;
    const int hkv = (int)(row / p.total_rows), in = (int)(row % p.total_rows);
    x[r].store(p, hkv * G + in % G, in / G, lane);
  }
}

cudaError_t launch_tree_rows(const CacheRows& p, const TreePhase& t, int d, cudaStream_t st) {
  const dim3 grid((unsigned)(p.B * p.w), (unsigned)((p.Hq + 31) / 32));
  return d == 128 ? launch_chained(tree_rows_kernel<128>, grid, dim3(256), 0, st, 1, p, t) : launch_chained(tree_rows_kernel<64>, grid, dim3(256), 0, st, 1, p, t);
}

namespace {
template <int D>
cudaError_t merge_t(const CacheMerge& p, int sm_count, cudaStream_t st) {
  const long long rows = (long long)p.q.Hkv * p.total_rows;
  if (rows > 64ll * sm_count) return launch_chained(tree_merge_kernel<D, 2>, dim3((unsigned)((rows + 7) / 8)), dim3(128), 0, st, 1, p);
  return launch_chained(tree_merge_kernel<D, 1>, dim3((unsigned)((rows + 3) / 4)), dim3(128), 0, st, 1, p);
}
}  // namespace
cudaError_t launch_tree_merge(const CacheMerge& p, int d, int sm_count, cudaStream_t st) {
  // few rows of many slots: four warps share a row
  if (p.n_slots > 4 && (long long)p.q.Hkv * p.total_rows <= 16ll * sm_count) return launch_cache_merge(p, d, st);
  return d == 128 ? merge_t<128>(p, sm_count, st) : merge_t<64>(p, sm_count, st);
}

}  // namespace pc
