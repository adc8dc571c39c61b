// What stands before and behind the attention kernels of pc_cache_attn: the queries as rows of a kv-head, and the join of a
// row's partial results with the new tokens' own keys.
// Both are latency, alone and cold: 256 rows of 8 kv-heads turned 4.5 to 5.1 us, 1024 8.4 to 9.0; 4 rows of 8 kv-heads joined from 17 slots 8.0.
#include "pc_cache_finish.cuh"
#include "pc_cache_rows.cuh"
#include "pc_kernels.h"
#include "pc_kv8.cuh"
#include "pc_sm100.cuh"

namespace pc {

// Rows into memory, for the kernel that fetches them with TMA: blocks of a token and eight of its heads, a warp per head.
template <int D>
__global__ void __launch_bounds__(256) cache_rows_kernel(const CacheRows p) {
  constexpr int E = D / 32;
  const int lane = threadIdx.x & 31, G = p.Hq / p.Hkv;
  RowTurner<D> turner(p.theta, lane);
  chain();
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) {
    if (p.clear != nullptr) p.clear[0] = p.clear[1] = 0;
    if (p.clear_too != nullptr) *p.clear_too = 0;
  }
  const int h = blockIdx.y * 8 + (threadIdx.x >> 5);
  if (h < p.Hq) {
    const int hkv = h / G, row = blockIdx.x * G + h % G;
    uint32_t x[E / 2];
    turner.row(p, false, hkv, row, lane, x);
    const size_t at = (size_t)hkv * p.B * p.w * G + row;
    RowTurner<D>::store(p.rows, at, lane, x);
    leave_beside<D>(p, at, lane, x);
  }
}

// Slots of the caches' splits and the new tokens' keys up to the row's own.  WARPS warps share a row: its slots and keys go round
// among them, and their sums meet in shared memory.
template <int D, int WARPS>
__global__ void __launch_bounds__(128) cache_merge_kernel(const CacheMerge p) {
  constexpr int E = D / 32;
  __shared__ float2 stat[4];
  __shared__ float part[4][D];
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, sub = wid % WARPS, G = p.q.Hq / p.q.Hkv;
  chain();
  const long long row = (long long)blockIdx.x * (4 / WARPS) + wid / WARPS;   // hkv * total_rows + (b * w + i) * G + g
  if (row >= (long long)p.q.Hkv * p.total_rows) return;                      // (of the last block, and whole rows: none waits for it)
  const int hkv = (int)(row / p.total_rows), in = (int)(row % p.total_rows), g = in % G, bi = in / G, i = bi % p.q.w, b = bi / p.q.w;
  RowSum<D> x;
  x.join_slots(p.part_ml + row * p.n_slots, p.part_o + row * p.n_slots * D, p.n_slots, sub, WARPS, lane);
  if (p.k_win != nullptr && sub <= i) {
    float q[E];
    RowSum<D>::load(static_cast<const uint16_t*>(p.q.rows) + row * D, lane, q);
    x.join_window(p, q, hkv, b, i, sub, WARPS, lane);
  }
  if constexpr (WARPS > 1) {
    if (lane == 0) stat[wid] = make_float2(x.top, x.sum);
#pragma unroll
    for (int e = 0; e < E; ++e) part[wid][lane * E + e] = x.acc[e];
    __syncthreads();
    if (sub != 0) return;
    RowSum<D> all;
    all.join(lane < WARPS ? stat[lane] : make_float2(-INFINITY, 0.0f), WARPS, [&](int s, float (&y)[E]) {
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] = part[s][lane * E + e];
    });
    x = all;
  }
  x.store(p, hkv * G + g, bi, lane);
}

cudaError_t launch_cache_rows(const CacheRows& p, int d, cudaStream_t st) {
  const dim3 grid((unsigned)(p.B * p.w), (unsigned)((p.Hq + 7) / 8));
  return d == 128 ? launch_chained(cache_rows_kernel<128>, grid, dim3(256), 0, st, 1, p) : launch_chained(cache_rows_kernel<64>, grid, dim3(256), 0, st, 1, p);
}
namespace {
template <int D>
cudaError_t merge_t(const CacheMerge& p, cudaStream_t st) {
  const long long rows = (long long)p.q.Hkv * p.total_rows;
  // a row's chain of slots and keys is shared by four warps where it is long
  if (p.n_slots > 4 || p.q.w > 8) return launch_chained(cache_merge_kernel<D, 4>, dim3((unsigned)rows), dim3(128), 0, st, 1, p);
  return launch_chained(cache_merge_kernel<D, 1>, dim3((unsigned)((rows + 3) / 4)), dim3(128), 0, st, 1, p);
}
}  // namespace
cudaError_t launch_cache_merge(const CacheMerge& p, int d, cudaStream_t st) { return d == 128 ? merge_t<128>(p, st) : merge_t<64>(p, st); }

}  // namespace pc
