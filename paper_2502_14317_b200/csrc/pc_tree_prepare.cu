// The rotated queries of pc_tree_attn as rows in memory, for kernels whose CTAs do not make them, and who sees whom.
#include "pc_kernels.h"
#include "pc_tree_rows.cuh"

namespace pc {

// blocks of a token and eight of its heads, a warp per head
template <int D>
__global__ void __launch_bounds__(256) tree_rows_kernel(const __grid_constant__ CacheRows p, const __grid_constant__ TreePhase t) {
  const int lane = threadIdx.x & 31, G = p.Hq / p.Hkv;
  TreeTurner<D> turner(t, lane);
  chain();
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) {
    if (p.clear != nullptr) p.clear[0] = p.clear[1] = 0;
    if (p.clear_too != nullptr) *p.clear_too = 0;
  }
  const int h = blockIdx.y * 8 + (threadIdx.x >> 5), seq = blockIdx.x / p.w, i = blockIdx.x - seq * p.w;
  if (h >= p.Hq) return;
  const unsigned long long sees = tree_seen(t.parents == nullptr ? nullptr : t.parents + seq * t.parent_stride, p.w, lane).of(i);
  if (h == 0 && lane == 0) t.sees[blockIdx.x] = sees;
  const int hkv = h / G, row = blockIdx.x * G + h % G;
  uint32_t x[D / 64];
  turner.place(p, seq, __ldg(t.lens + seq), __popcll(sees));
  turner.row(p, false, hkv, row, lane, x);
  const size_t at = (size_t)hkv * p.B * p.w * G + row;
  TreeTurner<D>::store(p.rows, at, lane, x);
  leave_beside<D>(p, at, lane, x);
}

cudaError_t launch_tree_rows(const CacheRows& p, const TreePhase& t, int d, cudaStream_t st) {
  const dim3 grid((unsigned)(p.B * p.w), (unsigned)((p.Hq + 7) / 8));
  return d == 128 ? launch_chained(tree_rows_kernel<128>, grid, dim3(256), 0, st, 1, p, t) : launch_chained(tree_rows_kernel<64>, grid, dim3(256), 0, st, 1, p, t);
}

}  // namespace pc
