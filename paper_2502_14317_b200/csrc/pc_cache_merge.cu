// What stands before and behind the attention kernels of pc_cache_attn: the queries as rows of a kv-head, and the join of a
// row's partial results with the new tokens' own keys.
#include "pc_cache_rows.cuh"
#include "pc_kernels.h"
#include "pc_kv8.cuh"
#include "pc_sm100.cuh"

namespace pc {

// Rows into memory, for the kernel that fetches them with TMA: a block per token, a warp per head.
template <int D>
__global__ void __launch_bounds__(256) cache_rows_kernel(const CacheRows p) {
  constexpr int E = D / 32;
  const int lane = threadIdx.x & 31, G = p.Hq / p.Hkv;
  RowTurner<D> turner(p.theta, lane);
  chain();
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    if (p.clear != nullptr) *p.clear = 0;
    if (p.clear_too != nullptr) *p.clear_too = 0;
  }
  for (int h = threadIdx.x >> 5; h < p.Hq; h += 8) {
    const int hkv = h / G, row = blockIdx.x * G + h % G;
    uint32_t x[E / 2];
    turner.row(p, false, hkv, row, lane, x);
    const size_t at = (size_t)hkv * p.B * p.w * G + row;
    RowTurner<D>::store(p.rows, at, lane, x);
    if (p.halves == nullptr) continue;
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < E / 2; ++i) m = __vmaxu2(m, x[i] & 0x7FFF7FFFu);
    float inv;
    const float f = row_factor(__reduce_max_sync(0xFFFFFFFFu, max(m & 0xFFFFu, m >> 16)), inv);
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {
      const __half2 z = __floats2half2_rn(__uint_as_float(x[i] << 16) * f, __uint_as_float(x[i] & 0xFFFF0000u) * f);
      x[i] = *reinterpret_cast<const uint32_t*>(&z);
    }
    RowTurner<D>::store(p.halves, at, lane, x);
    if (lane == 0) p.half_scale[at] = p.scale_log2 * inv;
  }
}

// Slots of the caches' splits and the new tokens' keys up to the row's own, joined.  WARPS warps share a row: its slots and keys go
// round among them, and their sums meet in shared memory; a lane holds D / 32 columns.
template <int D, int WARPS>
__global__ void __launch_bounds__(128) cache_merge_kernel(const CacheMerge p) {
  constexpr int E = D / 32, U = 4;
  __shared__ float2 stat[4];
  __shared__ float part[4][D];
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, sub = wid % WARPS;
  const int w = p.q.w, G = p.q.Hq / p.q.Hkv;
  chain();
  const long long row = (long long)blockIdx.x * (4 / WARPS) + wid / WARPS;   // hkv * total_rows + (b * w + i) * G + g
  const bool there = row < (long long)p.q.Hkv * p.total_rows;
  const int hkv = there ? (int)(row / p.total_rows) : 0, in = there ? (int)(row % p.total_rows) : 0, g = in % G, bi = in / G, i = bi % w, b = bi / w;
  float top = -INFINITY, sum = 0.0f, acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.0f;
  if (there) {
    const float2* const ml = p.part_ml + row * p.n_slots;
    const float* const po = p.part_o + row * p.n_slots * D + lane * E;
    // this warp's slots, sub, sub + WARPS, ...: a lane each for the statistics
    for (int s0 = 0; s0 * WARPS + sub < p.n_slots; s0 += 32) {
      const int mine_at = (s0 + lane) * WARPS + sub;
      const float2 mine = mine_at < p.n_slots ? ml[mine_at] : make_float2(-INFINITY, 0.0f);
      float most = mine.y == 0.0f ? -INFINITY : mine.x;                      // (0: a split without keys, which left no output)
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
      most = fmaxf(most, top);
      const float f = mine.y == 0.0f ? 0.0f : exp2f(mine.x - most), again = top == -INFINITY ? 0.0f : exp2f(top - most);
      top = most;
      sum *= again;
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] *= again;
      sum = fmaf(f, mine.y, lane == 0 ? sum : 0.0f);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
      const int left = (p.n_slots - sub + WARPS - 1) / WARPS - s0, n = left < 32 ? left : 32;
#pragma unroll 8
      for (int s = 0; s < n; ++s) {
        const float fs = __shfl_sync(0xFFFFFFFFu, f, s), ls = __shfl_sync(0xFFFFFFFFu, mine.y, s);
        const float* const o = po + (long long)((s0 + s) * WARPS + sub) * D;
        if constexpr (E == 4) {
          float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          if (ls != 0.0f) y = __ldg(reinterpret_cast<const float4*>(o));
          acc[0] = fmaf(fs, y.x, acc[0]); acc[1] = fmaf(fs, y.y, acc[1]); acc[2] = fmaf(fs, y.z, acc[2]); acc[3] = fmaf(fs, y.w, acc[3]);
        } else {
          float2 y = make_float2(0.0f, 0.0f);
          if (ls != 0.0f) y = __ldg(reinterpret_cast<const float2*>(o));
          acc[0] = fmaf(fs, y.x, acc[0]); acc[1] = fmaf(fs, y.y, acc[1]);
        }
      }
    }
    if (p.k_win != nullptr && sub <= i) {
      auto load = [&](const uint16_t* at, float (&x)[E]) {
        if constexpr (E == 4) {
          const uint2 y = __ldg(reinterpret_cast<const uint2*>(at) + lane);
          x[0] = __uint_as_float(y.x << 16); x[1] = __uint_as_float(y.x & 0xFFFF0000u);
          x[2] = __uint_as_float(y.y << 16); x[3] = __uint_as_float(y.y & 0xFFFF0000u);
        } else {
          const uint32_t y = __ldg(reinterpret_cast<const uint32_t*>(at) + lane);
          x[0] = __uint_as_float(y << 16); x[1] = __uint_as_float(y & 0xFFFF0000u);
        }
      };
      float q[E];
      load(static_cast<const uint16_t*>(p.q.rows) + row * D, q);
      const uint16_t* const kw = static_cast<const uint16_t*>(p.k_win) + b * p.k_stride[0] + hkv * p.k_stride[2];
      const uint16_t* const vw = static_cast<const uint16_t*>(p.v_win) + b * p.v_stride[0] + hkv * p.v_stride[2];
      for (int j0 = sub; j0 <= i; j0 += U * WARPS) {                         // U keys at a time
        float s[U], v[U][E];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int j = j0 + u * WARPS <= i ? j0 + u * WARPS : i;
          float k[E];
          load(kw + j * p.k_stride[1], k);
          load(vw + j * p.v_stride[1], v[u]);
          s[u] = 0.0f;
#pragma unroll
          for (int e = 0; e < E; ++e) s[u] = fmaf(q[e], k[e], s[u]);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
#pragma unroll
          for (int u = 0; u < U; ++u) s[u] += __shfl_xor_sync(0xFFFFFFFFu, s[u], o);
        float most = top;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          s[u] = j0 + u * WARPS <= i ? s[u] * p.q.scale_log2 : -INFINITY;
          most = fmaxf(most, s[u]);
        }
        const float base = most == -INFINITY ? 0.0f : most, f = exp2f(top - base);
        top = most;
        sum *= f;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] *= f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (j0 + u * WARPS > i) continue;
          const float x = exp2f(s[u] - base);
          sum += x;
#pragma unroll
          for (int e = 0; e < E; ++e) acc[e] = fmaf(x, v[u][e], acc[e]);
        }
      }
    }
  }
  if constexpr (WARPS > 1) {
    if (lane == 0) stat[wid] = make_float2(top, sum);
#pragma unroll
    for (int e = 0; e < E; ++e) part[wid][lane * E + e] = acc[e];
    __syncthreads();
    if (sub != 0) return;
#pragma unroll
    for (int k = 0; k < WARPS; ++k) if (stat[wid + k].y != 0.0f) top = fmaxf(top, stat[wid + k].x);
    sum = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.0f;
#pragma unroll
    for (int k = 0; k < WARPS; ++k) {
      const float2 x = stat[wid + k];
      if (x.y == 0.0f) continue;
      const float f = exp2f(x.x - top);
      sum = fmaf(f, x.y, sum);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = fmaf(f, part[wid + k][lane * E + e], acc[e]);
    }
  }
  if (!there) return;
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;                          // nothing seen: zeros
  const int h = hkv * G + g;
  uint16_t* const out = reinterpret_cast<uint16_t*>(p.out) + ((size_t)bi * p.q.Hq + h) * D;
  if constexpr (E == 4) reinterpret_cast<uint2*>(out)[lane] = make_uint2(pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv));
  else reinterpret_cast<uint32_t*>(out)[lane] = pack_bf16x2(acc[0] * inv, acc[1] * inv);
  if (p.lse != nullptr && lane == 0) p.lse[((size_t)b * p.q.Hq + h) * w + i] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
}

cudaError_t launch_cache_rows(const CacheRows& p, int d, cudaStream_t st) {
  const dim3 grid((unsigned)(p.B * p.w));
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
