// What stands before and behind the attention kernels of pc_cache_attn: the queries as rows of a kv-head, and the join of a
// row's partial results with the new tokens' own keys.
#include "pc_cache.h"
#include "pc_kernels.h"
#include "pc_sm100.cuh"

namespace pc {

// rows[hkv][(b * w + i) * G + g][:] = the fp64 rotation of q[b, i, hkv * G + g, :] rounded once to bf16, pairs (t, t + d/2).  A block
// per token: its angles are computed once, ahead of the wait for the kernel before (as far as they do not depend on it).
template <int D>
__global__ void __launch_bounds__(256) cache_rows_kernel(const CacheRows p) {
  constexpr int HALF = D / 2;
  __shared__ double cs[HALF], sn[HALF];
  const int b = blockIdx.x / p.w, i = blockIdx.x % p.w, G = p.Hq / p.Hkv;
  const int tid = threadIdx.x;
  const bool turn = p.theta > 0.0;
  double freq = 0.0;
  if (turn && tid < HALF) freq = pow(p.theta, -2.0 * (double)tid / (double)D);
  chain();
  if (turn && tid < HALF) {
    const long long pos = (long long)p.pos0 + (p.pos ? p.pos[b] : 0) + i;
    sincos((double)pos * freq, &sn[tid], &cs[tid]);
  }
  __syncthreads();
  const uint16_t* const q = static_cast<const uint16_t*>(p.q) + b * p.stride[0] + i * p.stride[1];
  uint16_t* const rows = static_cast<uint16_t*>(p.rows);
  for (int e = tid; e < p.Hq * HALF; e += 256) {
    const int h = e / HALF, t = e % HALF, hkv = h / G, g = h % G;
    uint16_t x = q[h * p.stride[2] + t], y = q[h * p.stride[2] + t + HALF];
    if (turn) {
      const double u = (double)__uint_as_float((uint32_t)x << 16), v = (double)__uint_as_float((uint32_t)y << 16);
      x = f64_to_bf16_rne(u * cs[t] - v * sn[t]);
      y = f64_to_bf16_rne(v * cs[t] + u * sn[t]);
    }
    uint16_t* const to = rows + (((size_t)hkv * p.B * p.w + blockIdx.x) * G + g) * D + t;
    to[0] = x;
    to[HALF] = y;
  }
}

// One warp per row: a lane holds D / 32 of its columns.  Slots of the caches' splits first, then the new tokens' keys up to the row's own.
template <int D>
__global__ void __launch_bounds__(128) cache_merge_kernel(const CacheMerge p) {
  constexpr int E = D / 32;
  chain();
  const int G = p.Hq / p.Hkv, lane = threadIdx.x & 31;
  const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);      // hkv * total_rows + (b * w + i) * G + g
  if (row >= (long long)p.Hkv * p.total_rows) return;
  const int hkv = (int)(row / p.total_rows), in = (int)(row % p.total_rows), g = in % G, bi = in / G, i = bi % p.w, b = bi / p.w;
  float top = -INFINITY, sum = 0.0f, acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.0f;
  const float2* const ml = p.part_ml + row * p.n_slots;
  const float* const po = p.part_o + row * p.n_slots * D + lane * E;
  for (int s = lane; s < p.n_slots; s += 32) { const float2 x = ml[s]; if (x.y != 0.0f) top = fmaxf(top, x.x); }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
  for (int s0 = 0; s0 < p.n_slots; s0 += 32) {
    const float2 mine = s0 + lane < p.n_slots ? ml[s0 + lane] : make_float2(-INFINITY, 0.0f);
    const float f = mine.y == 0.0f ? 0.0f : exp2f(mine.x - top);             // 0: a split without keys left no output
    const int n = p.n_slots - s0 < 32 ? p.n_slots - s0 : 32;
#pragma unroll 4
    for (int s = 0; s < n; ++s) {
      const float fs = __shfl_sync(0xFFFFFFFFu, f, s), ls = __shfl_sync(0xFFFFFFFFu, mine.y, s);
      if (ls == 0.0f) continue;
      sum = fmaf(fs, ls, sum);
      const float* const o = po + (long long)(s0 + s) * D;
      if constexpr (E == 4) {
        const float4 y = __ldg(reinterpret_cast<const float4*>(o));
        acc[0] = fmaf(fs, y.x, acc[0]); acc[1] = fmaf(fs, y.y, acc[1]); acc[2] = fmaf(fs, y.z, acc[2]); acc[3] = fmaf(fs, y.w, acc[3]);
      } else {
        const float2 y = __ldg(reinterpret_cast<const float2*>(o));
        acc[0] = fmaf(fs, y.x, acc[0]); acc[1] = fmaf(fs, y.y, acc[1]);
      }
    }
  }
  if (p.k_win != nullptr) {
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
    load(reinterpret_cast<const uint16_t*>(p.q_rows) + row * D, q);
    const uint16_t* const kw = static_cast<const uint16_t*>(p.k_win) + b * p.k_stride[0] + hkv * p.k_stride[2];
    const uint16_t* const vw = static_cast<const uint16_t*>(p.v_win) + b * p.v_stride[0] + hkv * p.v_stride[2];
    constexpr int U = 4;                                                     // keys at a time
    for (int j0 = 0; j0 <= i; j0 += U) {
      float s[U], v[U][E];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int j = j0 + u <= i ? j0 + u : i;
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
        s[u] = j0 + u <= i ? s[u] * p.scale_log2 : -INFINITY;
        most = fmaxf(most, s[u]);
      }
      const float base = most == -INFINITY ? 0.0f : most, f = exp2f(top - base);
      top = most;
      sum *= f;
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] *= f;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (j0 + u > i) continue;
        const float w = exp2f(s[u] - base);
        sum += w;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = fmaf(w, v[u][e], acc[e]);
      }
    }
  }
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;                          // nothing seen: zeros
  const int h = hkv * G + g;
  uint16_t* const out = reinterpret_cast<uint16_t*>(p.out) + ((size_t)bi * p.Hq + h) * D;
  if constexpr (E == 4) reinterpret_cast<uint2*>(out)[lane] = make_uint2(pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv));
  else reinterpret_cast<uint32_t*>(out)[lane] = pack_bf16x2(acc[0] * inv, acc[1] * inv);
  if (p.lse != nullptr && lane == 0) p.lse[((size_t)b * p.Hq + h) * p.w + i] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
}

cudaError_t launch_cache_rows(const CacheRows& p, int d, cudaStream_t st) {
  const dim3 grid((unsigned)(p.B * p.w));
  return d == 128 ? launch_chained(cache_rows_kernel<128>, grid, dim3(256), 0, st, 1, p) : launch_chained(cache_rows_kernel<64>, grid, dim3(256), 0, st, 1, p);
}
cudaError_t launch_cache_merge(const CacheMerge& p, int d, cudaStream_t st) {
  const dim3 grid((unsigned)(((long long)p.Hkv * p.total_rows + 3) / 4));
  return d == 128 ? launch_chained(cache_merge_kernel<128>, grid, dim3(128), 0, st, 1, p) : launch_chained(cache_merge_kernel<64>, grid, dim3(128), 0, st, 1, p);
}

}  // namespace pc
