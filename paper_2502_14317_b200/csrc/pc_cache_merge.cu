// What stands before and behind the attention kernels of pc_cache_attn: the queries as rows of a kv-head, and the join of a
// row's partial results with the new tokens' own keys.
#include "pc_cache.h"
#include "pc_kernels.h"
#include "pc_kv8.cuh"
#include "pc_sm100.cuh"
#include <type_traits>

namespace pc {

// rows[hkv][(b * w + i) * G + g][:] = q[b, i, hkv * G + g, :] rotated in fp32, pairs (t, t + d/2), and rounded to bf16.  A block per
// token, a warp per head: a lane holds one pair (d = 64) or two adjacent ones, whose angles it computes once.
// The angle is one fp32 product of the position and theta^(-2t/d), as models compute it: off by at most 2^-22 of itself, up to
// position 8192, the longest chunk, by less than half a step of the bf16 result.  From position 2^15 on it is computed in fp64, where the
// fp32 product would be off by whole steps; fp64 everywhere costs FP64_US.
template <int D>
__global__ void __launch_bounds__(256) cache_rows_kernel(const CacheRows p) {
  constexpr int E = D / 64;                                   // pairs of a lane
  using Word = typename std::conditional<E == 2, uint32_t, uint16_t>::type;
  const int b = blockIdx.x / p.w, i = blockIdx.x % p.w, G = p.Hq / p.Hkv, lane = threadIdx.x & 31;
  const bool turn = p.theta > 0.0f;
  float freq[E], c[E], s[E];
#pragma unroll
  for (int e = 0; e < E; ++e) freq[e] = turn ? powf(p.theta, -2.0f * (float)(E * lane + e) / (float)D) : 0.0f;
  chain();
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    if (p.clear != nullptr) *p.clear = 0;
    if (p.clear_too != nullptr) *p.clear_too = 0;
  }
  const long long pos = (long long)p.pos0 + (p.pos ? p.pos[b] : 0) + i;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if (pos < (1 << 15)) {
      const float a = __fmul_rn((float)pos, freq[e]);
      c[e] = cosf(a); s[e] = sinf(a);
    } else {
      double cd, sd;
      sincos((double)pos * pow((double)p.theta, -2.0 * (double)(E * lane + e) / (double)D), &sd, &cd);
      c[e] = (float)cd; s[e] = (float)sd;
    }
  }
  const uint16_t* const q = static_cast<const uint16_t*>(p.q) + b * p.stride[0] + i * p.stride[1];
  for (int h = threadIdx.x >> 5; h < p.Hq; h += 8) {
    const int hkv = h / G, g = h % G;
    const size_t row = ((size_t)hkv * p.B * p.w + blockIdx.x) * G + g;
    const Word xw = reinterpret_cast<const Word*>(q + h * p.stride[2])[lane], yw = reinterpret_cast<const Word*>(q + h * p.stride[2] + D / 2)[lane];
    uint16_t u[E], v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      u[e] = (uint16_t)(xw >> (16 * e)); v[e] = (uint16_t)(yw >> (16 * e));
      if (turn) {
        const float x = __uint_as_float((uint32_t)u[e] << 16), y = __uint_as_float((uint32_t)v[e] << 16);
        u[e] = __bfloat16_as_ushort(__float2bfloat16_rn(__fsub_rn(__fmul_rn(x, c[e]), __fmul_rn(y, s[e]))));
        v[e] = __bfloat16_as_ushort(__float2bfloat16_rn(__fadd_rn(__fmul_rn(y, c[e]), __fmul_rn(x, s[e]))));
      }
    }
    Word* const to = reinterpret_cast<Word*>(static_cast<uint16_t*>(p.rows) + row * D);
    if constexpr (E == 2) { to[lane] = u[0] | (uint32_t)u[1] << 16; to[32 + lane] = v[0] | (uint32_t)v[1] << 16; }
    else { to[lane] = u[0]; to[32 + lane] = v[0]; }
    if (p.halves == nullptr) continue;
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) m = max(m, (uint32_t)max(u[e] & 0x7FFF, v[e] & 0x7FFF));
    m = __reduce_max_sync(0xFFFFFFFFu, m);
    float inv;
    const float f = row_factor(m, inv);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      u[e] = __half_as_ushort(__float2half_rn(__uint_as_float((uint32_t)u[e] << 16) * f));
      v[e] = __half_as_ushort(__float2half_rn(__uint_as_float((uint32_t)v[e] << 16) * f));
    }
    Word* const th = reinterpret_cast<Word*>(static_cast<uint16_t*>(p.halves) + row * D);
    if constexpr (E == 2) { th[lane] = u[0] | (uint32_t)u[1] << 16; th[32 + lane] = v[0] | (uint32_t)v[1] << 16; }
    else { th[lane] = u[0]; th[32 + lane] = v[0]; }
    if (lane == 0) p.half_scale[row] = p.scale_log2 * inv;
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
