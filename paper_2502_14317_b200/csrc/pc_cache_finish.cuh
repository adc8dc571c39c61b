// A row's partial results joined, with the new tokens' own keys, into its output: shared by the kernel for few rows, which finishes
// its rows where it can, and the merge kernel.  A warp has a row, a lane D / 32 of its columns.
#pragma once
#include "pc_cache.h"
#include "pc_sm100.cuh"

namespace pc {

template <int D>
struct RowSum {
  static constexpr int E = D / 32;
  float top = -INFINITY, sum = 0.0f, acc[E];                 // maximum (log2 units), sum and output relative to it
  __device__ __forceinline__ RowSum() {
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.0f;
  }
  // Up to 32 results at a time: lane s has the statistics of the s-th (sum 0: none, and no output); fetch(s, x) loads its columns.
  template <class F>
  __device__ __forceinline__ void join(float2 mine, int n, const F& fetch) {
    float most = mine.y == 0.0f ? -INFINITY : mine.x;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
    most = fmaxf(most, top);
    const float f = mine.y == 0.0f ? 0.0f : exp2f(mine.x - most), again = top == -INFINITY ? 0.0f : exp2f(top - most);
    top = most;
    float l = mine.y == 0.0f ? 0.0f : f * mine.y;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, o);
    sum = fmaf(sum, again, l);
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] *= again;
#pragma unroll 8
    for (int s = 0; s < n; ++s) {
      const float fs = __shfl_sync(0xFFFFFFFFu, f, s), ls = __shfl_sync(0xFFFFFFFFu, mine.y, s);
      float x[E] = {};
      if (ls != 0.0f) fetch(s, x);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = fmaf(fs, x[e], acc[e]);
    }
  }
  // slots first, first + step, ... of the row's n in memory
  __device__ __forceinline__ void join_slots(const float2* ml, const float* po, int n, int first, int step, int lane) {
    const int mine = n > first ? (n - first + step - 1) / step : 0;
    for (int s0 = 0; s0 < mine; s0 += 32) {
      const float2 x = s0 + lane < mine ? ml[first + (s0 + lane) * step] : make_float2(-INFINITY, 0.0f);
      join(x, mine - s0 < 32 ? mine - s0 : 32, [&](int s, float (&y)[E]) {
        const float* const from = po + (long long)(first + (s0 + s) * step) * D + lane * E;
        if constexpr (E == 4) { const float4 z = *reinterpret_cast<const float4*>(from); y[0] = z.x; y[1] = z.y; y[2] = z.z; y[3] = z.w; }
        else { const float2 z = *reinterpret_cast<const float2*>(from); y[0] = z.x; y[1] = z.y; }
      });
    }
  }
  static __device__ __forceinline__ void unpack(const uint32_t (&y)[E / 2], float (&x)[E]) {
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = __uint_as_float(e % 2 ? y[e / 2] & 0xFFFF0000u : y[e / 2] << 16);
  }
  static __device__ __forceinline__ void load(const uint16_t* at, int lane, float (&x)[E]) {
    uint32_t y[E / 2];
    if constexpr (E == 4) { const uint2 z = __ldg(reinterpret_cast<const uint2*>(at) + lane); y[0] = z.x; y[1] = z.y; }
    else y[0] = __ldg(reinterpret_cast<const uint32_t*>(at) + lane);
    unpack(y, x);
  }
  // the keys first, first + step, ... of the new tokens up to i, the row's own; four at a time (eight: merge of a window of 64 15.0 -> 17.5 us)
  __device__ __forceinline__ void join_window(const CacheMerge& p, const float (&q)[E], int hkv, int b, int i, int first, int step, int lane) {
    constexpr int U = 4;
    const uint16_t* const kw = static_cast<const uint16_t*>(p.k_win) + b * p.k_stride[0] + hkv * p.k_stride[2];
    const uint16_t* const vw = static_cast<const uint16_t*>(p.v_win) + b * p.v_stride[0] + hkv * p.v_stride[2];
    for (int j0 = first; j0 <= i; j0 += U * step) {
      float s[U], v[U][E];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int j = j0 + u * step <= i ? j0 + u * step : i;
        float k[E];
        load(kw + j * p.k_stride[1], lane, k);
        load(vw + j * p.v_stride[1], lane, v[u]);
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
        s[u] = j0 + u * step <= i ? s[u] * p.q.scale_log2 : -INFINITY;
        most = fmaxf(most, s[u]);
      }
      const float base = most == -INFINITY ? 0.0f : most, f = exp2f(top - base);
      top = most;
      sum *= f;
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] *= f;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (j0 + u * step > i) continue;
        const float x = exp2f(s[u] - base);
        sum += x;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = fmaf(x, v[u][e], acc[e]);
      }
    }
  }
  // q-head h, token bi = b * w + i; nothing seen: zeros and -infinity
  __device__ __forceinline__ void store(const CacheMerge& p, int h, int bi, int lane) const {
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    uint16_t* const out = reinterpret_cast<uint16_t*>(p.out) + ((size_t)bi * p.q.Hq + h) * D;
    if constexpr (E == 4) reinterpret_cast<uint2*>(out)[lane] = make_uint2(pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv));
    else reinterpret_cast<uint32_t*>(out)[lane] = pack_bf16x2(acc[0] * inv, acc[1] * inv);
    if (p.lse != nullptr && lane == 0)
      p.lse[((size_t)(bi / p.q.w) * p.q.Hq + h) * p.q.w + bi % p.q.w] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
  }
};

}  // namespace pc
