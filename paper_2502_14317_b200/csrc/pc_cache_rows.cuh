// The rotated queries of pc_cache_attn, a row per warp: lane l holds the elements E l .. E l + E - 1, E = d / 32.
//
// In fp32, pairs (t, t + d/2), angle = position * theta^(-2t/d) as one fp32 product, as models compute it: off by at most 2^-22 of
// itself, up to position 8192, the longest chunk, by less than half a step of the bf16 result, at 2^15 by up to two.  From there on the angle is
// computed in fp64.  A caller who wants the fp64 rotation everywhere, as the keys of this library have it, rotates the queries and gives theta 0.
#pragma once
#include "pc_cache.h"
#include "pc_sm100.cuh"

namespace pc {

// Out of line: cold code costs a short kernel more than the calls do.
static __device__ __noinline__ float row_freq(float theta, float exponent) { return powf(theta, exponent); }
static __device__ __noinline__ float2 row_angle_far(long long pos, float theta, float exponent) {
  double c, s;
  sincos((double)pos * pow((double)theta, (double)exponent), &s, &c);
  return make_float2((float)c, (float)s);
}
static __device__ __noinline__ float2 row_angle(float freq, long long pos, float theta, float exponent) {
  if (pos >= (1 << 15) || pos < 0) return row_angle_far(pos, theta, exponent);
  const float a = __fmul_rn((float)pos, freq);
  return make_float2(cosf(a), sinf(a));
}

// Angles of a token's pairs: lanes l and l + 16 hold elements of the same E pairs and compute half of them each.
template <int D>
struct RowTurner {
  static constexpr int E = D / 32, H = E / 2;
  float freq[H], c[E], s[E];
  int token = -1;                                             // whose angles are held
  static __device__ __forceinline__ float exponent(int lane, int k) {   // exact: D is a power of two
    return -2.0f * (float)(E * (lane & 15) + (lane >> 4) * H + k) / (float)D;
  }
  // needs nothing from before the launch
  __device__ __forceinline__ RowTurner(float theta, int lane) {
#pragma unroll
    for (int k = 0; k < H; ++k) freq[k] = theta > 0.0f ? row_freq(theta, exponent(lane, k)) : 0.0f;
  }
  __device__ __forceinline__ void angles(const CacheRows& p, int t, int lane) {
    if (t == token) return;
    token = t;
    const long long pos = (long long)p.pos0 + (p.pos ? p.pos[t / p.w] : 0) + t % p.w;
#pragma unroll
    for (int k = 0; k < H; ++k) {
      const float2 a = row_angle(freq[k], pos, p.theta, exponent(lane, k));
      const float2 b = make_float2(__shfl_xor_sync(0xFFFFFFFFu, a.x, 16), __shfl_xor_sync(0xFFFFFFFFu, a.y, 16));
      c[k] = lane < 16 ? a.x : b.x; s[k] = lane < 16 ? a.y : b.y;
      c[H + k] = lane < 16 ? b.x : a.x; s[H + k] = lane < 16 ? b.y : a.y;
    }
  }
  // row `row` of kv-head hkv as bf16 pairs; the whole warp calls
  __device__ __forceinline__ void row(const CacheRows& p, bool in_memory, int hkv, int row, int lane, uint32_t (&x)[E / 2]) {
    const int G = p.Hq / p.Hkv;
    const uint16_t* at;
    if (in_memory) {
      at = static_cast<const uint16_t*>(p.rows) + ((size_t)hkv * p.B * p.w * G + row) * D;
    } else {
      const int t = row / G;
      at = static_cast<const uint16_t*>(p.q) + t / p.w * p.stride[0] + t % p.w * p.stride[1] + (hkv * G + row % G) * p.stride[2];
    }
    if constexpr (E == 4) {
      const uint2 y = __ldg(reinterpret_cast<const uint2*>(at) + lane);
      x[0] = y.x; x[1] = y.y;
    } else {
      x[0] = __ldg(reinterpret_cast<const uint32_t*>(at) + lane);
    }
    if (in_memory || !(p.theta > 0.0f)) return;
    angles(p, row / G, lane);
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {
      const uint32_t y = __shfl_xor_sync(0xFFFFFFFFu, x[i], 16);     // the other elements of the pairs
      uint32_t r = 0;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float u = __uint_as_float(e ? x[i] & 0xFFFF0000u : x[i] << 16), v = __uint_as_float(e ? y & 0xFFFF0000u : y << 16);
        const float a = __fmul_rn(u, c[2 * i + e]), b = __fmul_rn(v, s[2 * i + e]);
        const float z = lane < 16 ? __fsub_rn(a, b) : __fadd_rn(a, b);   // x cos - y sin, y cos + x sin
        r |= (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(z)) << (16 * e);
      }
      x[i] = r;
    }
  }
  static __device__ __forceinline__ void store(void* rows, size_t at, int lane, const uint32_t (&x)[E / 2]) {
    if constexpr (E == 4) reinterpret_cast<uint2*>(static_cast<uint16_t*>(rows) + at * D)[lane] = make_uint2(x[0], x[1]);
    else reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(rows) + at * D)[lane] = x[0];
  }
};

}  // namespace pc
