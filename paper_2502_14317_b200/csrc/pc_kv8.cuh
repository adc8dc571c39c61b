// Codes of the 8-bit caches (pc_kv_cache in pc.h): conversions shared by the kernels that write and read them.
#pragma once
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include "pc_sm100.cuh"

namespace pc {

enum Format { FMT_BF16 = 0, FMT_INT8 = 1, FMT_E4M3 = 2 };

constexpr float KV_TINY = 0x1p-100f;                       // rows whose largest magnitude is below this are held as zeros

__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t sel) { return __byte_perm(a, b, sel); }

// Two codes -> two halves, exactly: every int8 and every e4m3 value is a number of half precision.
// HI = 0: bytes 0 and 1 of x, 1: bytes 2 and 3.  int8: x has its sign bits flipped already (code + 128); put behind 0x64 the byte u
// reads as the half 1024 + u.
template <int FMT, int HI>
__device__ __forceinline__ uint32_t codes_to_half2(uint32_t x) {
  if constexpr (FMT == FMT_INT8) {
    const uint32_t h = prmt(x, 0x64646464u, HI ? 0x4342 : 0x4140);
    const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&h), __half2half2(__ushort_as_half(0x6480)));   // 1152
    return *reinterpret_cast<const uint32_t*>(&r);
  } else {
    uint32_t r;
    const uint16_t two = static_cast<uint16_t>(HI ? x >> 16 : x);
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(two));
    return r;
  }
}
template <int FMT>
__device__ __forceinline__ uint32_t flip_signs(uint32_t x) { return FMT == FMT_INT8 ? x ^ 0x80808080u : x; }

// Four codes times their scale, rounded once to bf16
template <int FMT>
__device__ __forceinline__ uint2 codes_to_bf16x4(uint32_t x, float scale) {
  const uint64_t s2 = pack_f32x2(scale, scale);
  uint64_t lo, hi;
  if constexpr (FMT == FMT_INT8) {                         // a byte u behind 0x4B0000 reads as 2^23 + u
    x = flip_signs<FMT>(x);
    const uint64_t bias = pack_f32x2(-8388736.0f, -8388736.0f);          // 2^23 + 128
    auto f = [&](uint32_t sel) { return __uint_as_float(prmt(x, 0x4B000000u, sel)); };
    lo = add_f32x2(pack_f32x2(f(0x7440), f(0x7441)), bias);
    hi = add_f32x2(pack_f32x2(f(0x7442), f(0x7443)), bias);
  } else {
    const uint32_t h0 = codes_to_half2<FMT, 0>(x), h1 = codes_to_half2<FMT, 1>(x);
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&h0)), b = __half22float2(*reinterpret_cast<const __half2*>(&h1));
    lo = pack_f32x2(a.x, a.y);
    hi = pack_f32x2(b.x, b.y);
  }
  float a, b, c, d;
  unpack_f32x2(mul_f32x2(lo, s2), a, b);
  unpack_f32x2(mul_f32x2(hi, s2), c, d);
  return make_uint2(pack_bf16x2(a, b), pack_bf16x2(c, d));
}

// Four values (already multiplied by Q / a) -> codes
template <int FMT>
__device__ __forceinline__ uint32_t values_to_codes(float a, float b, float c, float d) {
  if constexpr (FMT == FMT_INT8) {
    constexpr float MAGIC = 12582912.0f;                   // 1.5 * 2^23: the sum's low byte is the nearest integer, ties to even
    const uint32_t lo = prmt(__float_as_uint(__fadd_rn(a, MAGIC)), __float_as_uint(__fadd_rn(b, MAGIC)), 0x0040);
    const uint32_t hi = prmt(__float_as_uint(__fadd_rn(c, MAGIC)), __float_as_uint(__fadd_rn(d, MAGIC)), 0x0040);
    return prmt(lo, hi, 0x5410);
  } else {
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return static_cast<uint32_t>(lo) | (static_cast<uint32_t>(hi) << 16);
  }
}
// The power of two that brings a row of queries, whose largest magnitude has the bf16 bits `bits`, into the range of half
// precision (largest in [2^7, 2^8)), and its inverse; 1 where the row is not finite or next to nothing.  Elements 2^-22 below the
// largest become subnormal and lose bits, 2^-32 below it they are gone.
__device__ __forceinline__ float row_factor(uint32_t bits, float& inverse) {
  const int e = (int)(bits >> 7), up = e == 255 || e < 27 ? 0 : 127 + 7 - e;
  inverse = __uint_as_float((uint32_t)(127 - up) << 23);
  return __uint_as_float((uint32_t)(127 + up) << 23);
}

template <int FMT>
__device__ __forceinline__ constexpr float top_code() { return FMT == FMT_INT8 ? 127.0f : 448.0f; }

}  // namespace pc
