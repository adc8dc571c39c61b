// New keys and values into the pages of their sequences (pc_page_append): keys are rotated to their positions on the way.
//
// Bound by memory: a row of keys or values is read once (2 d bytes) and written once (2 d, or d + 4 in 8 bits).  d / 8 lanes hold a token's rows, four heads
// at a time, keys as four elements of either half, so that a lane has whole pairs and the angles of its four pairs serve all heads.  The angles are
// computed where they are used (pc_tree.cuh): a table of them would be read as often as the rows of one head.  16 (head size 64: 32) consecutive
// tokens of a block write 4 KB that lie together, if their page does not end.  A key that goes into 8 bits is not rounded to bf16 before.
// Measured: 65537 tokens of 8 heads of 128 in bf16 (537 MB) 85 to 88 us = 6.3 to 6.1 TB/s; one token 2.6 us as a graph, in a loop of calls 4.4 (the host).
#include "pc_kernels.h"
#include "pc_kv8.cuh"
#include "pc_tree.cuh"

namespace pc {

namespace {

constexpr int NT = 256, HEADS = 4;

__device__ __forceinline__ float lo16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi16(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// largest magnitude's bits of the row that LANES lanes hold
template <int LANES>
__device__ __forceinline__ uint32_t row_max(uint32_t m) {
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
  return m;
}
// Q / a (0: codes 0) and scale of a row (definition: pc_kv_cache in pc.h)
template <int FMT>
__device__ __forceinline__ float row_scale(uint32_t bits, float& scale) {
  const float a = __uint_as_float(bits);
  const bool held = a >= KV_TINY && bits < 0x7F800000u;
  scale = bits >= 0x7F800000u ? __uint_as_float(0x7FC00000u) : held ? __fdiv_rn(a, top_code<FMT>()) : 0.0f;
  return held ? __fdiv_rn(top_code<FMT>(), a) : 0.0f;
}
template <int FMT>
__device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d, float r) {
  return r == 0.0f ? 0u : values_to_codes<FMT>(__fmul_rn(a, r), __fmul_rn(b, r), __fmul_rn(c, r), __fmul_rn(d, r));
}

}  // namespace

// grid: (tokens of a sequence in blocks, heads in fours, sequences)
template <int D, int FMT>
__global__ void __launch_bounds__(NT) page_append_kernel(const __grid_constant__ PageWrite p) {
  constexpr int LANES = D / 8, GROUPS = NT / LANES;
  const int lane = threadIdx.x % LANES, h0 = blockIdx.y * HEADS;
  double part[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) part[t] = part_of_turn(p.turns, 4 * lane + t);
  chain();
  for (int b = blockIdx.z; b < p.B; b += gridDim.z) {
    const long long at = (long long)p.at0 + (p.at ? __ldg(p.at + b) : 0);
    if (at < 0) continue;                                      // no such sequence
    const int n = p.count ? min(max(__ldg(p.count + b), 0), p.n) : p.n;
    const long long pos = (long long)p.pos0 + (p.pos ? __ldg(p.pos + b) : at);
    Seen seen = {};
    if (p.parents != nullptr) seen = tree_seen(p.parents + b * p.parent_stride, p.n, threadIdx.x & 31);
    const int i = blockIdx.x * GROUPS + threadIdx.x / LANES;   // (whole warps go through the exchanges below)
    int from = i, step = i;
    bool there = i < n;
    if (p.pick != nullptr) {
      from = there ? __ldg(p.pick + b * p.pick_stride + i) : -1;
      there = from >= 0 && from < p.n_src;
    }
    if (p.parents != nullptr) {
      const unsigned long long mine = seen.of(i & 63);
      step = __popcll(mine) - 1;
      there = there && mine != 0;
    }
    if (__ballot_sync(0xFFFFFFFFu, there) == 0) continue;
    long long to = 0;                                          // row of head 0 in the pool
    if (there) {
      const long long e = at + i;
      int id = -1;
      long long in = 0;
      if (e < (long long)p.pages.n_table * p.pages.page) {
        const int which = page_of(p.pages, (int)e);
        id = __ldg(p.pages.table + b * p.pages.stride + which);
        in = e - (long long)which * p.pages.page;
      }
      if (id < 0 || id >= p.pages.n_pages) {
        there = false;
        if (lane == 0 && h0 == 0 && p.status) atomicCAS(p.status, 0, 421);
      }
      to = (long long)id * p.Hkv * p.pages.page + in;
    }
    const uint16_t* const ks = static_cast<const uint16_t*>(p.k_src) + b * p.k_stride[0] + from * p.k_stride[1];
    const uint16_t* const vs = static_cast<const uint16_t*>(p.v_src) + b * p.v_stride[0] + from * p.v_stride[1];
    uint2 k0[HEADS], k1[HEADS];
    uint4 v[HEADS];
#pragma unroll
    for (int u = 0; u < HEADS; ++u) {
      k0[u] = k1[u] = make_uint2(0, 0);
      v[u] = make_uint4(0, 0, 0, 0);
      if (there && h0 + u < p.Hkv) {
        const uint16_t* const k = ks + (h0 + u) * p.k_stride[2];
        k0[u] = __ldg(reinterpret_cast<const uint2*>(k) + lane);
        k1[u] = __ldg(reinterpret_cast<const uint2*>(k + D / 2) + lane);
        v[u] = __ldg(reinterpret_cast<const uint4*>(vs + (h0 + u) * p.v_stride[2]) + lane);
      }
    }
    float2 cs[4];
    if (p.turn) {
#pragma unroll
      for (int t = 0; t < 4; ++t) cs[t] = turned(part[t], pos + step);
    }
#pragma unroll
    for (int u = 0; u < HEADS; ++u) {
      if (h0 + u >= p.Hkv) break;
      float x[4] = {lo16(k0[u].x), hi16(k0[u].x), lo16(k0[u].y), hi16(k0[u].y)}, y[4] = {lo16(k1[u].x), hi16(k1[u].x), lo16(k1[u].y), hi16(k1[u].y)};
      if (p.turn) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const float a = x[t], c = y[t];
          x[t] = a * cs[t].x - c * cs[t].y;
          y[t] = c * cs[t].x + a * cs[t].y;
        }
      }
      const long long row = to + (long long)(h0 + u) * p.pages.page;
      if constexpr (FMT == FMT_BF16) {
        if (there) {
          uint16_t* const k = reinterpret_cast<uint16_t*>(p.k) + row * D;
          reinterpret_cast<uint2*>(k)[lane] = p.turn ? make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])) : k0[u];
          reinterpret_cast<uint2*>(k + D / 2)[lane] = p.turn ? make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])) : k1[u];
          reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(p.v) + row * D)[lane] = v[u];
        }
      } else {
        uint32_t mk = 0, mv;
#pragma unroll
        for (int t = 0; t < 4; ++t) mk = max(mk, max(magnitude(x[t]), magnitude(y[t])));
        const uint32_t m2 = __vmaxu2(__vmaxu2(v[u].x & 0x7FFF7FFFu, v[u].y & 0x7FFF7FFFu), __vmaxu2(v[u].z & 0x7FFF7FFFu, v[u].w & 0x7FFF7FFFu));
        mv = max(m2 << 16, m2 & 0x7FFF0000u);
        float sk, sv;
        const float rk = row_scale<FMT>(row_max<LANES>(mk), sk), rv = row_scale<FMT>(row_max<LANES>(mv), sv);
        if (there) {
          reinterpret_cast<uint32_t*>(p.k + row * D)[lane] = four_codes<FMT>(x[0], x[1], x[2], x[3], rk);
          reinterpret_cast<uint32_t*>(p.k + row * D + D / 2)[lane] = four_codes<FMT>(y[0], y[1], y[2], y[3], rk);
          reinterpret_cast<uint2*>(p.v + row * D)[lane] = make_uint2(four_codes<FMT>(lo16(v[u].x), hi16(v[u].x), lo16(v[u].y), hi16(v[u].y), rv),
                                                                     four_codes<FMT>(lo16(v[u].z), hi16(v[u].z), lo16(v[u].w), hi16(v[u].w), rv));
          if (lane == 0) { p.k_scale[row] = sk; p.v_scale[row] = sv; }
        }
      }
    }
  }
}

namespace {

template <int D, int FMT>
cudaError_t append_t(const PageWrite& w, cudaStream_t st) {
  constexpr int GROUPS = NT / (D / 8);
  const dim3 grid((unsigned)((w.n + GROUPS - 1) / GROUPS), (unsigned)((w.Hkv + HEADS - 1) / HEADS), (unsigned)(w.B < 65535 ? w.B : 65535));
  return launch_chained(page_append_kernel<D, FMT>, grid, dim3(NT), 0, st, 1, w);
}
template <int D>
cudaError_t append_d(const PageWrite& w, int format, cudaStream_t st) {
  return format == FMT_BF16 ? append_t<D, FMT_BF16>(w, st) : format == FMT_INT8 ? append_t<D, FMT_INT8>(w, st) : append_t<D, FMT_E4M3>(w, st);
}

}  // namespace

cudaError_t launch_page_append(const PageWrite& w, int format, int d, cudaStream_t st) {
  return d == 128 ? append_d<128>(w, format, st) : append_d<64>(w, format, st);
}

}  // namespace pc
