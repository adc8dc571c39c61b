// Log probabilities of given tokens, entropy and the most probable tokens of rows of logits (pc_token_logprobs).
//
// One pass over a row x of V logits.  A thread keeps, over its share, a reference logit m and with c = scale * log2 e, t = x c - m c, the sums
//     s = sum 2^t,      h = sum 2^t t,
// and raises m (s and h to be taken along) only where a logit exceeds it by more than 2^8.  With M the largest m, all joined,
//     log p(x) = (x - M) scale - ln s,      H = ln s - ln 2 h / s.
// The sums are taken against R = m c rounded, one fused operation a term, and moved to m c itself at the end.  Logits that are so far below m that their term
// is 0 are raised to where it still is, so that -inf has no product 0 * inf; in the types of 16 bits two at a time, before they are widened.  While a
// share has nothing but -inf and values next to the type's lowest, or R is so large that its rounding counts, t = (x - m) c.
//
// The top k: of each quarter of its share a thread also keeps the largest logit and the piece of 16 bytes in which it first stood.  With keys (order of the value,
// earlier piece first), of which no two are the same, let T be the k-th largest of the maxima of groups of four threads: k logits in k different pieces
// are not below T, so only logits that are not can be among the k largest, and only quarters whose own maximum is not below T have any.  Those are read
// once more (from L2, some k of 1024), everything else is left alone.  What is found, a few more than k, is ranked by counting: keys (order of the
// value, lower index first) are all different, so ties need no rule of their own.  Lists of a row's parts are merged, a warp's registers each.
//
// A row is the work of a cluster of 1 to 8 CTAs (rule at the launch).
//
// Bound, many rows, by the exponentials and the issue of instructions beside the reading: at 1024 x 128256 in bf16 with 8 alternatives (263 MB) the exponentials' unit
// is busy for 65 %, issue 70, memory 63: 53 to 59 us by the board = 5.0 to 4.5 TB/s; without alternatives 6 us less, with 32 of them 11 more.  276 rows of 50001 in fp16 whose pitch is odd
// 12 us; one row of 128256 in fp32 with 20 alternatives 8.5, a chain of latencies.
#include "pc_kernels.h"
#include "pc_logprob.h"
#include "pc_rank.cuh"
#include "pc_sm100.cuh"
#include <cfloat>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace pc {

namespace {

constexpr int NT = 256, WARPS = NT / 32, CTAS = 4, U = 4;
using Key = unsigned long long;                              // 0: none

template <int TYPE> struct Logit { static constexpr int BYTES = TYPE == LOGITS_F32 ? 4 : 2, VEC = 16 / BYTES; };

template <int TYPE>
__device__ __forceinline__ float one_logit(const uint8_t* at) {
  if constexpr (TYPE == LOGITS_F32) return __ldg(reinterpret_cast<const float*>(at));
  const uint16_t x = __ldg(reinterpret_cast<const uint16_t*>(at));
  return TYPE == LOGITS_BF16 ? __uint_as_float((uint32_t)x << 16) : __half2float(__ushort_as_half(x));
}
template <int TYPE>
__device__ __forceinline__ void values(uint4 v, float (&x)[Logit<TYPE>::VEC]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (TYPE == LOGITS_F32) {
      x[i] = __uint_as_float(w[i]);
    } else if constexpr (TYPE == LOGITS_BF16) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    } else {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      x[2 * i] = f.x; x[2 * i + 1] = f.y;
    }
  }
}
// largest of a piece, NaN left out; every element at least `least` (twice, of the type; fp32: the number), NaN kept
template <int TYPE>
__device__ __forceinline__ float top_of(uint4 v) {
  if constexpr (TYPE == LOGITS_F32) return fmaxf(fmax3(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z)), __uint_as_float(v.w));
  if constexpr (TYPE == LOGITS_BF16) {
    auto b = [](uint32_t x) { return *reinterpret_cast<const __nv_bfloat162*>(&x); };
    const __nv_bfloat162 m = __hmax2(__hmax2(b(v.x), b(v.y)), __hmax2(b(v.z), b(v.w)));
    return fmaxf(__low2float(m), __high2float(m));
  } else {
    auto h = [](uint32_t x) { return *reinterpret_cast<const __half2*>(&x); };
    const __half2 m = __hmax2(__hmax2(h(v.x), h(v.y)), __hmax2(h(v.z), h(v.w)));
    return fmaxf(__low2float(m), __high2float(m));
  }
}
template <int TYPE>
__device__ __forceinline__ uint32_t raised(uint32_t x, uint32_t least) {
  uint32_t r;
  if constexpr (TYPE == LOGITS_F32) asm("max.NaN.f32 %0, %1, %2;" : "=f"(*reinterpret_cast<float*>(&r)) : "f"(__uint_as_float(x)), "f"(__uint_as_float(least)));
  else if constexpr (TYPE == LOGITS_BF16) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(least));
  else asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(least));
  return r;
}
template <int TYPE>
__device__ __forceinline__ uint32_t twice(float x) {
  if constexpr (TYPE == LOGITS_F32) return __float_as_uint(x);
  if constexpr (TYPE == LOGITS_BF16) return pack_bf16x2(x, x);
  const __half2 h = __float2half2_rn(x);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <int N>
__device__ __forceinline__ float max_of(const float (&x)[N]) {
  float m = fmaxf(x[0], x[1]);
#pragma unroll
  for (int i = 2; i < N; i += 2) m = fmax3(m, x[i], x[i + 1]);
  return m;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

__device__ __forceinline__ Key key_of(float x, int id) { return (Key)rank_key(x, false) << 32 | (uint32_t)~id; }
__device__ __forceinline__ float value_of(Key k) {
  const uint32_t u = (uint32_t)(k >> 32);
  return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}
__device__ __forceinline__ int id_of(Key k) { return (int)~(uint32_t)k; }
__device__ __forceinline__ Key larger(Key a, Key b) { return a > b ? a : b; }
__device__ __forceinline__ Key smaller(Key a, Key b) { return a > b ? b : a; }

// Lists: lane l has the l-th largest.
__device__ __forceinline__ Key merged(Key x, Key reversed, int lane) {
  x = larger(x, reversed);
#pragma unroll
  for (int j = 16; j > 0; j /= 2) {
    const Key y = __shfl_xor_sync(0xFFFFFFFFu, x, j);
    x = (lane & j) == 0 ? larger(x, y) : smaller(x, y);
  }
  return x;
}
__device__ __forceinline__ Key inserted(Key x, Key y, int lane) {
  const int at = __popc(__ballot_sync(0xFFFFFFFFu, x > y));
  const Key up = __shfl_up_sync(0xFFFFFFFFu, x, 1);
  return lane < at ? x : lane == at ? y : up;
}

struct Sums { float m, s, h; };                              // relative to m (a logit, finite or +inf or NaN)
// Sums of the lanes (0 and up of them: N, a power of two) to one, in all of these lanes.
template <int N>
__device__ __forceinline__ Sums joined(const Sums& a, float c) {
  Sums r = {a.m, 0.0f, 0.0f};
#pragma unroll
  for (int o = N / 2; o > 0; o /= 2) r.m = fmaxf(r.m, __shfl_xor_sync(0xFFFFFFFFu, r.m, o));
  if (a.s != 0.0f) {                                         // (0: nothing, or nothing but -inf)
    const float t = (a.m - r.m) * c, f = fast_exp2(t);
    r.s = t == t ? f * a.s : t;                              // (+inf less +inf)
    r.h = f > 0.0f ? f * fmaf(a.s, t, a.h) : 0.0f;
  }
#pragma unroll
  for (int o = N / 2; o > 0; o /= 2) {
    r.s += __shfl_xor_sync(0xFFFFFFFFu, r.s, o);
    r.h += __shfl_xor_sync(0xFFFFFFFFu, r.h, o);
  }
  return r;
}

constexpr int FOUND = 1024, RING = 3;
struct __align__(16) Shared {
  union {
    uint4 ring[RING][U][NT];
    struct {                                                 // after the stream
      Key list[8][32];
      Key found[FOUND];                                      // (first the groups' maxima)
      Key least;
      int winners, n_found;
      uint16_t winner[U * NT];
    };
  };
  Sums sums[8];
};
__device__ __forceinline__ void copy_async16(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
// how many of n different keys are larger
__device__ __forceinline__ int rank_among(const Key* keys, int n, Key own) {
  int r = 0;
#pragma unroll 4
  for (int i = 0; i + 1 < n; i += 2) {
    const ulonglong2 y = *reinterpret_cast<const ulonglong2*>(keys + i);
    r += (y.x > own) + (y.y > own);
  }
  if (n % 2) r += keys[n - 1] > own;
  return r;
}
__device__ __forceinline__ Key ld_cluster_key(uint32_t addr) {
  Key x;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(x) : "r"(addr) : "memory");
  return x;
}
__device__ __forceinline__ float ld_cluster_f32(uint32_t addr) {
  float x;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(addr) : "memory");
  return x;
}

// the eight lists of sh (a warp's own among them, in x) to one, in list[0] and warp 0's registers; the whole CTA calls
__device__ __forceinline__ Key merge_lists(Shared& sh, Key x, int n, int warp, int lane) {
  sh.list[warp][lane] = x;
  __syncthreads();
  for (int half = n / 2; half > 0; half /= 2) {
    if (warp < half) {
      x = merged(x, sh.list[warp + half][31 - lane], lane);
      sh.list[warp][lane] = x;
    }
    __syncthreads();
  }
  return x;
}

}  // namespace

template <int TYPE>
__global__ void __launch_bounds__(NT, CTAS) token_logprobs_kernel(const LogProb p, const int split) {
  constexpr int VEC = Logit<TYPE>::VEC, BYTES = Logit<TYPE>::BYTES;
  extern __shared__ __align__(16) uint8_t smem[];
  Shared& sh = *reinterpret_cast<Shared*>(smem);
  chain();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const long long row = blockIdx.x / split;
  const int rank = blockIdx.x % split;
  const float c = p.scale * 1.4426950408889634f;
  // 16-byte pieces of the row: piece j has elements j VEC - head ..; the first and the last may have neighbours' elements beside the row's
  const uint8_t* const first = static_cast<const uint8_t*>(p.logits) + row * p.stride * BYTES;
  const int head = (int)(reinterpret_cast<uintptr_t>(first) & 15u) / BYTES;
  const uint4* const pieces = reinterpret_cast<const uint4*>(first - head * BYTES);
  const int n = (p.V + head + VEC - 1) / VEC;
  const int lo = (int)((long long)n * rank / split), hi = (int)((long long)n * (rank + 1) / split);
  auto whole = [&](int j) { return j * VEC >= head && (long long)(j + 1) * VEC - head <= p.V; };
  auto there = [&](int j, int i) { return j * VEC + i >= head && j * VEC + i - head < p.V; };
  auto part = [&](int j) {                                   // a piece that has neighbours' elements beside the row's: -inf in their place
    uint32_t w[4] = {};
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      constexpr uint32_t NONE = TYPE == LOGITS_F32 ? 0xFF800000u : TYPE == LOGITS_BF16 ? 0xFF80u : 0xFC00u;
      const uint8_t* const e = reinterpret_cast<const uint8_t*>(pieces + j) + i * BYTES;
      if constexpr (BYTES == 4) w[i] = there(j, i) ? __ldg(reinterpret_cast<const uint32_t*>(e)) : NONE;
      else w[i / 2] |= (there(j, i) ? (uint32_t)__ldg(reinterpret_cast<const uint16_t*>(e)) : NONE) << (i % 2 * 16);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  };
  auto load = [&](int j, float (&x)[VEC]) { values<TYPE>(whole(j) ? __ldg(pieces + j) : part(j), x); };

  // the present reference: logit m, R, the logit that raises it, what a term is 0 at; low: m is next to the lowest or R too large, t = (x - m) c
  int token = -1;                                            // of warp 0: its logit is on its way while the row goes through
  float token_logit = 0.0f;
  if (warp == 0 && rank == 0 && p.logprob != nullptr) {
    token = __ldg(p.tokens + row);
    if (token >= 0 && token < p.V) token_logit = one_logit<TYPE>(first + (long long)token * BYTES);
  }
  Sums a = {-FLT_MAX, 0.0f, 0.0f};
  float R = 0.0f, limit = -FLT_MAX;
  uint32_t floor2 = 0;
  bool low = true;
  float best[U];
  int at[U];
#pragma unroll
  for (int u = 0; u < U; ++u) { best[u] = -INFINITY; at[u] = -1; }
  uint64_t s2 = 0, h2 = 0;
  const uint64_t c2 = pack_f32x2(c, c);
  constexpr float LOWEST = TYPE == LOGITS_F16 ? -65504.0f : -3.3895314e38f;
  auto raise = [&](float top) {
    const float R_new = top * c, below = fmaf(fabsf(top), -0.015625f, top - 150.0f / c);       // (under every rounding of itself to the type)
    const bool low_new = !(top > -1e30f && below > LOWEST && fabsf(R_new) < 2147483648.0f);       // (R is off by 64 at most: terms up to 2^64)
    const float t = low ? (a.m - top) * c : low_new ? -INFINITY : R - R_new, f = fast_exp2(t);
    float s0, s1, h0, h1;
    unpack_f32x2(s2, s0, s1);
    unpack_f32x2(h2, h0, h1);
    s2 = pack_f32x2(s0 * f, s1 * f);
    h2 = f > 0.0f ? pack_f32x2(f * fmaf(s0, t, h0), f * fmaf(s1, t, h1)) : 0;
    a.m = top;
    R = R_new;
    limit = top + 8.0f / c;
    low = low_new;
    floor2 = twice<TYPE>(below);
  };
  // U pieces at a time, one branch for all: a piece's own branches took a tenth of the instructions
  auto take = [&](const uint4 (&v)[U], int j) {
    float top[U], most;
#pragma unroll
    for (int u = 0; u < U; ++u) top[u] = top_of<TYPE>(v[u]);
    most = max_of(top);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (top[u] > best[u]) { best[u] = top[u]; at[u] = j + u * NT; }
    if (most > limit) raise(most);                           // rare after the first pieces
    if (!low) {
      const uint64_t r2 = pack_f32x2(-R, -R);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float x[VEC];
        values<TYPE>(make_uint4(raised<TYPE>(v[u].x, floor2), raised<TYPE>(v[u].y, floor2), raised<TYPE>(v[u].z, floor2), raised<TYPE>(v[u].w, floor2)), x);
#pragma unroll
        for (int i = 0; i < VEC; i += 2) {
          const uint64_t t2 = fma_f32x2(pack_f32x2(x[i], x[i + 1]), c2, r2);
          float t0, t1;
          unpack_f32x2(t2, t0, t1);
          const uint64_t e2 = pack_f32x2(fast_exp2(t0), fast_exp2(t1));
          s2 = add_f32x2(s2, e2);
          h2 = fma_f32x2(e2, t2, h2);
        }
      }
    } else {
#pragma unroll 1
      for (int u = 0; u < U; ++u) {
        float x[VEC];
        values<TYPE>(u == 0 ? v[0] : u == 1 ? v[1] : u == 2 ? v[2] : v[3], x);
#pragma unroll
        for (int i = 0; i < VEC; i += 2) {
          const float t0 = max_nan((x[i] - a.m) * c, -200.0f), t1 = max_nan((x[i + 1] - a.m) * c, -200.0f);
          const uint64_t e2 = pack_f32x2(fast_exp2(t0), fast_exp2(t1));
          s2 = add_f32x2(s2, e2);
          h2 = fma_f32x2(e2, pack_f32x2(t0, t1), h2);
        }
      }
    }
  };
  {
    // Piece lo + tid + i NT, of quarter i % U, U of them at a time through this thread's places of a ring in shared memory: three such groups are on their
    // way, or being taken, which keeps 190 KB of an SM in flight.
    const int from = lo + (lo < hi && !whole(lo) ? 1 : 0), to = hi - (lo < hi && hi - 1 > lo && !whole(hi - 1) ? 1 : 0);      // whole pieces
    const int groups = (hi - lo + U * NT - 1) / (U * NT);
    auto fetch = [&](int g) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int j = lo + tid + (g * U + u) * NT;
        if (j >= from && j < to) copy_async16(&sh.ring[g % RING][u][tid], pieces + j);
      }
      copy_async_commit();
    };
#pragma unroll
    for (int g = 0; g < RING; ++g) fetch(g);
    for (int g = 0; g < groups; ++g) {
      copy_async_wait<RING - 1>();
      const int j = lo + tid + g * (U * NT);
      uint4 v[U];
      if (j >= from && j + (U - 1) * NT < to) {
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = sh.ring[g % RING][u][tid];
      } else {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int k = j + u * NT;
          constexpr uint32_t NONE = TYPE == LOGITS_F32 ? 0xFF800000u : TYPE == LOGITS_BF16 ? 0xFF80FF80u : 0xFC00FC00u;
          v[u] = k >= from && k < to ? sh.ring[g % RING][u][tid] : k < hi ? part(k) : make_uint4(NONE, NONE, NONE, NONE);
        }
      }
      take(v, j);
      fetch(g + RING);
    }
  }
  {
    float s0, s1, h0, h1;
    unpack_f32x2(s2, s0, s1);
    unpack_f32x2(h2, h0, h1);
    a.s = s0 + s1;
    a.h = h0 + h1;
    if (!low) {                                              // from R to m c
      const float off = fmaf(a.m, c, -R), f = exp2f(-off);
      a.h = f * fmaf(-off, a.s, a.h);
      a.s *= f;
    }
  }
  a = joined<32>(a, c);
  if (lane == 0) sh.sums[warp] = a;

  Key x = 0;
  if (p.top > 0) {
    copy_async_wait<0>();
    __syncthreads();                                         // the ring's place is free
    Key mine[U], group = 0;                                  // of the quarters' maxima; 0: an empty one
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = lo + tid + u * NT;                       // (nothing but -inf: its first piece)
      mine[u] = j >= hi ? 0 : (Key)rank_key(best[u], false) << 32 | (uint32_t)~(at[u] < 0 ? j : at[u]);
      group = larger(group, mine[u]);
    }
    group = larger(group, __shfl_xor_sync(0xFFFFFFFFu, group, 1));
    group = larger(group, __shfl_xor_sync(0xFFFFFFFFu, group, 2));
    if (lane % 4 == 0) sh.found[tid / 4] = group;
    if (tid == 0) { sh.least = 0; sh.winners = sh.n_found = 0; }
    __syncthreads();
    if (tid < NT / 4) {
      const Key own = sh.found[tid];
      if (own != 0 && rank_among(sh.found, NT / 4, own) == p.top - 1) sh.least = own;     // (fewer groups than that: everything is looked at)
    }
    __syncthreads();
    const Key least = sh.least;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (mine[u] != 0 && mine[u] >= least) sh.winner[atomicAdd(&sh.winners, 1)] = (uint16_t)(tid + u * NT);
    if (warp == 0) sh.list[0][lane] = 0;
    __syncthreads();
    // What these quarters hold that is not below `least`, by pieces, half a warp each.  In no order; the counting below puts it into one.
    const int winners = sh.winners;
    for (int k = 2 * warp + lane / 16; k < winners; k += 2 * WARPS) {
      for (int j = lo + sh.winner[k] + lane % 16 * (U * NT); j < hi; j += 16 * U * NT) {
        float y[VEC];
        load(j, y);
        if (((Key)rank_key(max_of(y), false) << 32 | (uint32_t)~j) < least) continue;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          if (there(j, i) && ((Key)rank_key(y[i], false) << 32 | (uint32_t)~j) >= least) {
            const int n = atomicAdd(&sh.n_found, 1);
            if (n < FOUND) sh.found[n] = key_of(y[i], j * VEC + i - head);
          }
        }
      }
    }
    __syncthreads();
    const int n_found = sh.n_found;
    if (n_found <= FOUND) {
      for (int i = tid; i < n_found; i += NT) {
        const Key own = sh.found[i];
        const int r = rank_among(sh.found, n_found, own);
        if (r < 32) sh.list[0][r] = own;
      }
      __syncthreads();
      if (warp == 0) x = sh.list[0][lane];
    } else {
      // far more of them than there is room for: each warp keeps a list of the largest of its part of the row's
      for (int k = warp; k < winners; k += WARPS) {
        for (int j0 = lo + sh.winner[k]; j0 < hi; j0 += 32 * U * NT) {
          const int j = j0 + lane * (U * NT);
          float y[VEC];
          if (j < hi) load(j, y);
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            const Key one = j < hi && there(j, i) ? key_of(y[i], j * VEC + i - head) : 0;
            unsigned some = __ballot_sync(0xFFFFFFFFu, one > __shfl_sync(0xFFFFFFFFu, x, 31));
            while (some) {
              const int from = __ffs(some) - 1;
              some &= some - 1;
              x = inserted(x, __shfl_sync(0xFFFFFFFFu, one, from), lane);
            }
          }
        }
      }
      x = merge_lists(sh, x, WARPS, warp, lane);
    }
  } else {
    __syncthreads();
  }
  if (warp == 0) a = joined<WARPS>(sh.sums[lane % WARPS], c);
  if (split > 1) {
    // the other CTAs' lists and sums, a warp each
    if (tid == 0) sh.sums[0] = a;
    cluster_sync_all();
    if (rank == 0) {
      Key y = 0;
      Sums b = {-FLT_MAX, 0.0f, 0.0f};
      if (warp < split) {
        if (p.top > 0) y = ld_cluster_key(map_to_cta(&sh.list[0][lane], warp));
        b = {ld_cluster_f32(map_to_cta(&sh.sums[0].m, warp)), ld_cluster_f32(map_to_cta(&sh.sums[0].s, warp)), ld_cluster_f32(map_to_cta(&sh.sums[0].h, warp))};
      }
      __syncthreads();
      if (lane == 0) sh.sums[warp] = b;
      x = merge_lists(sh, y, split, warp, lane);
      if (warp == 0) a = joined<WARPS>(sh.sums[lane % WARPS], c);        // (warps behind the last CTA left nothing)
    }
    cluster_sync_all();                                      // no CTA exits while another may read its shared memory
    if (rank != 0) return;
  }
  if (warp != 0) return;
  // nothing but -inf: every log probability is -inf and the entropy 0; a NaN or +inf: no number, no tokens
  const bool none = a.s == 0.0f, odd = !(a.s < INFINITY);
  const float ln_s = none ? 0.0f : odd ? __int_as_float(0x7FC00000) : logf(a.s);
  // (by halves: the difference of two logits may be more than the largest number)
  auto logprob = [&](float y) { return none ? -INFINITY : fmaf(0.5f * y - 0.5f * a.m, 2.0f * p.scale, -ln_s); };
  if (lane == 0) {
    if (p.logprob != nullptr) p.logprob[row] = token < 0 ? 0.0f : token >= p.V ? __int_as_float(0x7FC00000) : logprob(token_logit);
    if (p.entropy != nullptr) p.entropy[row] = none ? 0.0f : ln_s - 0.6931471805599453f * (a.h / a.s);
  }
  if (lane < p.top) {
    p.top_id[row * p.top + lane] = odd ? -1 : id_of(x);
    p.top_logprob[row * p.top + lane] = odd ? __int_as_float(0x7FC00000) : logprob(value_of(x));
  }
}

// sums over groups of rows, in an order that does not change: a warp each
__global__ void __launch_bounds__(128) group_nll_kernel(const float* logprob, int groups, int group, float* nll) {
  chain();
  const int g = blockIdx.x * 4 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (g >= groups) return;
  float s = 0.0f;
  for (int i = lane; i < group; i += 32) s += logprob[(long long)g * group + i];
#pragma unroll
  for (int o = 16; o > 0; o /= 2) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  if (lane == 0) nll[g] = -s;
}

namespace {
template <int TYPE>
cudaError_t logprobs_t(const LogProb& p, int split, int sm_count, cudaStream_t st) {
  static_assert(CTAS * (sizeof(Shared) + 1024) <= 233472, "CTAs per SM");
  const long long ctas = (long long)p.N * split, each = (ctas + sm_count - 1) / sm_count;
  // Two or three CTAs an SM: no SM takes more.  CTAs that start while the kernel ahead still runs would go where there is room, four to some SMs and none to
  // others.  Measured, 276 / 300 / 400 rows of 50001 in fp16, one call behind the other, 12.1 / 15.3 / 16.0 us against 15.0 / 18.3 / 19.1 with room for four everywhere.
  const size_t smem = each == 2 || each == 3 ? 233472 / (size_t)each - 1024 : sizeof(Shared);
  constexpr int MOST = 233472 / 2 - 1024;                    // one number for all calls: another thread's call may come between this line and the launch
  if (cudaError_t e = cudaFuncSetAttribute(token_logprobs_kernel<TYPE>, cudaFuncAttributeMaxDynamicSharedMemorySize, MOST); e != cudaSuccess) return e;
  return launch_chained(token_logprobs_kernel<TYPE>, dim3((unsigned)ctas), dim3(NT), smem, st, split, p, split);
}
}  // namespace

cudaError_t launch_token_logprobs(const LogProb& p, int type, int sm_count, cudaStream_t st) {
  // Parts of a row: as many as leave each its SM and 6000 logits.  Measured, us, 1 / 2 / 4 / 8 parts: one row of 128256 in bf16, top 8, 13.5 / 10.9 / 9.0 / 8.4, 32 rows
  // 13.7 / 11.1 / 10.2 / 10.7, 64 13.8 / 11.3 / 11.6 / 13.5, 148 14.8 / 15.8 / 23.0 / 31.5; one row of 8000 6.3 / 7.5 / 8.0 / 8.2, 64 of 50001 in fp16 9.9 / 9.7 / 10.2 / 11.9.
  int split = 1;
  while (split < 8 && (long long)p.N * split * 2 <= sm_count && p.V / (2 * split) >= 6000) split *= 2;
  cudaError_t e = type == LOGITS_F32    ? logprobs_t<LOGITS_F32>(p, split, sm_count, st)
                  : type == LOGITS_BF16 ? logprobs_t<LOGITS_BF16>(p, split, sm_count, st)
                                        : logprobs_t<LOGITS_F16>(p, split, sm_count, st);
  if (e != cudaSuccess || p.nll == nullptr) return e;
  const int groups = p.N / p.group;
  return launch_chained(group_nll_kernel, dim3((unsigned)((groups + 3) / 4)), dim3(128), 0, st, 1, (const float*)p.logprob, groups, p.group, p.nll);
}

}  // namespace pc
