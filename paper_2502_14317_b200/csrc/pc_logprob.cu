// Log probabilities of given tokens, entropy and the most probable tokens of rows of logits (pc_token_logprobs).
//
// One pass over a row x of V logits.  A thread keeps, over its share, a reference maximum m and with c = scale * log2 e, t = (x - m) c, the sums
//     s = sum 2^t,      h = sum 2^t t,
// and raises m (s and h to be taken along) only where a logit exceeds it by more than 2^8.  With M the largest m, all joined,
//     log p(x) = (x - M) scale - ln s,      H = ln s - ln 2 h / s.
// x - m comes before the factor, so that rows of the type's lowest value do not overflow.
//
// The top k: a thread also keeps the largest logit of its share and where it stood.  Only the shares with the k largest of these maxima can hold one of
// the k largest logits, and only logits not below the k-th of them can be one: those k shares, a few 16-byte pieces each, are read once more (from
// L2) and everything else is left alone.  Keys are (order of the value, lowest index first), 64 bits, all different, so ties
// need no rule of their own.  Lists of 32 keys are a warp's registers: sorted, merged (largest against smallest), and inserted into.
//
// A row is the work of a cluster of 1 to 8 CTAs: as many as one round of the grid has room for.
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
__device__ __forceinline__ uint4 ld_stream(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
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
__device__ __forceinline__ Key sorted(Key x, int lane) {
#pragma unroll
  for (int k = 2; k <= 32; k *= 2)
#pragma unroll
    for (int j = k / 2; j > 0; j /= 2) {
      const Key y = __shfl_xor_sync(0xFFFFFFFFu, x, j);
      x = ((lane & j) == 0) == ((lane & k) == 0) ? larger(x, y) : smaller(x, y);
    }
  return x;
}
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
__device__ __forceinline__ Sums joined(const Sums& a, const Sums& b, float c) {
  Sums r = {fmaxf(a.m, b.m), 0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const Sums& x = i ? b : a;
    if (x.s == 0.0f) continue;                               // (nothing, or nothing but -inf)
    const float t = (x.m - r.m) * c, f = fast_exp2(t);
    r.s = fmaf(f, x.s, r.s);
    r.h = fmaf(f, f > 0.0f ? fmaf(x.s, t, x.h) : 0.0f, r.h);
    if (t != t) r.s = r.h = t;
  }
  return r;
}
__device__ __forceinline__ Sums shuffled(const Sums& a, int o) {
  return {__shfl_xor_sync(0xFFFFFFFFu, a.m, o), __shfl_xor_sync(0xFFFFFFFFu, a.s, o), __shfl_xor_sync(0xFFFFFFFFu, a.h, o)};
}

struct __align__(16) Shared {
  Key list[8][32];
  Sums sums[8];
};
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
  __shared__ Shared sh;
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
  auto load = [&](int j, float (&x)[VEC]) {                  // -inf in the place of elements that are not the row's
    if (whole(j)) { values<TYPE>(__ldg(pieces + j), x); return; }
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[i] = there(j, i) ? one_logit<TYPE>(reinterpret_cast<const uint8_t*>(pieces + j) + i * BYTES) : -INFINITY;
  };

  Sums a = {-FLT_MAX, 0.0f, 0.0f};
  float best = -INFINITY;
  int at = -1;
  uint64_t s2 = 0, h2 = 0;
  const uint64_t c2 = pack_f32x2(c, c);
  auto take = [&](const float (&x)[VEC], int j) {
    const float top = max_of(x);
    if (top > best || at < 0) { best = top; at = j; }
    if ((top - a.m) * c > 8.0f) {                            // rare after the first pieces
      const float t = (a.m - top) * c, f = fast_exp2(t);
      float s0, s1, h0, h1;
      unpack_f32x2(s2, s0, s1);
      unpack_f32x2(h2, h0, h1);
      s2 = pack_f32x2(s0 * f, s1 * f);
      h2 = f > 0.0f ? pack_f32x2(f * fmaf(s0, t, h0), f * fmaf(s1, t, h1)) : 0;
      a.m = top;
    }
    const uint64_t m2 = pack_f32x2(-a.m, -a.m);
#pragma unroll
    for (int i = 0; i < VEC; i += 2) {
      float t0, t1;
      unpack_f32x2(mul_f32x2(add_f32x2(pack_f32x2(x[i], x[i + 1]), m2), c2), t0, t1);
      t0 = max_nan(t0, -200.0f); t1 = max_nan(t1, -200.0f);   // 2^-200 is 0, and 0 times it a number
      const uint64_t e2 = pack_f32x2(fast_exp2(t0), fast_exp2(t1));
      s2 = add_f32x2(s2, e2);
      h2 = fma_f32x2(e2, pack_f32x2(t0, t1), h2);
    }
  };
  {
    const int from = lo + (lo < hi && !whole(lo) ? 1 : 0), to = hi - (lo < hi && hi - 1 > lo && !whole(hi - 1) ? 1 : 0);      // whole pieces
    int j = lo + tid;
    if (j < from) j += NT;
    for (; j + (U - 1) * NT < to; j += U * NT) {
      uint4 v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = ld_stream(pieces + j + u * NT);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float x[VEC];
        values<TYPE>(v[u], x);
        take(x, j + u * NT);
      }
    }
    for (; j < to; j += NT) {
      float x[VEC];
      values<TYPE>(ld_stream(pieces + j), x);
      take(x, j);
    }
    if (lo < hi && tid == 0 && from > lo) {                  // (the first piece: of its elements none is preferred to an equal one behind it)
      float x[VEC];
      load(lo, x);
      const float was = best;
      const int stood = at;
      take(x, lo);
      if (stood >= 0 && max_of(x) == was) at = lo;
    }
    if (to < hi && tid == (hi - 1 - lo) % NT) {
      float x[VEC];
      load(hi - 1, x);
      take(x, hi - 1);
    }
  }
  {
    float s0, s1, h0, h1;
    unpack_f32x2(s2, s0, s1);
    unpack_f32x2(h2, h0, h1);
    a.s = s0 + s1;
    a.h = h0 + h1;
  }
#pragma unroll
  for (int o = 16; o > 0; o /= 2) a = joined(a, shuffled(a, o), c);
  if (lane == 0) sh.sums[warp] = a;

  Key x = 0;
  if (p.top > 0) {
    // the shares' maxima, the k largest of them, and what these shares hold that is not below the last of them
    if (at >= 0) {
      float y[VEC];
      load(at, y);
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        if (there(at, i)) x = larger(x, key_of(y[i], at * VEC + i - head));
    }
    merge_lists(sh, sorted(x, lane), WARPS, warp, lane);
    const Key winner = sh.list[0][lane], least = sh.list[0][p.top - 1];
    __syncthreads();
    x = 0;
    for (int k = warp; k < p.top; k += WARPS) {
      const Key w = __shfl_sync(0xFFFFFFFFu, winner, k);
      if (w == 0) break;
      const int share = ((id_of(w) + head) / VEC - lo) % NT;
      for (int j0 = lo + share; j0 < hi; j0 += 32 * NT) {
        const int j = j0 + lane * NT;
        float y[VEC];
        if (j < hi) load(j, y);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const Key mine = j < hi && there(j, i) ? key_of(y[i], j * VEC + i - head) : 0;
          unsigned some = __ballot_sync(0xFFFFFFFFu, mine != 0 && mine >= least);
          while (some) {
            const int from = __ffs(some) - 1;
            some &= some - 1;
            x = inserted(x, __shfl_sync(0xFFFFFFFFu, mine, from), lane);
          }
        }
      }
    }
    x = merge_lists(sh, x, WARPS, warp, lane);
  } else {
    __syncthreads();
  }
  if (warp == 0) {
    a = lane < WARPS ? sh.sums[lane] : Sums{-FLT_MAX, 0.0f, 0.0f};
#pragma unroll
    for (int o = 16; o > 0; o /= 2) a = joined(a, shuffled(a, o), c);
  }
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
      if (warp == 0) {
        a = lane < split ? sh.sums[lane] : Sums{-FLT_MAX, 0.0f, 0.0f};
#pragma unroll
        for (int o = 16; o > 0; o /= 2) a = joined(a, shuffled(a, o), c);
      }
    }
    cluster_sync_all();                                      // no CTA exits while another may read its shared memory
    if (rank != 0) return;
  }
  if (warp != 0) return;
  // nothing but -inf: every log probability is -inf and the entropy 0; a NaN or +inf: no number, no tokens
  const bool none = a.s == 0.0f, odd = !(a.s < INFINITY);
  const float ln_s = none ? 0.0f : odd ? __int_as_float(0x7FC00000) : logf(a.s);
  auto logprob = [&](float y) { return none ? -INFINITY : fmaf(y - a.m, p.scale, -ln_s); };
  if (lane == 0) {
    if (p.logprob != nullptr) {
      const int t = __ldg(p.tokens + row);
      p.logprob[row] = t < 0 ? 0.0f : t >= p.V ? __int_as_float(0x7FC00000) : logprob(one_logit<TYPE>(first + (long long)t * BYTES));
    }
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

cudaError_t launch_token_logprobs(const LogProb& p, int type, int sm_count, cudaStream_t st) {
  int split = 1;
  while (split < 8 && (long long)p.N * split * 2 <= (long long)CTAS * sm_count && p.V / (2 * split) >= 2 * NT) split *= 2;
  const dim3 grid((unsigned)((long long)p.N * split));
  cudaError_t e = type == LOGITS_F32    ? launch_chained(token_logprobs_kernel<LOGITS_F32>, grid, dim3(NT), 0, st, split, p, split)
                  : type == LOGITS_BF16 ? launch_chained(token_logprobs_kernel<LOGITS_BF16>, grid, dim3(NT), 0, st, split, p, split)
                                        : launch_chained(token_logprobs_kernel<LOGITS_F16>, grid, dim3(NT), 0, st, split, p, split);
  if (e != cudaSuccess || p.nll == nullptr) return e;
  const int groups = p.N / p.group;
  return launch_chained(group_nll_kernel, dim3((unsigned)((groups + 3) / 4)), dim3(128), 0, st, 1, (const float*)p.logprob, groups, p.group, p.nll);
}

}  // namespace pc
