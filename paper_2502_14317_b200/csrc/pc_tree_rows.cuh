// Parts of the attention of drafted tokens over pages that its kernels share: the rotated queries, lengths, pages that are none, values that are no number.
#pragma once
#include "pc_cache_rows.cuh"
#include "pc_kv8.cuh"
#include "pc_tree.cuh"
#include <climits>

namespace pc {

// entries of a sequence with its w new tokens: 0 where there is no such sequence, -1 where its length is not one (beyond max_len or the table)
__device__ __forceinline__ int tree_entries(const TreePhase& t, int w, int len) {
  if (len < 0) return 0;
  return len > t.max_len || (long long)len + w > (long long)t.pages.n_table * t.pages.page ? -1 : len + w;
}
// A page that is none is read behind the pool's end: the copy has zeros there.
__device__ __forceinline__ int page_checked(const Pages& p, int id, int* status) {
  if (id >= 0 && id < p.n_pages) return id;
  if (status) atomicCAS(status, 0, 421);
  return p.n_pages;
}

// A row turned by the angles of its pairs: lane l has the elements E l .. E l + E - 1, lanes l and l + 16 those of the same pairs.
template <int D>
__device__ __forceinline__ void turn_row(uint32_t (&x)[D / 64], const float (&c)[D / 32], const float (&s)[D / 32], int lane) {
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    const uint32_t y = __shfl_xor_sync(0xFFFFFFFFu, x[i], 16);     // the other elements of the pairs
    float z[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float u = __uint_as_float(e ? x[i] & 0xFFFF0000u : x[i] << 16), v = __uint_as_float(e ? y & 0xFFFF0000u : y << 16);
      const float sn = lane < 16 ? -s[2 * i + e] : s[2 * i + e];   // x cos - y sin, y cos + x sin
      z[e] = fmaf(v, sn, u * c[2 * i + e]);
    }
    x[i] = pack_bf16x2(z[0], z[1]);
  }
}

// Queries as rows, as RowTurner makes them, with the angles of pc_tree.cuh.  A warp has a row, a lane D / 32 elements.
template <int D>
struct TreeTurner {
  static constexpr int E = D / 32, H = E / 2;
  double per[H];
  float c[E], s[E];
  long long pos = 0, held = LLONG_MIN;                        // position of the row that comes, and whose angles are held (no position is LLONG_MIN)
  bool turn;
  __device__ __forceinline__ TreeTurner(const TreePhase& t, int lane) : turn(t.turn != 0) {
#pragma unroll
    for (int k = 0; k < H; ++k) per[k] = part_of_turn(t.turns, E * (lane & 15) + (lane >> 4) * H + k);
  }
  // sequence, its entries before the new tokens, how many of these the row's token sees
  __device__ __forceinline__ void place(const CacheRows& p, int seq, int entries, int sees) {
    pos = (long long)p.pos0 + (p.pos ? __ldg(p.pos + seq) : entries) + (sees > 0 ? sees - 1 : 0);
  }
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
    if (in_memory || !turn) return;
    if (pos != held) {
      held = pos;
#pragma unroll
      for (int k = 0; k < H; ++k) {                            // lanes l and l + 16 hold elements of the same E pairs and compute half of them each
        const float2 a = turned(per[k], pos);
        const float2 b = make_float2(__shfl_xor_sync(0xFFFFFFFFu, a.x, 16), __shfl_xor_sync(0xFFFFFFFFu, a.y, 16));
        c[k] = lane < 16 ? a.x : b.x; s[k] = lane < 16 ? a.y : b.y;
        c[H + k] = lane < 16 ? b.x : a.x; s[H + k] = lane < 16 ? b.y : a.y;
      }
    }
    turn_row<D>(x, c, s, lane);
  }
  static __device__ __forceinline__ void store(void* rows, size_t at, int lane, const uint32_t (&x)[E / 2]) { RowTurner<D>::store(rows, at, lane, x); }
};

// ones in the places of the word's values (two of bf16, four of e4m3) that are numbers
template <int FMT>
__device__ __forceinline__ uint32_t finite_parts(uint32_t x) {
  uint32_t r = 0xFFFFFFFFu;
  if constexpr (FMT == FMT_BF16) {
    if ((x & 0x7F80u) == 0x7F80u) r &= 0xFFFF0000u;
    if ((x & 0x7F800000u) == 0x7F800000u) r &= 0x0000FFFFu;
  } else if constexpr (FMT == FMT_E4M3) {
#pragma unroll
    for (int i = 0; i < 32; i += 8)
      if ((x >> i & 0x7Fu) == 0x7Fu) r &= ~(0xFFu << i);
  }
  return r;
}

// What the kernels have left out of a row's sum: values that are no number of the new tokens in `odd` that the row sees, columns col .. col + N - 1 of
// kv-head hkv.  Their weight is positive, so that an infinity stays one.  Next to never; not unrolled.
template <int D, int FMT, int N>
__device__ __forceinline__ void add_odd(const TreePhase& t, const CachePhase& p, int hkv, int seq, int entries, unsigned long long odd, int col, float* o) {
#pragma unroll 1
  while (odd) {
    const int e = entries + __ffsll((long long)odd) - 1, which = page_of(t.pages, e), id = __ldg(t.pages.table + seq * t.pages.stride + which);
    odd &= odd - 1;
    if (id < 0 || id >= t.pages.n_pages) continue;
    const size_t row = ((size_t)id * p.Hkv + hkv) * t.pages.page + (e - which * t.pages.page);
#pragma unroll 1
    for (int i = 0; i < N; ++i) {
      float x;
      if constexpr (FMT == FMT_BF16) {
        x = __uint_as_float((uint32_t)__ldg(reinterpret_cast<const uint16_t*>(t.v) + row * D + col + i) << 16);
      } else {
        const uint32_t h = codes_to_half2<FMT, 0>(flip_signs<FMT>(__ldg(t.v + row * D + col + i)));
        x = __half2float(__ushort_as_half((unsigned short)(h & 0xFFFFu))) * __ldg(p.v_scale + row);
      }
      if (!(fabsf(x) < INFINITY)) o[i] += x;
    }
  }
}

}  // namespace pc
