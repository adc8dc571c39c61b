// The body of the kernels for many query rows: pc_cache_wide.cu (caches of pc_cache_attn) and pc_tree_wide.cu (pages, drafted tokens).  What it does
// and what bounds it: pc_cache_wide.cu.
#pragma once
#include "pc_cache.h"
#include "pc_flash.cuh"
#include "pc_kernels.h"
#include "pc_kv8.cuh"
#include "pc_tree_rows.cuh"
#include <type_traits>

namespace pc {
namespace wide {

using namespace flash;

// Ring and slots of the 8-bit builds: stages of a tile of K or V, of a pair 64 keys of K and 64 columns of V, as for bf16; raw slots of
// the codes of a stage.
template <int D_, bool PAIR_>
struct Cfg8 : Cfg<D_, PAIR_> {
  static constexpr bool WHOLE = D_ == 128 && !PAIR_;                          // stages of 32 KB
  static constexpr int NK = WHOLE ? 1 : 3, NV = WHOLE ? 2 : 3, NS = NK + NV, NQ = 2;
  static constexpr int RAW = PAIR_ ? 6 : 3, RAW_BYTES = TILE * D_ / (PAIR_ ? 2 : 1);
};
template <class C>
struct Off8 {
  static constexpr int Q = 0, RING = 2 * C::Q_BYTES, RAW = RING + C::NS * C::STAGE_BYTES, MISC = RAW + C::RAW * C::RAW_BYTES;
  static constexpr int EXTRA = MISC + (int)sizeof(Misc2);
};
// key_scale: a tile's scales stay until its softmax has read them.  The converter is at most NK + 2 tiles ahead of that: a key stage is
// free once the products of its tile have run, and those wait for the softmax to have read the logits before theirs.
struct __align__(16) Extra8 {
  uint64_t sc_full[8], raw_full[6], raw_free[6];
  float key_scale[8][TILE];
};
static_assert(Off8<Cfg8<128, false>>::EXTRA + sizeof(Extra8) <= 232448 && Off8<Cfg8<128, true>>::EXTRA + sizeof(Extra8) <= 232448,
              "shared memory of a CTA");

// TREE: the cache is pages, the last w of a sequence's entries are its new tokens, each of which sees its ancestors.
struct NoTree {};
template <class T>
constexpr bool is_tree() { return std::is_same<T, TreePhase>::value; }

struct Item { int seq, hkv, rg, split, keys, j0, n; };          // keys: entries of the sequence; n tiles from j0, 0: none
template <class T>
__device__ __forceinline__ Item decode_item(const WidePhase& p, [[maybe_unused]] const T& tr, int item) {
  Item it;
  it.split = item % p.c.n_split;
  int x = item / p.c.n_split;
  it.rg = x % p.c.n_rg;
  x /= p.c.n_rg;
  it.hkv = x % p.c.Hkv;
  it.seq = x / p.c.Hkv;
  it.keys = p.c.n_keys;
  if constexpr (is_tree<T>()) {
    it.keys = tree_entries(tr, p.c.q.w, __ldg(p.c.len + it.seq));
    if (it.keys < 0) { if (p.c.status) atomicCAS(p.c.status, 0, 422); it.keys = 0; }
  } else if (p.c.len != nullptr) {
    it.keys = max(0, min(it.keys, __ldg(p.c.len + it.seq)));
  }
  const int tiles = (it.keys + TILE - 1) / TILE;
  int n_split = p.c.n_split;
  if constexpr (is_tree<T>()) {                                 // short sequences in fewer pieces
    n_split = min(n_split, (tiles + tr.least_tiles - 1) / tr.least_tiles);
    if (it.split >= n_split) { it.j0 = it.n = 0; return it; }
  }
  it.j0 = (int)((long long)tiles * it.split / n_split);
  it.n = (int)((long long)tiles * (it.split + 1) / n_split) - it.j0;
  return it;
}

// TREE: barriers beside Misc2.  fix_go: the values of a tile with new tokens, or entries behind the last, have landed (bf16: what is no number there is taken out
// by the epilogue's warps); fix_done: they have.  odd: what each of these warps took out, of the present item and the one before.
struct __align__(16) ExtraTree {
  uint64_t fix_go, fix_done, odd_full;
  unsigned long long odd[2][4];
};
// TREE, 8 bits: of a tile's values log2 of the scales and their inverses (softmax_codes_tile), and for each of the converting warps' quarters of the tile whether a scale
// is not between 2^-40 and 2^40; they stay as long as the keys' scales.  sums: as lm of Misc2, [block][maximum / sum][row], weights_apart.
struct __align__(16) ExtraValues {
  float log2[8][TILE], inverse[8][TILE];
  uint8_t far[8][4];
  float sums[2][2][TILE];
};
constexpr float NEAR_VALUE = 0x1p40f;
template <class T>
__device__ __forceinline__ bool tail_tile(const T& tr, const WidePhase& p, int keys, int j) {       // whether tile j has new tokens or less than 128 entries
  if constexpr (is_tree<T>()) return (j + 1) * TILE > keys - p.c.q.w;
  return false;
}
// Boxes of 2^log_box entries that hold entries of tile j.
__device__ __forceinline__ int tile_boxes(const TreePhase& t, int keys, int j) {
  const int some = (keys - j * TILE + (1 << t.log_box) - 1) >> t.log_box, all = TILE >> t.log_box;
  return some < all ? some : all;
}
// Pages of a sequence's table, 64 at a time in a warp's registers, the second half on its way while the first is used.
struct PageIds {
  int ids, next, first;
  __device__ __forceinline__ int at(const TreePhase& t, const Item& it, int which, int lane) const {
    return which + lane <= page_of(t.pages, it.keys - 1) ? __ldg(t.pages.table + it.seq * t.pages.stride + which + lane) : -1;
  }
  __device__ __forceinline__ PageIds(const TreePhase& t, const Item& it, int lane) : first(page_of(t.pages, it.j0 * TILE)) {
    ids = at(t, it, first, lane);
    next = at(t, it, first + 32, lane);
  }
  __device__ __forceinline__ void reach(const TreePhase& t, const Item& it, int which, int lane) {        // no page before `which` is asked for again
    if (which - first < 32) return;
    first += 32;
    ids = next;
    next = at(t, it, first + 32, lane);
  }
  __device__ __forceinline__ int of(int which) const {                                                   // the whole warp calls
    const int i = which - first, x = __shfl_sync(0xFFFFFFFFu, ids, i & 31);
    if (!__any_sync(0xFFFFFFFFu, i >= 32)) return x;                                     // (does not wait for what is still on its way)
    const int y = __shfl_sync(0xFFFFFFFFu, next, i & 31);
    return i < 32 ? x : y;
  }
};

// f16 operands, fp32 accumulation
__host__ __device__ constexpr uint32_t make_idesc_f16_f32(int M, int N, bool b_mn_major = false) {
  return (1u << 4) | (static_cast<uint32_t>(b_mn_major) << 16) | (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}

// hooks of the softmax warps: columns times the scales of their keys (8-bit formats)
template <class C>
struct ScaledHooks : Hooks<C> {
  const float* scale;
  __device__ __forceinline__ ScaledHooks(const Ctx2& c, int b) : Hooks<C>(c, b), scale(nullptr) {}
  __device__ __forceinline__ void scale32(uint32_t (&c)[32], const float* s) const {
#pragma unroll
    for (int i = 0; i < 32; i += 4) {
      const float4 f = *reinterpret_cast<const float4*>(s + i);
      float a, b;
      unpack_f32x2(mul_f32x2(pack_f32x2(__uint_as_float(c[i]), __uint_as_float(c[i + 1])), pack_f32x2(f.x, f.y)), a, b);
      c[i] = __float_as_uint(a); c[i + 1] = __float_as_uint(b);
      unpack_f32x2(mul_f32x2(pack_f32x2(__uint_as_float(c[i + 2]), __uint_as_float(c[i + 3])), pack_f32x2(f.z, f.w)), a, b);
      c[i + 2] = __float_as_uint(a); c[i + 3] = __float_as_uint(b);
    }
  }
  __device__ __forceinline__ void scale_keys(uint32_t (&c0)[32], uint32_t (&c1)[32], uint32_t (&c2)[32], uint32_t (&c3)[32]) const {
    scale32(c0, scale); scale32(c1, scale + 32); scale32(c2, scale + 64); scale32(c3, scale + 96);
  }
};

// Columns that a row sees of a tile with new tokens, a bit each: those before column `first`, and column first + k if bit k of `sees` is set.
__device__ __forceinline__ uint32_t columns_seen(unsigned long long sees, int first, int col) {
  const int at = col - first;                                    // of sees, at column col
  return at >= 64 ? 0u : at >= 0 ? (uint32_t)(sees >> at) : at <= -32 ? 0xFFFFFFFFu : ((uint32_t)sees << -at) | ((1u << -at) - 1u);
}
template <class Base>
struct TreeHooks : Base {
  uint32_t seen[4];
  bool tail;
  template <class... A>
  __device__ __forceinline__ explicit TreeHooks(const A&... a) : Base(a...), tail(false) {}
  __device__ __forceinline__ void mask(uint32_t (&c)[32], uint32_t bits) const {
#pragma unroll
    for (int i = 0; i < 32; ++i)
      if (!(bits & (1u << i))) c[i] = 0xFF800000u;
  }
  __device__ __forceinline__ void scale_keys(uint32_t (&c0)[32], uint32_t (&c1)[32], uint32_t (&c2)[32], uint32_t (&c3)[32]) const { hide(c0, c1, c2, c3); }
  __device__ __forceinline__ void hide(uint32_t (&c0)[32], uint32_t (&c1)[32], uint32_t (&c2)[32], uint32_t (&c3)[32]) const {
    if (tail) { mask(c0, seen[0]); mask(c1, seen[1]); mask(c2, seen[2]); mask(c3, seen[3]); }
  }
};

// One tile over 8-bit codes, for TREE: the keys' codes are exact operands, and the values' are too, because their scales go into the logits.  With z
// the logit of a key in log2 units and v the scale of its value, z' = z + log2 v,
//     O = sum 2^(z' - m) code,      l = sum 2^(z' - m) / v,
// where m is a reference for z': what is held to its range is the weight that a code has, so that probabilities can be halves (11 bits; rounded to bf16 beside
// values rounded to bf16 the largest error against 64 bits was 2.8e-3 where that of fp32 probabilities was 1.7e-3, now 1.9e-3), and the conversion of values is that of keys.
template <int D, class Hooks>
__device__ __forceinline__ void softmax_codes_tile(uint32_t s_taddr, uint32_t p_taddr, uint32_t o_taddr, bool first_tile, float scale_log2, RowState& st,
                                                   const Hooks& hk, const float* key_scale, const float* value_log2, const float* value_inverse) {
  uint32_t c[4][32];
#pragma unroll
  for (int i = 0; i < 4; ++i) tmem_ld32(s_taddr + 32 * i, c[i]);
  tmem_wait_ld();
#pragma unroll
  for (int i = 0; i < 4; ++i) loaded(c[i]);
  hk.on_read();
  const uint64_t scale2 = dup2(scale_log2);
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 32; j += 4) {
      const float4 f = *reinterpret_cast<const float4*>(key_scale + 32 * i + j), g = *reinterpret_cast<const float4*>(value_log2 + 32 * i + j);
      float a, b;
      unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(c[i][j]), __uint_as_float(c[i][j + 1])), mul_f32x2(pack_f32x2(f.x, f.y), scale2), pack_f32x2(g.x, g.y)), a, b);
      c[i][j] = __float_as_uint(a); c[i][j + 1] = __float_as_uint(b);
      unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(c[i][j + 2]), __uint_as_float(c[i][j + 3])), mul_f32x2(pack_f32x2(f.z, f.w), scale2), pack_f32x2(g.z, g.w)), a, b);
      c[i][j + 2] = __float_as_uint(a); c[i][j + 3] = __float_as_uint(b);
    }
  hk.hide(c[0], c[1], c[2], c[3]);
  const float mx = fmaxf(fmaxf(max32(c[0]), max32(c[1])), fmaxf(max32(c[2]), max32(c[3])));
  hk.before_p();
  const bool raise = first_tile || mx > st.m + LAZY_RESCALE_LOG2;
  if (__any_sync(0xFFFFFFFFu, raise)) {                            // rare; warp-uniform: each warp owns its 32 lanes of O
    float alpha = 1.0f;
    if (raise) {
      const float m_new = fmaxf(st.m, mx);
      alpha = (st.m == -INFINITY) ? 0.0f : fast_exp2(st.m - m_new);
      st.m = m_new;
      st.l *= alpha;
    }
    if (!first_tile) rescale_rows<D>(o_taddr, alpha);
  }
  const uint64_t negm2 = dup2(st.m == -INFINITY ? 0.0f : -st.m);
  uint64_t sum2[2] = {0ull, 0ull};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t pk[16];
#pragma unroll
    for (int j = 0; j < 32; j += 4) {
      const float4 g = *reinterpret_cast<const float4*>(value_inverse + 32 * i + j);
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        float x0, x1;
        unpack_f32x2(add_f32x2(pack_f32x2(__uint_as_float(c[i][j + e]), __uint_as_float(c[i][j + e + 1])), negm2), x0, x1);
        const float p0 = fast_exp2(x0), p1 = fast_exp2(x1);
        sum2[e / 2] = fma_f32x2(pack_f32x2(p0, p1), e ? pack_f32x2(g.z, g.w) : pack_f32x2(g.x, g.y), sum2[e / 2]);
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(pk[(j + e) / 2]) : "f"(p1), "f"(p0));
      }
    }
    tmem_st16(p_taddr + 16 * i, pk);
    if (i == 1) { tmem_wait_st(); hk.on_half(); }
  }
  tmem_wait_st();
  hk.on_full();
  float a0, a1;
  unpack_f32x2(add_f32x2(sum2[0], sum2[1]), a0, a1);
  st.l += a0 + a1;
}
// The weights of a tile's keys by themselves, from z and relative to their own maximum.  2^(z' - m) is 0 below 2^-126, and with it the weight of a key whose value is that
// much smaller than another's, or zeros.  While all scales are between 2^-40 and 2^40 those are weights below 2^-46 of the row's; from an item's first tile with another
// scale on a row is summed here, by another 128 exponentials (16 tokens of 16 sequences of up to 12000 int8 entries, 32/8 heads of 128: 163 us, with a row of zeros in four 219).
static __device__ __noinline__ float2 weights_apart(uint32_t s_taddr, float scale_log2, float m, float l, const float* key_scale, bool tail, uint4 seen) {
#pragma unroll 1
  for (int i = 0; i < 4; ++i) {
    uint32_t c[32];
    tmem_ld32(s_taddr + 32 * i, c);
    tmem_wait_ld();
    loaded(c);
    const uint32_t bits = !tail ? 0xFFFFFFFFu : i == 0 ? seen.x : i == 1 ? seen.y : i == 2 ? seen.z : seen.w;
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      const float z = __uint_as_float(c[j]) * (key_scale[32 * i + j] * scale_log2);
      c[j] = bits >> j & 1 ? __float_as_uint(z) : 0xFF800000u;
    }
    const float top = fmaxf(m, max32(c)), base = top == -INFINITY ? 0.0f : top;
    l = m == -INFINITY ? 0.0f : l * fast_exp2(m - base);
#pragma unroll
    for (int j = 0; j < 32; ++j) l += fast_exp2(__uint_as_float(c[j]) - base);
    m = top;
  }
  return make_float2(m, l);
}

// Halves (keys or values of a tile) of an item's n tiles in the order in which the issuers want them: K of the first `lag` tiles, then
// V of tile t, K of tile t + lag.
__device__ __forceinline__ void half_of(int h, int n, int lag, bool& values, int& t) {
  if (lag > n) lag = n;
  if (h < lag) { values = false; t = h; return; }
  h -= lag;
  const int both = n - lag;                                // tiles whose V is followed by a K
  if (h < 2 * both) { values = (h & 1) == 0; t = (h >> 1) + (values ? 0 : lag); }
  else { values = true; t = both + (h - 2 * both); }
}

// The epilogue's warps between the raw slots and the ring; a warp has a quarter of a stage's rows.
template <class C, int FMT, class T>
struct Converter {
  static constexpr int D = C::D;
  const Ctx2& cx;
  const WidePhase& prm;
  Extra8& ex;
  uint8_t* raw;
  int warp, lane;
  uint32_t k = 0, v = 0, raws = 0, tile = 0;               // uses of the stages and of the slots; tiles of earlier items
  const T& tr;
  ExtraValues* values;                                     // TREE
  unsigned long long odd = 0;                              // TREE: new tokens of the present item with a value that is no number, of this lane's
  __device__ __forceinline__ Converter(const Ctx2& c, const WidePhase& p, Extra8& e, uint8_t* raw_smem, int w, int l, const T& t, ExtraValues* values_)
      : cx(c), prm(p), ex(e), raw(raw_smem), warp(w), lane(l), tr(t), values(values_) {}

  // scale of key warp * 32 + lane of the tile, 0 behind the last entry
  __device__ __forceinline__ float scale_of(const Item& it, int h, int lag) const {
    bool values;
    int t;
    half_of(h, it.n, lag, values, t);
    const int key = (it.j0 + t) * TILE + warp * 32 + lane;
    return key < it.keys ? __ldg((values ? prm.c.v_scale : prm.c.k_scale) + ((size_t)it.seq * prm.c.Hkv + it.hkv) * prm.c.capacity + key) : 0.0f;
  }
  // TREE: key warp * 32 + lane of tile t: its page (-1: none), and with that the scales of the key and its value
  __device__ __forceinline__ int page_of_key(const Item& it, int t) const {
    if constexpr (is_tree<T>()) {
      const int key = (it.j0 + t) * TILE + warp * 32 + lane;
      if (t < it.n && key < it.keys) return __ldg(tr.pages.table + it.seq * tr.pages.stride + page_of(tr.pages, key));
    }
    return -1;
  }
  __device__ __forceinline__ float2 scales_in(const Item& it, int t, int id) const {
    if constexpr (is_tree<T>()) {
      if (id >= 0 && id < tr.pages.n_pages) {
        const int key = (it.j0 + t) * TILE + warp * 32 + lane;
        const size_t at = ((size_t)id * prm.c.Hkv + it.hkv) * tr.pages.page + (key - page_of(tr.pages, key) * tr.pages.page);
        return make_float2(__ldg(prm.c.k_scale + at), __ldg(prm.c.v_scale + at));
      }
    }
    return make_float2(0.0f, 0.0f);
  }
  template <bool VALUES>
  __device__ __forceinline__ bool convert(int t, float scale, int valid, [[maybe_unused]] int mine = 0, [[maybe_unused]] float value_scale = 0.0f) {       // valid: rows of the tile that are entries; TREE: from mine on new tokens
    Misc2& mi = *cx.mi;
    uint32_t& n = VALUES ? v : k;
    constexpr int FIRST = VALUES ? C::NK : 0, STAGES = VALUES ? C::NV : C::NK;
    // rows of a stage and their bytes as codes; the steps in which a warp goes through its rows
    constexpr int ROWS = C::PAIR && !VALUES ? 64 : 128, BYTES = C::PAIR && VALUES ? 64 : D, LPR = BYTES / 16, STEPS = ROWS / 4 * LPR / 32;
    // Row and 16-byte piece of this lane in a step: of the eight lanes that store together in rows of 128 codes, four are in the next row,
    // whose swizzle puts their chunks into the other banks.
    const int lane_row = LPR == 8 ? (lane >> 4) * 2 + ((lane >> 2) & 1) : lane / 4, piece = LPR == 8 ? (lane & 3) | ((lane >> 1) & 4) : lane & 3;
    const int st = FIRST + n % STAGES, slot = raws % C::RAW;
    if (!WAIT2S(&mi.kv_free[st], free_par(n / STAGES), W2_KVFREE) || !WAIT2S(&ex.raw_full[slot], full_par(raws / C::RAW), W2_KVFULL)) return false;
    uint8_t* const to = cx.ring + st * C::STAGE_BYTES;
    uint8_t* const from = raw + slot * C::RAW_BYTES;
    // What stands behind a sequence's length may be codes that are no number, and those times 0 are none either.  (Behind n_keys a copy has zeros.)
    if constexpr (VALUES && FMT == FMT_E4M3) {
      if (prm.c.len != nullptr && valid < TILE) {
        for (int i = lane; i < ROWS / 4 * LPR; i += 32)
          if (warp * (ROWS / 4) + i / LPR >= valid) *reinterpret_cast<uint4*>(from + (warp * (ROWS / 4) * LPR + i) * 16) = make_uint4(0, 0, 0, 0);
        __syncwarp();
      }
    }
    if constexpr (VALUES && is_tree<T>() && FMT == FMT_E4M3) {     // (one CTA: rows 32 warp + lane)
      const int row = warp * 32 + lane;
      if (row >= mine && row < valid) {
        bool is_odd = false;
        for (int i = 0; i < BYTES; i += 16) {              // (the places of a row's pieces do not matter here)
          uint4 x = *reinterpret_cast<const uint4*>(from + row * BYTES + i);
          const uint4 y = make_uint4(x.x & finite_parts<FMT>(x.x), x.y & finite_parts<FMT>(x.y), x.z & finite_parts<FMT>(x.z), x.w & finite_parts<FMT>(x.w));
          if (x.x != y.x || x.y != y.y || x.z != y.z || x.w != y.w) { is_odd = true; *reinterpret_cast<uint4*>(from + row * BYTES + i) = y; }
        }
        if (is_odd) odd |= 1ull << (row - mine);
      }
      __syncwarp();
    }
#pragma unroll
    for (int i0 = 0; i0 < STEPS; i0 += 4) {                // four pieces at a time, their latencies side by side
      uint4 in[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        uint32_t off = (warp * (ROWS / 4) + (i0 + u) * (32 / LPR) + lane_row) * BYTES + piece * 16;
        off ^= ((off >> 7) & (BYTES == 128 ? 7 : 3)) << 4;
        in[u] = *reinterpret_cast<const uint4*>(from + off);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int local = (i0 + u) * (32 / LPR) + lane_row, row = warp * (ROWS / 4) + local;
        const uint4 x = in[u];
        uint4 a, b;
        if constexpr (VALUES && !is_tree<T>()) {
          const float s = __shfl_sync(0xFFFFFFFFu, scale, local);
          const uint2 y0 = codes_to_bf16x4<FMT>(x.x, s), y1 = codes_to_bf16x4<FMT>(x.y, s), y2 = codes_to_bf16x4<FMT>(x.z, s), y3 = codes_to_bf16x4<FMT>(x.w, s);
          a = make_uint4(y0.x, y0.y, y1.x, y1.y);
          b = make_uint4(y2.x, y2.y, y3.x, y3.y);
        } else {
          const uint32_t z0 = flip_signs<FMT>(x.x), z1 = flip_signs<FMT>(x.y), z2 = flip_signs<FMT>(x.z), z3 = flip_signs<FMT>(x.w);
          a = make_uint4(codes_to_half2<FMT, 0>(z0), codes_to_half2<FMT, 1>(z0), codes_to_half2<FMT, 0>(z1), codes_to_half2<FMT, 1>(z1));
          b = make_uint4(codes_to_half2<FMT, 0>(z2), codes_to_half2<FMT, 1>(z2), codes_to_half2<FMT, 0>(z3), codes_to_half2<FMT, 1>(z3));
        }
        uint8_t* const base = to + (piece / 4) * (ROWS * 128);               // elements 16 piece .. 16 piece + 15 of the row
        *reinterpret_cast<uint4*>(base + sw128_offset(row, (2 * piece) % 8)) = a;
        *reinterpret_cast<uint4*>(base + sw128_offset(row, (2 * piece + 1) % 8)) = b;
      }
    }
    if constexpr (!VALUES) {
      const uint32_t at = tile + t;
      const int row = warp * 32 + lane;
      ex.key_scale[at % 8][row] = scale;
      if constexpr (is_tree<T>()) {
        float s = value_scale;
        if (row >= mine && row < valid && !(fabsf(s) < INFINITY)) { odd |= 1ull << (row - mine); s = 1.0f; }       // added with the output: whatever is summed here
        const bool near = s >= 1.0f / NEAR_VALUE && s <= NEAR_VALUE;
        const float l = log2f(s);                          // (zeros: -infinity.  What is no number must not raise the reference.)
        values->log2[at % 8][row] = s < INFINITY ? l : __int_as_float(0x7FC00000);
        values->inverse[at % 8][row] = near ? exp2f(-l) : 0.0f;
        const bool far = __any_sync(0xFFFFFFFFu, !near && row < valid);
        if (lane == 0) values->far[at % 8][warp] = far;
      }
      warp_arrive(&ex.sc_full[at % 8]);
    }
    fence_proxy_async_smem();
    // Behind the stores, which need what was loaded.  An arrival waits for no load that is still on its way: right behind the loads it let
    // the next copy overtake them where the SM's shared memory was busy.
    warp_arrive(&ex.raw_free[slot]);
    warp_arrive(&mi.kv_full[st]);                          // (of a pair's peer: an issuer's warp there passes it on to the leader)
    ++n;
    ++raws;
    return true;
  }
  __device__ __forceinline__ void item(const Item& it, int lag) {
    if constexpr (is_tree<T>()) {
      // (a page is looked up two tiles ahead, so that no warp waits for it to ask for its scales)
      int page = page_of_key(it, 1);
      float2 next = scales_in(it, 0, page_of_key(it, 0));
      for (int h = 0; h < 2 * it.n; ++h) {
        bool is_values;
        int t;
        half_of(h, it.n, lag, is_values, t);
        const int valid = it.keys - (it.j0 + t) * TILE, mine = valid - prm.c.q.w;
        if (is_values) {
          if (!convert<true>(t, 0.0f, valid, mine)) break;
        } else {
          const float2 s = next;
          next = scales_in(it, t + 1, page);
          page = page_of_key(it, t + 2);
          if (!convert<false>(t, s.x, valid, mine, s.y)) break;
        }
      }
    } else {
      float next = scale_of(it, 0, lag);
      for (int h = 0; h < 2 * it.n; ++h) {
        const float scale = next;
        if (h + 1 < 2 * it.n) next = scale_of(it, h + 1, lag);
        bool is_values;
        int t;
        half_of(h, it.n, lag, is_values, t);
        const int valid = it.keys - (it.j0 + t) * TILE;
        if (!(is_values ? convert<true>(t, scale, valid) : convert<false>(t, scale, valid))) break;
      }
    }
    tile += it.n;
  }
};

// The issuers' warps of a pair's peer: a stage that the peer's warps have filled is made known to the leader, with what they have written
// (a release at the cluster's scope takes some 1400 cycles, which the converting warps do not have).
template <class C>
__device__ __forceinline__ void pass_on(const Ctx2& cx, bool values) {
  Misc2& mi = *cx.mi;
  uint32_t nd = 0, n = 0;
  while (true) {
    const Desc d = next_desc<C>(cx, nd, false);
    if (d.kind == KIND_DONE) break;
    for (int t = 0; t < d.t[1]; ++t, ++n) {
      const int st = values ? C::NK + n % C::NV : n % C::NK;
      if (!WAIT2I(&mi.kv_full[st], full_par(n / (values ? C::NV : C::NK)), W2_KVFULL)) break;
      mbar_arrive_cluster(map_to_cta(&mi.kv_full[st], 0));
    }
  }
}
// the issuers' wait for a stage: of a pair also for what the peer has written
template <class C>
__device__ __forceinline__ void wait_operand(const Ctx2& cx, uint64_t* bar, uint32_t parity) {
  if constexpr (C::PAIR) mbar_wait_cluster(bar, parity, cx.abort_flag, cx.status, C::CODE + W2_KVFULL);
  else WAIT2I(bar, parity, W2_KVFULL);
}

// shared memory of a kernel; TREE: its barriers behind the rest
template <int D, int FMT, bool PAIR>
constexpr int extra_tree_at() { return FMT == FMT_BF16 ? Off<Cfg<D, PAIR>>::TOTAL : Off8<Cfg8<D, PAIR>>::EXTRA + (int)sizeof(Extra8); }
template <int D, int FMT, bool PAIR, class T>
constexpr int smem_bytes() { return extra_tree_at<D, FMT, PAIR>() + (is_tree<T>() ? (int)sizeof(ExtraTree) + (FMT != FMT_BF16 ? (int)sizeof(ExtraValues) : 0) : 0); }

// tensor maps: tm_q (rows of a kv-head, 64 x 128); bf16 (boxes of 64 d): tm_k (64 entries of a pair or 128), tm_v (128); 8 bits: codes of 128
// entries, of a pair 64 entries of the keys and 64 columns of the values.  Rows behind the end
// of a tensor read as zeros; the softmax masks the entries behind the last.
// TREE (one CTA): maps of the pool with boxes of 2^log_box entries.
template <int D, int FMT, bool PAIR, class T>
__device__ __forceinline__ void wide_body(const CUtensorMap& tm_q, const CUtensorMap& tm_k, const CUtensorMap& tm_v, const WidePhase& prm,
                                          [[maybe_unused]] const T& tr) {
  constexpr bool TREE = is_tree<T>();
  static_assert(!(TREE && PAIR), "pages are read by single CTAs");
  constexpr bool Q8 = FMT != FMT_BF16;
  using C = typename std::conditional<Q8, Cfg8<D, PAIR>, Cfg<D, PAIR>>::type;
  using O = typename std::conditional<Q8, Off8<Cfg8<D, PAIR>>, Off<Cfg<D, PAIR>>>::type;
  constexpr int NCTA = C::NCTA, NQ = C::NQ;
  extern __shared__ __align__(1024) uint8_t smem[];
  const int tid = threadIdx.x, warp = tid >> 5;
  const uint32_t rank = PAIR ? cluster_ctarank() : 0;
  const bool leader = (rank == 0), alt = prm.alt != 0;
  const int block_rows = TILE * NCTA, group_rows = block_rows * (alt ? 1 : 2), rows = prm.c.rows;
  // first row of block b of CTA `r` in row group rg
  auto first_row = [&](int rg, int b, int r) { return rg * group_rows + (alt ? 0 : b * block_rows) + r * TILE; };
  if (tid == WARP_PRODUCER * 32) { tma_prefetch_desc(&tm_q); tma_prefetch_desc(&tm_k); tma_prefetch_desc(&tm_v); }
  Ctx2 cx;
  cx.mi = reinterpret_cast<Misc2*>(smem + O::MISC);
  cx.sQ = smem + O::Q;
  cx.ring = smem + O::RING;
  cx.abort_flag = &cx.mi->abort_flag;
  cx.status = prm.c.status;
  Misc2& mi = *cx.mi;
  Extra8& ex = *reinterpret_cast<Extra8*>(smem + Off8<Cfg8<D, PAIR>>::EXTRA);       // (8-bit formats)
  [[maybe_unused]] ExtraTree& et = *reinterpret_cast<ExtraTree*>(smem + extra_tree_at<D, FMT, PAIR>());
  [[maybe_unused]] ExtraValues& ev = *reinterpret_cast<ExtraValues*>(smem + extra_tree_at<D, FMT, PAIR>() + sizeof(ExtraTree));
  if (tid == 0) {
    if constexpr (TREE) { mbar_init(&et.fix_go, 1); mbar_init(&et.fix_done, 4); mbar_init(&et.odd_full, 4); }
    // Four converting warps, and the peer's word, in the place of a copy.  Test hook: the second message, of a CTA with one item the last, asks
    // for an arrival more than it gets, and the waits for it run out.
    init_barriers2<C>(mi, prm.c.wait_kcycles, leader, !Q8 ? 1 : PAIR && leader ? 5 : 4, Q8, prm.c.skip_final_publication != 0 ? 2 : 1);
    if constexpr (Q8) {
      for (int i = 0; i < 8; ++i) mbar_init(&ex.sc_full[i], 4);
      for (int i = 0; i < 6; ++i) { mbar_init(&ex.raw_full[i], 1); mbar_init(&ex.raw_free[i], 4); }
      fence_mbar_init();
    }
  }
  if (warp == WARP_QK) { if constexpr (PAIR) tmem_alloc_pair(&mi.tmem_base, 512); else tmem_alloc(&mi.tmem_base, 512); }
  tc_fence_before_sync();
  __syncthreads();
  if constexpr (PAIR) cluster_sync_all();
  tc_fence_after_sync();
  cx.tmem = mi.tmem_base;
  if (!TREE || warp != WARP_PRODUCER) chain();

  if (warp >= WARP_PRODUCER) {
    setmaxnreg_dec<REGS_PARALLEL.service>();
    if (warp == WARP_PRODUCER) {
      // ================================================================ work queue, queries, and for bf16 the cache (both CTAs of a pair)
      if constexpr (TREE) {
        // The whole warp: one lane waits, expects and publishes, each has a box of a tile.  (One thread for all boxes, 64 tokens of one sequence over 32768 bf16
        // entries, a block an item: pages of 16 entries 88 us, of 128 59; so 84 and 58.  With two blocks an item, which read a page once, 60 and 53.)
        constexpr int PARTS = Q8 ? 1 : C::ATOMS, ROW = Q8 ? D : 128;                 // copies of a box, bytes of their rows
        const int lane = tid & 31, n_items = prm.c.seqs * prm.c.Hkv * prm.c.n_rg * prm.c.n_split, lag = alt ? 2 : 1;
        const int part = lane >> (7 - tr.log_box), lane_box = part < PARTS ? lane - (part << (7 - tr.log_box)) : TILE;
        const int lane_to = part * 16384 + (lane_box << tr.log_box) * ROW;
        Prod p;
        uint32_t raws = 0;                                 // uses of the raw slots
        for (bool first_item = true;; first_item = false) {
          int item = n_items;                              // (the first without asking the queue)
          if (lane == 0 && !*cx.abort_flag) item = first_item ? (int)blockIdx.x : (int)gridDim.x + atomicAdd(prm.counter, 1);
          item = __shfl_sync(0xFFFFFFFFu, item, 0);
          if (item >= n_items) break;
          const Item it = decode_item(prm, tr, item);
          if (it.n == 0) {                                   // (its slots say so already)
            if (first_item) chain();
            continue;
          }
          PageIds ids(tr, it, lane);
          auto queries = [&]() {
            if (lane == 0) {
              for (int b = 0; b < (!alt && first_row(it.rg, 1, 0) < rows ? 2 : 1); ++b) {
                const int qs = p.q % NQ;
                WAIT2(&mi.q_free[qs], free_par(p.q / NQ), W2_QFREE);
                mbar_arrive_expect_tx(&mi.q_full[qs], C::Q_BYTES);
                for (int a = 0; a < C::ATOMS; ++a)           // (rows behind the last are zeros and count as copied)
                  load_box<C>(cx.sQ + qs * C::Q_BYTES + a * 16384, &tm_q, smem_u32(&mi.q_full[qs]), a * 64, it.seq * rows + first_row(it.rg, b, 0), it.hkv, 0);
                ++p.q;
              }
            }
            __syncwarp();
          };
          if (lane == 0) {
            Desc d;
            d.kind = KIND_FLASH;
            d.c = it.seq; d.hkv = it.hkv; d.len = it.split;
            d.h[0] = it.rg; d.h[1] = it.keys;
            d.t[0] = it.j0; d.t[1] = it.n;
            d.n[0] = alt ? (it.n + 1) / 2 : it.n;
            d.n[1] = alt ? it.n / 2 : (first_row(it.rg, 1, 0) < rows ? it.n : 0);
            publish<C>(cx, p, d);
          }
          // The first item's first copies go out before the rows are made: all that stands before the launch for the rows is done when that lets this one
          // start.  (64 tokens of one sequence over 32768 entries 52.6 -> 51.1 us.)
          const int early = first_item ? lag + 1 < 2 * it.n ? lag + 1 : 2 * it.n : 0;
          if (!first_item) queries();
          for (int h = 0; h < 2 * it.n; ++h) {
            if (first_item && h == early) { chain(); queries(); }
            bool values;
            int t;
            half_of(h, it.n, lag, values, t);
            const int j = it.j0 + t, first = page_of(tr.pages, j * TILE), boxes = tile_boxes(tr, it.keys, j);
            if (values) ids.reach(tr, it, first, lane);      // (keys are ahead of the values)
            const int e = j * TILE + (lane_box << tr.log_box), which = lane_box < boxes ? page_of(tr.pages, e) : first, id = ids.of(which);
            uint32_t& n = Q8 ? raws : values ? p.v : p.k;
            int slot;
            uint64_t *free_bar, *full_bar;
            uint8_t* to;
            uint32_t par;
            if constexpr (Q8) {
              slot = raws % C::RAW; par = free_par(raws / C::RAW);
              free_bar = &ex.raw_free[slot]; full_bar = &ex.raw_full[slot];
              to = smem + O::RAW + slot * C::RAW_BYTES;
            } else {
              slot = values ? stage_of<C, true>(n) : stage_of<C, false>(n);
              par = free_par(values ? lap_of<C, true>(n) : lap_of<C, false>(n));
              free_bar = &mi.kv_free[slot]; full_bar = &mi.kv_full[slot];
              to = cx.ring + slot * C::STAGE_BYTES;
            }
            int ok = 1;
            if (lane == 0) {
              ok = !*cx.abort_flag && WAIT2I(free_bar, par, W2_KVFREE);
              if (ok) mbar_arrive_expect_tx(full_bar, (uint32_t)(boxes * PARTS * ROW) << tr.log_box);
            }
            if (!__shfl_sync(0xFFFFFFFFu, ok, 0)) break;
            ++n;
            if (lane_box < boxes)
              load_box<C>(to + lane_to, values ? &tm_v : &tm_k, smem_u32(full_bar), Q8 ? 0 : part * 64, e - which * tr.pages.page, it.hkv,
                          page_checked(tr.pages, id, cx.status));
            __syncwarp();
          }
          if (first_item && early == 2 * it.n) { chain(); queries(); }
        }
        if (lane == 0) {
          Desc d;
          d.kind = KIND_DONE; d.c = d.hkv = d.len = 0;
          publish<C>(cx, p, d);
          if constexpr (!Q8) drain_copies<C>(cx, p, leader);
          else if (*cx.abort_flag) {                          // every copy issued has landed before the exit
            for (uint32_t i = (p.q > NQ ? p.q - NQ : 0); i < p.q; ++i) mbar_wait_drain(&mi.q_full[i % NQ], full_par(i / NQ), cx.abort_flag);
            for (uint32_t i = (raws > C::RAW ? raws - C::RAW : 0); i < raws; ++i) mbar_wait_drain(&ex.raw_full[i % C::RAW], full_par(i / C::RAW), cx.abort_flag);
            abort_grace_pause(cx.abort_flag);
          }
        }
      } else if (elect_one()) {
        const int n_items = prm.c.seqs * prm.c.Hkv * prm.c.n_rg * prm.c.n_split;
        Prod p;
        [[maybe_unused]] uint32_t raws = 0;                // uses of the raw slots
        while (!*cx.abort_flag) {
          const int item = next_item<C>(cx, p, leader, prm.counter, n_items);
          if (item >= n_items) break;
          const Item it = decode_item(prm, tr, item);
          if (it.n == 0) continue;                           // (its slots say so already)
          Desc d;
          d.kind = KIND_FLASH;
          d.c = it.seq; d.hkv = it.hkv; d.len = it.split;
          d.h[0] = it.rg; d.h[1] = it.keys;
          d.t[0] = it.j0; d.t[1] = it.n;
          d.n[0] = alt ? (it.n + 1) / 2 : it.n;
          d.n[1] = alt ? it.n / 2 : (first_row(it.rg, 1, 0) < rows ? it.n : 0);
          publish<C>(cx, p, d);
          for (int b = 0; b < (alt ? 1 : 2); ++b) {
            if (d.n[b] == 0) continue;
            const int qs = p.q % NQ;
            WAIT2(&mi.q_free[qs], free_par(p.q / NQ), W2_QFREE);
            if (leader) mbar_arrive_expect_tx(&mi.q_full[qs], NCTA * C::Q_BYTES);
            const uint32_t bar = in_cta<C>(&mi.q_full[qs], 0);
            for (int a = 0; a < C::ATOMS; ++a)             // (rows behind the last are zeros and count as copied)
              load_box<C>(cx.sQ + qs * C::Q_BYTES + a * 16384, &tm_q, bar, a * 64, it.seq * rows + first_row(it.rg, b, rank), it.hkv, 0);
            ++p.q;
          }
          if constexpr (Q8) {
            for (int h = 0; h < 2 * it.n; ++h, ++raws) {
              bool values;
              int t;
              half_of(h, it.n, alt ? 2 : 1, values, t);
              const int slot = raws % C::RAW;
              if (!WAIT2I(&ex.raw_free[slot], free_par(raws / C::RAW), W2_KVFREE)) break;
              mbar_arrive_expect_tx(&ex.raw_full[slot], C::RAW_BYTES);
              tma_load_4d(smem + O::RAW + slot * C::RAW_BYTES, values ? &tm_v : &tm_k, &ex.raw_full[slot], PAIR && values ? (int)rank * 64 : 0,
                          (it.j0 + t) * TILE + (PAIR && !values ? (int)rank * 64 : 0), it.hkv, it.seq);
            }
          } else {
            uint8_t* dst;
            auto load_k = [&](int t) {
              const uint32_t bar = ring_stage<C, false>(cx, p, leader, &dst);
              if (!bar) return;
              for (int a = 0; a < C::ATOMS; ++a)
                load_box<C>(dst + a * (PAIR ? 8192 : 16384), &tm_k, bar, a * 64, (it.j0 + t) * TILE + (PAIR ? (int)rank * 64 : 0), it.hkv, it.seq);
            };
            const int lag = alt ? 2 : 1;
            for (int t = 0; t < lag && t < it.n; ++t) load_k(t);
            for (int t = 0; t < it.n; ++t) {
              const uint32_t bar = ring_stage<C, true>(cx, p, leader, &dst);
              if (bar)
                for (int a = 0; a < (PAIR ? 1 : C::ATOMS); ++a)
                  load_box<C>(dst + a * 16384, &tm_v, bar, PAIR ? (int)rank * 64 : a * 64, (it.j0 + t) * TILE, it.hkv, it.seq);
              if (t + lag < it.n) load_k(t + lag);
            }
          }
        }
        Desc d;
        d.kind = KIND_DONE; d.c = d.hkv = d.len = 0;
        publish<C>(cx, p, d);
        if constexpr (!Q8) drain_copies<C>(cx, p, leader);
        else if (*cx.abort_flag) {                          // every copy issued has landed before the exit
          for (uint32_t i = (p.q > NQ ? p.q - NQ : 0); i < p.q && leader; ++i) mbar_wait_drain(&mi.q_full[i % NQ], full_par(i / NQ), cx.abort_flag);
          for (uint32_t i = (raws > C::RAW ? raws - C::RAW : 0); i < raws; ++i) mbar_wait_drain(&ex.raw_full[i % C::RAW], full_par(i / C::RAW), cx.abort_flag);
          abort_grace_pause(cx.abort_flag);                // (of a pair the peer cannot see its last copy of queries land)
        }
      }
      __syncwarp();
    } else if (warp == WARP_QK && leader) {
      // ================================================================ issuer of Q K^T (of a pair: leader CTA)
      if (elect_one()) {
        IssuerQK<C> is(cx);
        while (true) {
          const Desc d = next_desc<C>(cx, is.nd, false);
          if (d.kind == KIND_DONE) break;
          const int n = d.t[1];
          is.qa[0] = is.qa[1] = is.wait_q();
          if (!alt && d.n[1] > 0) is.qa[1] = is.wait_q();
          for (int t = 0; t < n; ++t) {
            uint32_t k_u32;
            if constexpr (Q8) {
              const int st = is.k % C::NK;
              wait_operand<C>(cx, &mi.kv_full[st], full_par(is.k / C::NK));
              k_u32 = smem_u32(cx.ring) + st * C::STAGE_BYTES;
            } else {
              k_u32 = is.wait_k();
            }
            const int first = alt ? t & 1 : 0, last = alt ? first : (d.n[1] > 0 ? 1 : 0);
#pragma unroll 1
            for (int b = first; b <= last; ++b) {
              if constexpr (Q8) {
                constexpr uint32_t idesc = make_idesc_f16_f32(TILE * NCTA, TILE);
                const int sb = C::TWO_S ? b : 0;
                WAIT2I(&mi.s_read[sb], free_par(is.ns >> sb), W2_SREAD);
                is.ns ^= 1u << sb;
                tc_fence_after_sync();
                if constexpr (PAIR) mma_ss_pair_k128<true>(cx.tmem + C::tm_s(b), b ? is.qa[1] : is.qa[0], k_u32, idesc);
                else if constexpr (D == 128) mma_ss_k128(cx.tmem + C::tm_s(b), b ? is.qa[1] : is.qa[0], k_u32, idesc);
                else mma_ss_k64(cx.tmem + C::tm_s(b), b ? is.qa[1] : is.qa[0], k_u32, idesc);
                commit<C>(&mi.s_full[b]);
              } else {
                is.qk(b, k_u32);
              }
            }
            if constexpr (Q8) commit<C>(&mi.kv_free[is.k++ % C::NK]);
            else is.free_k();
          }
          if constexpr (TREE) {                                // the queries are free behind the last product that reads them: the next item's come under this one's end
            for (uint32_t i = is.nq - (!alt && d.n[1] > 0 ? 2 : 1); i != is.nq; ++i) commit<C>(&mi.q_free[i % NQ]);
          }
        }
        commit<C>(&mi.mma_done);
      }
      __syncwarp();
    } else if (Q8 && PAIR && !leader && (warp == WARP_QK || warp == WARP_PV)) {
      if constexpr (Q8 && PAIR)
        if (elect_one()) pass_on<C>(cx, warp == WARP_PV);
      __syncwarp();
    } else if (warp == WARP_PV && leader) {
      // ================================================================ issuer of P V (of a pair: leader CTA)
      if (elect_one()) {
        IssuerPV<C> is(cx);
        [[maybe_unused]] uint32_t fixes = 0;
        while (true) {
          const Desc d = next_desc<C>(cx, is.nd, false);
          if (d.kind == KIND_DONE) break;
          const int n = d.t[1];
          for (int t = 0; t < n; ++t) {
            const int first = alt ? t & 1 : 0, last = alt ? first : (d.n[1] > 0 ? 1 : 0), step = alt ? 2 : 1;
            if constexpr (TREE && !Q8) {
              if (tail_tile(tr, prm, d.h[1], d.t[0] + t)) {
                wait_stage<C, true>(cx, is.v);
                mbar_arrive(&et.fix_go);
                WAIT2I(&et.fix_done, full_par(fixes), W2_KVFULL);
                ++fixes;
              }
            }
#pragma unroll 1
            for (int b = first; b <= last; ++b) {
              if constexpr (Q8) {
                constexpr uint32_t idesc = TREE ? make_idesc_f16_f32(TILE * NCTA, D, true) : make_idesc_bf16_f32(TILE * NCTA, D, false, true);
                const uint32_t tO = cx.tmem + C::TM_O + b * D, tP = cx.tmem + C::TM_P + b * 64;
                if (t < step) { is.wait_read_out(b); is.blocks ^= 1u << b; }
                const uint32_t par = full_par(is.tiles >> b);
                is.tiles ^= 1u << b;
                WAIT2I(&mi.p_half[b], par, W2_PHALF);
                const int st = C::NK + is.v % C::NV;
                wait_operand<C>(cx, &mi.kv_full[st], full_par(is.v / C::NV));
                const uint32_t v_smem = smem_u32(cx.ring) + st * C::STAGE_BYTES;
                tc_fence_after_sync();
                mma_ts_k64<PAIR>(tO, tP, v_smem, idesc, t >= step);
                WAIT2I(&mi.p_full[b], par, W2_PFULL);
                tc_fence_after_sync();
                mma_ts_k64<PAIR>(tO, tP + 32, v_smem + 8192, idesc, true);
                commit<C>(&mi.pv_done[b]);
                if (t + step >= n) commit<C>(&mi.o_full[b]);
              } else {
                is.pv(b, t < step, t + step >= n);
              }
            }
            if constexpr (Q8) commit<C>(&mi.kv_free[C::NK + is.v++ % C::NV]);
            else is.free_v();
          }
        }
        commit<C>(&mi.mma_done);
      }
      __syncwarp();
    }
  } else if (warp >= WARP_EPI) {
    // ================================================================ 8-bit: operands of the codes; then the epilogue, thread = query row
    setmaxnreg_dec<REGS_PARALLEL.epilogue>();
    const int r = tid & 127;
    const uint32_t lane_sel = static_cast<uint32_t>((warp & 3) * 32) << 16;
    uint32_t nd = 0, nq = 0, no[2] = {0, 0};
    using Conv = Converter<Cfg8<D, PAIR>, Q8 ? FMT : FMT_INT8, T>;
    Conv conv(cx, prm, ex, smem + Off8<Cfg8<D, PAIR>>::RAW, warp - WARP_EPI, tid & 31, tr, &ev);
    [[maybe_unused]] uint32_t values_used = 0, fixes = 0, odd_items = 0;
    while (true) {
      const Desc d = next_desc<C>(cx, nd, true);
      if (d.kind == KIND_DONE) break;
      if constexpr (Q8) conv.item(Item{d.c, d.hkv, d.h[0], d.len, d.h[1], d.t[0], d.t[1]}, alt ? 2 : 1);
      [[maybe_unused]] unsigned long long item_odd = 0;
      if constexpr (TREE) {
        const int before = d.h[1] - prm.c.q.w;                               // entries before the new tokens
        if (tail_tile(tr, prm, d.h[1], d.t[0] + d.t[1] - 1)) {
          unsigned long long odd = conv.odd;
          if constexpr (!Q8) {
            // Values of these tiles, thread = entry: behind the last one zeros, and of the new tokens' what is a number: a value that is none would reach the
            // rows that do not see it, times their zero.  Those that do get it with the output.
            const int t0 = before / TILE > d.t[0] ? before / TILE - d.t[0] : 0;
#pragma unroll 1
            for (int t = t0; t < d.t[1]; ++t) {
              const uint32_t use = values_used + t;
              const int s = stage_of<C, true>(use);
              if (!WAIT2S(&et.fix_go, full_par(fixes), W2_KVFULL) || !WAIT2S(&mi.kv_full[s], full_par((lap_of<C, true>(use))), W2_KVFULL)) break;
              ++fixes;
              const int e = (d.t[0] + t) * TILE + r;
              if (e >= before) {
                for (int i = 0; i < C::ATOMS * 8; ++i) {
                  uint4* const at = reinterpret_cast<uint4*>(cx.ring + s * C::STAGE_BYTES + (i >> 3) * 16384 + r * 128) + (i & 7);
                  uint4 x = make_uint4(0, 0, 0, 0);
                  if (e < d.h[1]) {
                    const uint4 y = *at;
                    x = make_uint4(y.x & finite_parts<FMT_BF16>(y.x), y.y & finite_parts<FMT_BF16>(y.y), y.z & finite_parts<FMT_BF16>(y.z), y.w & finite_parts<FMT_BF16>(y.w));
                    if (x.x == y.x && x.y == y.y && x.z == y.z && x.w == y.w) continue;
                    odd |= 1ull << (e - before);
                  }
                  *at = x;
                }
              }
              fence_proxy_async_smem();
              warp_arrive(&et.fix_done);
            }
          }
          // what the four warps took out, together
          unsigned long long* const all = et.odd[odd_items & 1];
          const uint32_t lo = __reduce_or_sync(0xFFFFFFFFu, (uint32_t)odd), hi = __reduce_or_sync(0xFFFFFFFFu, (uint32_t)(odd >> 32));
          if ((tid & 31) == 0) all[warp - WARP_EPI] = (unsigned long long)hi << 32 | lo;
          warp_arrive(&et.odd_full);
          if (WAIT2S(&et.odd_full, full_par(odd_items), W2_KVFULL)) item_odd = all[0] | all[1] | all[2] | all[3];
          ++odd_items;
          conv.odd = 0;
        }
        values_used += d.t[1];
      }
#pragma unroll 1
      for (int b0 = 0; b0 < (alt ? 1 : 2); ++b0) {
        // one output block: block b0, or with alt the sum of both (the second may have had no tile)
        if ((b0 ? d.n[1] : d.n[0]) == 0) continue;
        const bool two = alt && d.n[1] > 0;
        float m = -INFINITY, f[2] = {0.0f, 0.0f}, l = 0.0f;
        {
          float mb[2] = {-INFINITY, -INFINITY}, lb[2] = {0.0f, 0.0f};
          [[maybe_unused]] float ms[2] = {-INFINITY, -INFINITY}, ls[2] = {0.0f, 0.0f};             // weights by themselves
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int b = alt ? i : b0;
            if (i == 1 && !two) break;
            const uint32_t ph = b ? no[1] : no[0];
            WAIT2(&mi.lm_full[b], full_par(ph), W2_LM);
            mb[i] = mi.lm[b][0][r];
            lb[i] = mi.lm[b][1][r];
            if constexpr (TREE && Q8) { ms[i] = ev.sums[b][0][r]; ls[i] = ev.sums[b][1][r]; }
            warp_arrive(&mi.lm_free[b]);
            WAIT2S(&mi.o_full[b], full_par(ph), W2_OFULL);
            if (b) ++no[1]; else ++no[0];
          }
          m = fmaxf(mb[0], mb[1]);
          if constexpr (TREE && Q8) m = fmaxf(m, fmaxf(ms[0], ms[1]));
#pragma unroll
          for (int i = 0; i < 2; ++i) f[i] = mb[i] == -INFINITY ? 0.0f : fast_exp2(mb[i] - m);
          l = f[0] * lb[0] + f[1] * lb[1];
          if constexpr (TREE && Q8) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
              if (ms[i] != -INFINITY) l = fmaf(fast_exp2(ms[i] - m), ls[i], l);
          }
        }
        tc_fence_after_sync();
        if (!TREE && r == 0) mbar_arrive(&mi.q_free[nq % NQ]);               // every MMA that reads the query slot has completed
        ++nq;
        const int row = first_row(d.h[0], b0, rank) + r;
        const bool valid = row < rows;
        [[maybe_unused]] unsigned long long sees = 0;
        if constexpr (TREE) { if (valid) sees = __ldg(tr.sees + d.c * prm.c.q.w + row / (prm.c.q.Hq / prm.c.q.Hkv)); }
        const size_t prow = ((size_t)d.hkv * prm.c.total_rows + (size_t)d.c * rows + row) * prm.c.n_slots + prm.c.slot0 + d.len;
        uint4* const out = reinterpret_cast<uint4*>(prm.c.part_o + prow * D);
        const uint32_t tO = cx.tmem + C::TM_O + (alt ? 0 : b0 * D) + lane_sel;
#pragma unroll 1
        for (int q = 0; q < D / 16; ++q) {
          uint32_t oa[16], ob[16];
          tmem_ld16(tO + q * 16, oa);
          if (two) tmem_ld16(tO + D + q * 16, ob);
          tmem_wait_ld();
          float x[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            asm volatile("" : "+r"(oa[i]));                                  // no use moves above the wait
            x[i] = __uint_as_float(oa[i]) * f[0];
          }
          if (two) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              asm volatile("" : "+r"(ob[i]));
              x[i] = fmaf(__uint_as_float(ob[i]), f[1], x[i]);
            }
          }
          if (valid) {
            st_global_f32x8(out + q * 4, &x[0]);                             // (the workspace's parts are aligned to 32 bytes)
            st_global_f32x8(out + q * 4 + 2, &x[8]);
          }
        }
        warp_arrive_leader(in_cta<C>(&mi.o_free[alt ? 0 : b0], 0));
        if (two) warp_arrive_leader(in_cta<C>(&mi.o_free[1], 0));
        if constexpr (TREE) {
          if (sees == 0) l = 0.0f;                                             // the token is not there
          if (item_odd & sees) add_odd<D, FMT, D>(tr, prm.c, d.hkv, d.c, d.h[1] - prm.c.q.w, item_odd & sees, 0, prm.c.part_o + prow * D);
        }
        if (valid) prm.c.part_ml[prow] = l == 0.0f ? make_float2(-INFINITY, 0.0f) : make_float2(m, l);
      }
    }
  } else {
    // ================================================================ softmax
    setmaxnreg_inc<REGS_PARALLEL.softmax>();
    const int b = warp >> 2;
    const int r = tid & 127;
    const uint32_t lane_sel = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tS = cx.tmem + C::tm_s(b) + lane_sel, tP = cx.tmem + C::TM_P + b * 64 + lane_sel;
    const uint32_t tO = cx.tmem + C::TM_O + b * D + lane_sel;
    using H0 = typename std::conditional<Q8, ScaledHooks<C>, Hooks<C>>::type;
    using H = typename std::conditional<TREE, TreeHooks<H0>, H0>::type;
    H hk(cx, b);
    uint32_t nd = 0, n_s = 0, n_blk = 0, tile = 0;
    while (true) {
      const Desc d = next_desc<C>(cx, nd, true);
      if (d.kind == KIND_DONE) break;
      const int n = b ? d.n[1] : d.n[0];
      if (n > 0) {
        float scale_log2 = prm.c.q.scale_log2;
        if constexpr (Q8) {
          const int row = first_row(d.h[0], b, rank) + r;
          if (row < rows) scale_log2 = __ldg(prm.half_scale + (size_t)d.hkv * prm.c.total_rows + (size_t)d.c * rows + row);
        }
        RowState st = {-INFINITY, 0.0f};
        [[maybe_unused]] float2 sums = make_float2(-INFINITY, 0.0f);             // weights by themselves
        // TREE: a warp whose rows are behind the last only keeps the barriers going; what P and the accumulator hold for it reaches no row
        [[maybe_unused]] const bool idle = TREE && first_row(d.h[0], b, rank) + (r & ~31) >= rows;
        // TREE: tile j has new tokens: which columns the row sees
        [[maybe_unused]] auto look_at = [&](int j) {
          if constexpr (TREE) {
            hk.tail = tail_tile(tr, prm, d.h[1], j);
            if (hk.tail) {
              const int row = first_row(d.h[0], b, rank) + r, first = d.h[1] - prm.c.q.w - j * TILE;
              const unsigned long long sees = row < rows ? __ldg(tr.sees + d.c * prm.c.q.w + row / (prm.c.q.Hq / prm.c.q.Hkv)) : 0;
#pragma unroll
              for (int i = 0; i < 4; ++i) hk.seen[i] = columns_seen(sees, first, 32 * i);
            }
          }
        };
        if constexpr (TREE && Q8) {
          // Tiles up to the first whose values' scales lie far from 1, and the rest, in loops of their own: the call in the first one's loop cost 3 to 5 % of the time.
          int i = 0;
          auto tiles = [&](auto by_themselves) {
            constexpr bool APART = decltype(by_themselves)::value;
#pragma unroll 1
            for (; i < n; ++i) {
              const int t = alt ? 2 * i + b : i, at = (tile + t) % 8;
              WAIT2S(&mi.s_full[b], full_par(n_s), W2_SFULL);
              WAIT2S(&ex.sc_full[at], full_par((tile + t) / 8), W2_KVFULL);
              if (!APART && !idle && *reinterpret_cast<const uint32_t*>(ev.far[at]) != 0) return;
              ++n_s;
              tc_fence_after_sync();
              if (idle) {
                hk.on_read();
                hk.before_p();
                hk.on_half();
                hk.on_full();
              } else {
                look_at(d.t[0] + t);
                if constexpr (APART)
                  sums = weights_apart(tS, scale_log2, sums.x, sums.y, ex.key_scale[at], hk.tail, make_uint4(hk.seen[0], hk.seen[1], hk.seen[2], hk.seen[3]));
                softmax_codes_tile<D>(tS, tP, tO, i == 0, scale_log2, st, hk, ex.key_scale[at], ev.log2[at], ev.inverse[at]);
              }
              ++hk.tiles;
            }
          };
          tiles(std::false_type());
          if (i < n) {
            sums = make_float2(st.m, st.l);                      // (of the tiles before)
            tiles(std::true_type());
            st.l = 0.0f;
          }
        } else {
#pragma unroll 1
          for (int i = 0; i < n; ++i) {
            const int t = alt ? 2 * i + b : i, j = d.t[0] + t, vis = d.h[1] - j * TILE;                  // ragged last tile
            WAIT2S(&mi.s_full[b], full_par(n_s), W2_SFULL);
            ++n_s;
            if constexpr (Q8) {
              const uint32_t at = tile + t;
              WAIT2S(&ex.sc_full[at % 8], full_par(at / 8), W2_KVFULL);
              hk.scale = ex.key_scale[at % 8];
            }
            tc_fence_after_sync();
            if (TREE && idle) {
              hk.on_read();
              hk.before_p();
              hk.on_half();
              hk.on_full();
            } else if constexpr (TREE) {
              look_at(j);
              if (i > 0 && !hk.tail) softmax_tile<D, false>(tS, tP, tO, TILE, false, scale_log2, st, hk);
              else softmax_tile<D, true>(tS, tP, tO, TILE, i == 0, scale_log2, st, hk);
            } else if (i > 0 && vis >= TILE) softmax_tile<D, false>(tS, tP, tO, TILE, false, scale_log2, st, hk);
            else softmax_tile<D, true>(tS, tP, tO, vis, i == 0, scale_log2, st, hk);
            ++hk.tiles;
          }
        }
        WAIT2S(&mi.lm_free[b], free_par(n_blk), W2_LMFREE);
        ++n_blk;
        mi.lm[b][0][r] = st.m;
        mi.lm[b][1][r] = st.l;
        if constexpr (TREE && Q8) { ev.sums[b][0][r] = sums.x; ev.sums[b][1][r] = sums.y; }
        warp_arrive(&mi.lm_full[b]);
      }
      tile += d.t[1];
    }
  }

  teardown<C>(cx);
}

}  // namespace wide
}  // namespace pc
