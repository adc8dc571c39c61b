// Attention of many query rows over the caches of pc_cache_attn, in bf16 or 8 bits: the shared prefix with the rows of all sequences, or each
// sequence's own cache with its own.
//
// Two 128-row blocks per CTA with a softmax warpgroup each, roles, rings and work queue as in pc_flash.cuh; rows are the new tokens
// (of all sequences over a prefix) times the q-heads of a kv-head, so a tile of the cache is read once for 256 of them (512 on CTA pairs: head
// size 128).  alt = 1: both blocks hold the same rows and take alternate key tiles.  Every item (sequence, kv-head, row group, key split) leaves
// partial results, which the merge kernel joins with the others' and the new tokens' own keys; an item without keys is left out.
//
// 8-bit caches: the epilogue's warps, which have nothing to do while an item's tiles go through, make operands of the codes.  These
// arrive in three slots of a tile's keys or values (pairs: six of half of them), and go into the ring's stages as halves (keys, exactly; the scale of a
// key multiplies its column of S in the softmax warps, the power of two of a query row is part of the row's softmax scale) or as bf16 (values,
// code * scale rounded once, as they are read back: the probabilities beside them are rounded to bf16 too).
//
// Bound by the products and exponentials of a row (4 d operations and an exponential per key) from some 256 rows on, below by the step of a tile itself:
// 65536 entries, 8 kv-heads, d = 128, us: 64 rows bf16 54 (268 MB, 5.0 TB/s), int8 69; 256 rows 72, 98; 1024 rows bf16 230 (1195 TFLOP/s), int8 267
// (1030).  Over codes the converting warps are busy throughout, 900 to 1100 of a tile's 2500 to 3000 cycles (256 rows, pair) in conversions, and the softmax
// waits for them; keys and values on two warps each, with slots of their own, took 1.2 to 1.5 times as long.  A whole call with a tile or two for
// every CTA takes 13 (24 rows over 2000 bf16 entries): three launches.
#include "pc_cache.h"
#include "pc_flash.cuh"
#include "pc_kernels.h"
#include "pc_kv8.cuh"
#include <type_traits>

namespace pc {

namespace {

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

struct Item { int seq, hkv, rg, split, keys, j0, n; };          // keys: entries of the sequence; n tiles from j0, 0: none
__device__ __forceinline__ Item decode_item(const WidePhase& p, int item) {
  Item it;
  it.split = item % p.c.n_split;
  int x = item / p.c.n_split;
  it.rg = x % p.c.n_rg;
  x /= p.c.n_rg;
  it.hkv = x % p.c.Hkv;
  it.seq = x / p.c.Hkv;
  it.keys = p.c.n_keys;
  if (p.c.len != nullptr) it.keys = max(0, min(it.keys, __ldg(p.c.len + it.seq)));
  const int tiles = (it.keys + TILE - 1) / TILE;
  it.j0 = (int)((long long)tiles * it.split / p.c.n_split);
  it.n = (int)((long long)tiles * (it.split + 1) / p.c.n_split) - it.j0;
  return it;
}

// f16 operands, fp32 accumulation
__host__ __device__ constexpr uint32_t make_idesc_f16_f32(int M, int N) {
  return (1u << 4) | (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
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
template <class C, int FMT>
struct Converter {
  static constexpr int D = C::D;
  const Ctx2& cx;
  const WidePhase& prm;
  Extra8& ex;
  uint8_t* raw;
  int warp, lane;
  uint32_t k = 0, v = 0, raws = 0, tile = 0;               // uses of the stages and of the slots; tiles of earlier items
  __device__ __forceinline__ Converter(const Ctx2& c, const WidePhase& p, Extra8& e, uint8_t* raw_smem, int w, int l)
      : cx(c), prm(p), ex(e), raw(raw_smem), warp(w), lane(l) {}

  // scale of key warp * 32 + lane of the tile, 0 behind the last entry
  __device__ __forceinline__ float scale_of(const Item& it, int h, int lag) const {
    bool values;
    int t;
    half_of(h, it.n, lag, values, t);
    const int key = (it.j0 + t) * TILE + warp * 32 + lane;
    return key < it.keys ? __ldg((values ? prm.c.v_scale : prm.c.k_scale) + ((size_t)it.seq * prm.c.Hkv + it.hkv) * prm.c.capacity + key) : 0.0f;
  }
  template <bool VALUES>
  __device__ __forceinline__ bool convert(int t, float scale, int valid) {             // valid: rows of the tile that are entries
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
        if constexpr (VALUES) {
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
      ex.key_scale[at % 8][warp * 32 + lane] = scale;
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
    float next = scale_of(it, 0, lag);
    for (int h = 0; h < 2 * it.n; ++h) {
      const float scale = next;
      if (h + 1 < 2 * it.n) next = scale_of(it, h + 1, lag);
      bool values;
      int t;
      half_of(h, it.n, lag, values, t);
      const int valid = it.keys - (it.j0 + t) * TILE;
      if (!(values ? convert<true>(t, scale, valid) : convert<false>(t, scale, valid))) break;
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

}  // namespace

// tensor maps: tm_q (rows of a kv-head, 64 x 128); bf16 (boxes of 64 d): tm_k (64 entries of a pair or 128), tm_v (128); 8 bits: codes of 128
// entries, of a pair 64 entries of the keys and 64 columns of the values.  Rows behind the end
// of a tensor read as zeros; the softmax masks the entries behind the last.
template <int D, int FMT, bool PAIR>
__global__ void __launch_bounds__(NT2, 1)
cache_wide_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                  const __grid_constant__ WidePhase prm) {
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
  if (tid == 0) {
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
  chain();

  if (warp >= WARP_PRODUCER) {
    setmaxnreg_dec<REGS_PARALLEL.service>();
    if (warp == WARP_PRODUCER) {
      // ================================================================ work queue, queries, and for bf16 the cache (both CTAs of a pair)
      if (elect_one()) {
        const int n_items = prm.c.seqs * prm.c.Hkv * prm.c.n_rg * prm.c.n_split;
        Prod p;
        [[maybe_unused]] uint32_t raws = 0;                // uses of the raw slots
        while (!*cx.abort_flag) {
          const int item = next_item<C>(cx, p, leader, prm.counter, n_items);
          if (item >= n_items) break;
          const Item it = decode_item(prm, item);
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
        while (true) {
          const Desc d = next_desc<C>(cx, is.nd, false);
          if (d.kind == KIND_DONE) break;
          const int n = d.t[1];
          for (int t = 0; t < n; ++t) {
            const int first = alt ? t & 1 : 0, last = alt ? first : (d.n[1] > 0 ? 1 : 0), step = alt ? 2 : 1;
#pragma unroll 1
            for (int b = first; b <= last; ++b) {
              if constexpr (Q8) {
                constexpr uint32_t idesc = make_idesc_bf16_f32(TILE * NCTA, D, false, true);
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
    using Conv = Converter<Cfg8<D, PAIR>, Q8 ? FMT : FMT_INT8>;
    Conv conv(cx, prm, ex, smem + Off8<Cfg8<D, PAIR>>::RAW, warp - WARP_EPI, tid & 31);
    while (true) {
      const Desc d = next_desc<C>(cx, nd, true);
      if (d.kind == KIND_DONE) break;
      if constexpr (Q8) conv.item(Item{d.c, d.hkv, d.h[0], d.len, d.h[1], d.t[0], d.t[1]}, alt ? 2 : 1);
#pragma unroll 1
      for (int b0 = 0; b0 < (alt ? 1 : 2); ++b0) {
        // one output block: block b0, or with alt the sum of both (the second may have had no tile)
        if ((b0 ? d.n[1] : d.n[0]) == 0) continue;
        const bool two = alt && d.n[1] > 0;
        float m = -INFINITY, f[2] = {0.0f, 0.0f}, l = 0.0f;
        {
          float mb[2] = {-INFINITY, -INFINITY}, lb[2] = {0.0f, 0.0f};
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int b = alt ? i : b0;
            if (i == 1 && !two) break;
            const uint32_t ph = b ? no[1] : no[0];
            WAIT2(&mi.lm_full[b], full_par(ph), W2_LM);
            mb[i] = mi.lm[b][0][r];
            lb[i] = mi.lm[b][1][r];
            warp_arrive(&mi.lm_free[b]);
            WAIT2S(&mi.o_full[b], full_par(ph), W2_OFULL);
            if (b) ++no[1]; else ++no[0];
          }
          m = fmaxf(mb[0], mb[1]);
#pragma unroll
          for (int i = 0; i < 2; ++i) f[i] = mb[i] == -INFINITY ? 0.0f : fast_exp2(mb[i] - m);
          l = f[0] * lb[0] + f[1] * lb[1];
        }
        tc_fence_after_sync();
        if (r == 0) mbar_arrive(&mi.q_free[nq % NQ]);                        // every MMA that reads the query slot has completed
        ++nq;
        const int row = first_row(d.h[0], b0, rank) + r;
        const bool valid = row < rows;
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
    using H = typename std::conditional<Q8, ScaledHooks<C>, Hooks<C>>::type;
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
          if (i > 0 && vis >= TILE) softmax_tile<D, false>(tS, tP, tO, TILE, false, scale_log2, st, hk);
          else softmax_tile<D, true>(tS, tP, tO, vis, i == 0, scale_log2, st, hk);
          ++hk.tiles;
        }
        WAIT2S(&mi.lm_free[b], free_par(n_blk), W2_LMFREE);
        ++n_blk;
        mi.lm[b][0][r] = st.m;
        mi.lm[b][1][r] = st.l;
        warp_arrive(&mi.lm_full[b]);
      }
      tile += d.t[1];
    }
  }

  teardown<C>(cx);
}

namespace {

template <int D, int FMT, bool PAIR>
cudaError_t wide_t(const CUtensorMap* maps, const WidePhase& p, int sm_count, cudaStream_t st) {
  using C = Cfg<D, PAIR>;
  constexpr int SMEM = FMT == FMT_BF16 ? Off<C>::TOTAL : Off8<Cfg8<D, PAIR>>::EXTRA + (int)sizeof(Extra8);
  if (cudaError_t e = cudaFuncSetAttribute(cache_wide_kernel<D, FMT, PAIR>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM); e != cudaSuccess) return e;
  const long long n_items = (long long)p.c.seqs * p.c.Hkv * p.c.n_rg * p.c.n_split;
  const int units = sm_count / C::NCTA;
  if (units < 1) return cudaErrorInvalidConfiguration;
  return launch_chained(cache_wide_kernel<D, FMT, PAIR>, dim3((unsigned)((n_items < units ? (int)n_items : units) * C::NCTA)), dim3(NT2), SMEM, st, C::NCTA,
                        maps[0], maps[1], maps[2], p);
}

template <int FMT>
cudaError_t wide_d(const CUtensorMap* maps, const WidePhase& p, int d, bool pair, int sm_count, cudaStream_t st) {
  if (d == 64) return wide_t<64, FMT, false>(maps, p, sm_count, st);
  return pair ? wide_t<128, FMT, true>(maps, p, sm_count, st) : wide_t<128, FMT, false>(maps, p, sm_count, st);
}

}  // namespace

cudaError_t launch_cache_wide(const CUtensorMap* maps, const WidePhase& p, int format, int d, bool pair, int sm_count, cudaStream_t st) {
  return format == FMT_BF16   ? wide_d<FMT_BF16>(maps, p, d, pair, sm_count, st)
         : format == FMT_INT8 ? wide_d<FMT_INT8>(maps, p, d, pair, sm_count, st)
                              : wide_d<FMT_E4M3>(maps, p, d, pair, sm_count, st);
}

}  // namespace pc
