// Host side that the entry points on caches share: checks of arguments, plans of the attention kernels.
#pragma once
#include "../../include/pc.h"
#include "pc_cache.h"
#include "pc_kernels.h"

#include <atomic>
#include <cmath>

namespace pc {
namespace plan {

constexpr size_t ALIGN = 256;
inline size_t align_up(size_t x) { return (x + ALIGN - 1) / ALIGN * ALIGN; }
constexpr int32_t MOST_ENTRIES = 1 << 30;        // of a call, inside a cache or not: the kernels round up to whole pieces in 32 bits
inline bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline int32_t launched(cudaError_t e) {
  const cudaError_t pending = cudaGetLastError();
  return e == cudaSuccess && pending == cudaSuccess ? PC_OK : PC_ERR_CUDA;
}

// Strides (sequence, token, head) of a tensor [B,n,H,d] in elements; zeros: contiguous.
inline bool strides(const int64_t* in, int64_t n, int64_t H, int64_t d, long long out[3]) {
  if (in == nullptr || (in[0] == 0 && in[1] == 0 && in[2] == 0)) { out[0] = n * H * d; out[1] = H * d; out[2] = d; return true; }
  for (int i = 0; i < 3; ++i) {
    if (in[i] < 0 || in[i] % 8 != 0) return false;
    out[i] = in[i];
  }
  return true;
}

inline int32_t check_cache(const pc_kv_cache* c, bool only8) {
  if (c == nullptr) return PC_ERR_INVALID_ARG;
  if (c->B < 1 || c->Hkv < 1 || c->capacity < 1 || !c->k || !c->v || !aligned(c->k, 16) || !aligned(c->v, 16)) return PC_ERR_INVALID_ARG;
  if (c->d != 64 && c->d != 128) return PC_ERR_UNSUPPORTED;
  if (c->capacity > (1ll << 28) || (int64_t)c->B * c->Hkv > (1 << 24)) return PC_ERR_UNSUPPORTED;
  if (c->format == PC_KV_BF16) return only8 ? PC_ERR_UNSUPPORTED : PC_OK;
  if (c->format != PC_KV_INT8 && c->format != PC_KV_E4M3) return PC_ERR_INVALID_ARG;
  if (!c->k_scale || !c->v_scale || !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4)) return PC_ERR_INVALID_ARG;
  return PC_OK;
}

struct PhasePlan { bool wide, pair, brief, finish; int alt, group, n_rg, n_split; };

// Clusters of n <= 8 CTAs of the kernel for few rows that the current device runs at a time (asked once per device).
inline int few_fit(int n) {
  static std::atomic<int> known[64][9];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
  std::atomic<int>& k = known[dev][n];
  int v = k.load(std::memory_order_relaxed);
  if (v == 0) k.store(v = pc::few_clusters(n) + 1, std::memory_order_relaxed);
  return v - 1;
}

// Splits of the keys, and whether the kernel finishes its rows itself (the last phase; up to 8 splits, the CTAs of a cluster)
// or leaves slots for the merge.  Least time by a model in microseconds: rounds of the grid, two CTAs per SM, x (7.5 for the queries, the
// first unit and the join + its tiles, at a unit in 1.1 (8 rows) or 1.4 for a warp, 0.63 or 0.95 where the SM has one CTA, or at the
// CTA's share of the rate of L2 and memory), and for
// slots 1 + 0.1 a split for writing and merging them.  Measured, us, finished / slots, best split of each: one token over 16401 int8
// entries, 8 kv-heads 19.8 (8) / 15.7 (16); 2000 entries, four sequences 11.2 (8) / 11.8 (4); 4 tokens of 23 sequences of up to 5000,
// head size 64 22.3 (3) / 23.9 (3); 40 sequences of 4000, one kv-head 16.4 (3) / 17.7 (3).
inline PhasePlan few_plan(int64_t seqs, int64_t rows, int Hkv, int d, int format, int n_keys, bool last, int sm_count) {
  PhasePlan p = {};
  p.group = rows <= 8 ? 8 : 16;
  p.n_rg = (int)((rows + p.group - 1) / p.group);
  const double items = (double)seqs * Hkv * p.n_rg;
  // Short caches: four smaller CTAs per SM (16 rows: three) where they take fewer rounds than two; up to 2048 entries for half the rounds, else 1024.
  // Measured, us, two / four (three), int8 caches, G = 8, full and (ragged).
  // 8 rows, head size 128: 320 items of 60 entries 15.4 / 11.2 (15.8 / 10.9), of 1000 30.5 / 29.7 (21.5 / 25.2), of 2000 51.3 / 50.1 (35.8 / 40.9);
  // 512 of 1000 39.7 / 33.8 (31.7 / 27.9); 768 of 1000 56.6 / 60.9 (45.1 / 43.6), of 2000 86.9 / 94.9 (61.4 / 64.3).  Head size 64: 320 of 1000 25.8 / 20.4
  // (18.6 / 18.5); 512 of 2000 43.4 / 35.9 (35.3 / 30.3); 768 of 2000 62.3 / 63.3 (48.5 / 45.2).
  // 16 rows, head size 128: 320 of 1000 56.6 / 40.9 (43.7 / 36.2), of 2000 76.0 / 65.1 (52.0 / 56.6); 512 (as many rounds) of 1000 61.8 / 70.6 (50.7 / 52.4);
  // 768 of 1000 89.2 / 84.4 (73.1 / 70.1).  Head size 64: 320 of 2000 51.4 / 37.9 (36.9 / 33.6); 512 of 1000 40.8 / 45.8 (35.8 / 37.9); 768 of 1000 61.7 / 55.3
  // (50.3 / 46.0), of 2000 85.0 / 78.0 (67.2 / 64.5).
  // The rule goes by the most entries that lengths may name, not by the lengths, which the host does not see.  Where it loses most: ragged, one round of
  // short CTAs at head size 128, up to 17 % (8 rows), 9 % (16); 593 to 600 items of 16 rows at head size 64, ragged bf16, 11 %; else up to 8 %.
  const double small = (p.group == 8 ? 4.0 : 3.0) * sm_count, rounds2 = std::ceil(items / (2.0 * sm_count)), rounds4 = std::ceil(items / small);
  p.brief = rounds4 < rounds2 && n_keys <= (2.0 * rounds4 <= rounds2 ? 2048 : 1024);
  const int keys = pc::few_keys(format, d, p.brief), tiles = (n_keys + keys - 1) / keys;
  p.n_split = 1;
  p.finish = last;
  if (p.brief) return p;
  const double tile_us = 2.0 * keys * d * (format == PC_KV_BF16 ? 2 : 1) / 8.0e6, units = keys / 16;
  double least = -1.0;
  auto look = [&](int s, bool finish) {
    const double fit = finish && s > 1 ? few_fit(s) : std::floor(2.0 * sm_count / s);
    if (fit < 1.0) return;
    const double rounds = std::ceil(items / fit), active = (items < fit ? items : fit) * s;
    const bool single = active <= sm_count;                          // a CTA has its SM for itself
    const double alone = units * (p.group == 8 ? (single ? 0.63 : 1.1) / 7 : (single ? 0.95 : 1.4) / (d == 64 ? 7 : 5)), bytes = tile_us * active;
    const double cost = rounds * (7.5 + (bytes > alone ? bytes : alone) * std::ceil((double)tiles / s)) + (finish ? 0.0 : 1.0 + 0.1 * s);
    if (least < 0.0 || cost < least) { least = cost; p.n_split = s; p.finish = finish; }
  };
  for (int s = 1; s <= 64 && s <= tiles; ++s) {
    if (last && s <= 8) look(s, true);
    look(s, false);
  }
  return p;
}

// Row groups and splits of the kernel for many rows: least time by a model in microseconds, as for the query windows - rounds
// of the grid x (5 for an item + a tile), and the partial results through memory twice.  A tile has one price for all formats and head sizes, that of alt 1.2
// (measured on CTA pairs at head size 128: bf16 0.9, codes 1.3); it weighs rounds against splits and no more.
inline PhasePlan wide_plan(int64_t seqs, int64_t rows, int Hkv, int d, int n_keys, int sm_count) {
  PhasePlan p = {};
  p.wide = true;
  // CTA pairs for more rows than a block has.  Measured, us, without / with, 65536 entries: 128 rows bf16 57.5 / 66.9, int8 72.8 / 91.6; 256 rows 78.8 / 73.0,
  // 127.3 / 96.7; 1024 rows 266.0 / 245.4, 314.7 / 268.1.
  p.pair = d == 128 && rows > 128 && sm_count >= 2;
  const int64_t block = p.pair ? 256 : 128, blocks = (rows + block - 1) / block, units = p.pair ? sm_count / 2 : sm_count;
  const int tiles = (n_keys + 127) / 128;
  double least = -1.0;
  for (int alt = blocks % 2 && blocks < 3 ? 1 : 0; alt <= 1; ++alt) {
    const int64_t n_rg = alt ? blocks : (blocks + 1) / 2;
    const double tile_us = alt ? 1.2 : 2.2;
    for (int s = 1; s <= 64 && (s == 1 || 2 * s <= tiles + 1); ++s) {
      const double rounds = std::ceil((double)seqs * (double)(Hkv * n_rg * s) / (double)units);
      const double cost = rounds * (5.0 + tile_us * std::ceil((double)tiles / s)) + (double)seqs * (double)(rows * Hkv * s) * d * 8.0 / 4.0e6;
      if (least < 0.0 || cost < least) { least = cost; p.alt = alt; p.n_rg = (int)n_rg; p.n_split = s; }
    }
  }
  return p;
}

}  // namespace plan
}  // namespace pc
