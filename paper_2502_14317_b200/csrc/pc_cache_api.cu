// C ABI of the 8-bit caches and of the attention over shared and own caches: argument checks, plans, launches.
#include "../../include/pc.h"
#include "pc_cache.h"
#include "pc_kernels.h"
#include "pc_tmap.h"

#include <atomic>
#include <cmath>

namespace {

constexpr size_t ALIGN = 256;
size_t align_up(size_t x) { return (x + ALIGN - 1) / ALIGN * ALIGN; }
constexpr int32_t MOST_ENTRIES = 1 << 30;        // of a call, inside a cache or not: the kernels round up to whole pieces in 32 bits
bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
int32_t launched(cudaError_t e) {
  const cudaError_t pending = cudaGetLastError();
  return e == cudaSuccess && pending == cudaSuccess ? PC_OK : PC_ERR_CUDA;
}

// Strides (sequence, token, head) of a tensor [B,n,H,d] in elements; zeros: contiguous.
bool strides(const int64_t* in, int64_t n, int64_t H, int64_t d, long long out[3]) {
  if (in == nullptr || (in[0] == 0 && in[1] == 0 && in[2] == 0)) { out[0] = n * H * d; out[1] = H * d; out[2] = d; return true; }
  for (int i = 0; i < 3; ++i) {
    if (in[i] < 0 || in[i] % 8 != 0) return false;
    out[i] = in[i];
  }
  return true;
}

int32_t check_cache(const pc_kv_cache* c, bool only8) {
  if (c == nullptr) return PC_ERR_INVALID_ARG;
  if (c->B < 1 || c->Hkv < 1 || c->capacity < 1 || !c->k || !c->v || !aligned(c->k, 16) || !aligned(c->v, 16)) return PC_ERR_INVALID_ARG;
  if (c->d != 64 && c->d != 128) return PC_ERR_UNSUPPORTED;
  if (c->capacity > (1ll << 28) || (int64_t)c->B * c->Hkv > (1 << 24)) return PC_ERR_UNSUPPORTED;
  if (c->format == PC_KV_BF16) return only8 ? PC_ERR_UNSUPPORTED : PC_OK;
  if (c->format != PC_KV_INT8 && c->format != PC_KV_E4M3) return PC_ERR_INVALID_ARG;
  if (!c->k_scale || !c->v_scale || !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4)) return PC_ERR_INVALID_ARG;
  return PC_OK;
}

}  // namespace

extern "C" {

int32_t pc_kv_quantize(const pc_kv_cache* cache, const void* k_src, const int64_t* k_stride, const void* v_src, const int64_t* v_stride,
                       int32_t n, int32_t at0, const int32_t* at, int32_t* status_word, void* stream) {
  if (int32_t rc = check_cache(cache, true); rc != PC_OK) return rc;
  if (!k_src || !v_src || !aligned(k_src, 16) || !aligned(v_src, 16) || n < 1 || n > MOST_ENTRIES) return PC_ERR_INVALID_ARG;
  if (at == nullptr && (at0 < 0 || (int64_t)at0 + n > cache->capacity)) return PC_ERR_INVALID_ARG;
  pc::KvWrite w = {};
  if (!strides(k_stride, n, cache->Hkv, cache->d, w.k_stride) || !strides(v_stride, n, cache->Hkv, cache->d, w.v_stride)) return PC_ERR_INVALID_ARG;
  if (pc::sm100_count() == 0) return PC_ERR_UNSUPPORTED;
  w.k_src = k_src; w.v_src = v_src;
  w.k = static_cast<uint8_t*>(cache->k); w.v = static_cast<uint8_t*>(cache->v);
  w.k_scale = cache->k_scale; w.v_scale = cache->v_scale;
  w.capacity = cache->capacity;
  w.B = cache->B; w.Hkv = cache->Hkv; w.n = n; w.at0 = at0; w.at = at; w.status = status_word;
  return launched(pc::launch_kv_quantize(w, cache->format, cache->d, false, static_cast<cudaStream_t>(stream)));
}

int32_t pc_gather_kv_quantize(const void* k_src, const void* v_src, const int64_t* kv_stride, const int32_t* kept, const int32_t* idx,
                              int32_t m, int32_t k, const pc_kv_cache* cache, int32_t* pos_out, void* stream) {
  if (int32_t rc = check_cache(cache, true); rc != PC_OK) return rc;
  if (!k_src || !v_src || !kv_stride || !kept || !idx || !aligned(k_src, 16) || !aligned(v_src, 16) || m < 1 || k < 1) return PC_ERR_INVALID_ARG;
  if (cache->B != 1 || (int64_t)m * k > cache->capacity) return PC_ERR_INVALID_ARG;
  pc::KvWrite w = {};
  for (int i = 0; i < 3; ++i) {
    if (kv_stride[i] <= 0 || kv_stride[i] % 8 != 0) return PC_ERR_INVALID_ARG;
    w.k_stride[i] = w.v_stride[i] = kv_stride[i];
  }
  if (pc::sm100_count() == 0) return PC_ERR_UNSUPPORTED;
  w.k_src = k_src; w.v_src = v_src;
  w.k = static_cast<uint8_t*>(cache->k); w.v = static_cast<uint8_t*>(cache->v);
  w.k_scale = cache->k_scale; w.v_scale = cache->v_scale;
  w.capacity = cache->capacity;
  w.B = 1; w.Hkv = cache->Hkv; w.n = m * k;
  w.kept = kept; w.idx = idx; w.per_chunk = k; w.pos_out = pos_out;
  unsigned bits = 0;                             // 2^bits >= k: with 2^(28 + bits) / k rounded up the product is off by less than 1 / k for e < 2^28
  while ((1ll << bits) < k) ++bits;
  w.chunk_shift = 28 + bits;
  w.chunk_mul = (unsigned)(((1ull << w.chunk_shift) + k - 1) / k);
  return launched(pc::launch_kv_quantize(w, cache->format, cache->d, true, static_cast<cudaStream_t>(stream)));
}

int32_t pc_kv_dequantize(const pc_kv_cache* cache, int32_t n, int32_t at0, const int32_t* at, void* k_out, void* v_out, void* stream) {
  if (int32_t rc = check_cache(cache, true); rc != PC_OK) return rc;
  if (!k_out || !v_out || !aligned(k_out, 16) || !aligned(v_out, 16) || n < 1 || n > MOST_ENTRIES) return PC_ERR_INVALID_ARG;
  if (pc::sm100_count() == 0) return PC_ERR_UNSUPPORTED;
  const pc::KvRead r = {static_cast<const uint8_t*>(cache->k), static_cast<const uint8_t*>(cache->v), cache->k_scale, cache->v_scale,
                        cache->capacity, cache->B, cache->Hkv, n, at0, at, k_out, v_out, aligned(k_out, 32) && aligned(v_out, 32)};
  return launched(pc::launch_kv_dequantize(r, cache->format, cache->d, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"

// ------------------------------------------------------------------------------------ attention over shared and own caches
namespace {

struct PhasePlan { bool wide, pair, brief, finish; int alt, group, n_rg, n_split; };
struct CachePlan {
  PhasePlan prefix, own, window;                 // window: the new tokens' keys as a phase of their own (n_split 0: not)
  int n_slots;                                   // results of a row in memory
  bool finished;                                 // the last phase finishes the rows: no merge
  int64_t total_rows;
  bool rows, halves, mark;                       // a launch for the rows (for a wide phase, or no phase at all), as halves as well (over 8-bit codes);
                                                 // it marks the slots as empty (a wide phase over lengths)
  size_t off_counter, off_rows, off_halves, off_scale, off_ml, off_o, total;
};

// Clusters of n <= 8 CTAs of the kernel for few rows that the current device runs at a time (asked once per device).
int few_fit(int n) {
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
PhasePlan few_plan(int64_t seqs, int64_t rows, int Hkv, int d, int format, int n_keys, bool last, int sm_count) {
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
PhasePlan wide_plan(int64_t seqs, int64_t rows, int Hkv, int d, int n_keys, int sm_count) {
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

// whether rows [B,w,Hkv,d] with these strides can be fetched with TMA: none is 0 where it counts
bool tma_strides(const int64_t* s, int64_t B, int64_t w, int64_t H) {
  return (s[0] == 0 && s[1] == 0 && s[2] == 0) || ((s[0] != 0 || B == 1) && (s[1] != 0 || w == 1) && (s[2] != 0 || H == 1));
}

// More new tokens than these: their keys go through the matrix units, behind the caches' (up to them each row takes them one by one).  Measured, us, one by
// one / units, 32/8 heads of 128 over 2000 int8 entries, a sequence and 16 of them: 12 tokens 18.1 / 24.2, 70.8 / 76.6; 24 22.2 / 25.1, 144.8 / 134.5;
// 32 24.4 / 26.0, 197.7 / 167.7; 64 47.9 / 32.4, 442 / 320.
constexpr int WINDOW_TOKENS = 24;
bool window_phase(const pc_cache_attn_args* a) {
  return a->k_win != nullptr && a->w > WINDOW_TOKENS && tma_strides(a->k_win_stride, a->B, a->w, a->Hkv) && tma_strides(a->v_win_stride, a->B, a->w, a->Hkv);
}

// window: the new tokens' keys are a phase of their own; lens: the own caches have lengths.  Nothing else is read of `a` but its sizes and the caches' descriptors.
int32_t cache_plan(const pc_cache_attn_args* a, bool window, bool lens, int sm_count, CachePlan& p) {
  if (a->B < 1 || a->w < 1 || a->Hq < 1 || a->Hkv < 1 || a->Hq % a->Hkv != 0 || a->n_prefix < 0 || a->n_own < 0) return PC_ERR_INVALID_ARG;
  if (a->d != 64 && a->d != 128) return PC_ERR_UNSUPPORTED;
  if (a->w > 128 || a->Hq > (1 << 18) || (int64_t)a->B * a->w * a->Hq > (1 << 24)) return PC_ERR_UNSUPPORTED;
  const int G = a->Hq / a->Hkv;
  p.total_rows = (int64_t)a->B * a->w * G;
  p.n_slots = 0;
  p.prefix = p.own = p.window = {};
  p.rows = p.halves = p.mark = p.finished = false;
  for (int own = 0; own <= 1; ++own) {
    const pc_kv_cache* const c = own ? a->own : a->prefix;
    const int n = own ? a->n_own : a->n_prefix;
    if (n == 0) continue;
    if (int32_t rc = check_cache(c, false); rc != PC_OK) return rc;
    if (c->B != (own ? a->B : 1) || c->Hkv != a->Hkv || c->d != a->d || n > c->capacity) return PC_ERR_INVALID_ARG;
    PhasePlan& ph = own ? p.own : p.prefix;
    // More than 32 rows over the prefix: the kernel for many; at head size 128 more than 16, over codes, whose conversion it makes in each of its few CTAs, up
    // to 16384 entries.  Measured, us, few / many, 16 rows 12.7 / 12.9 (bf16, 2000 entries), 22.7 / 27.8 (int8, 16000); 24 rows 14.3 / 13.3, 103.8 / 90.2
    // (131072), int8 16.0 / 14.4, 28.5 / 27.6, 117.3 / 119.8, e4m3 15.7 / 14.5, 26.8 / 26.8, 101.0 / 118.7; 40 rows int8 16.5 / 14.7, 166.0 / 121.0; head size
    // 64, 24 rows over 8000 bf16 14.7 / 16.3.
    const int64_t seqs = own ? a->B : 1, rows = p.total_rows / seqs;
    // Own caches: more than 48 rows of a sequence; bf16 more than 16, at head size 64 and little work 32 (what stands behind a length may be no number, and bf16
    // values go to the matrix unit as they are: with lengths never).  Measured, us, few / many, 16 sequences of 2000 entries, 8 kv-heads: int8 d = 128 32 rows
    // 46.7 / 54.7, 48 70.8 / 67.6, 64 94.5 / 73.1, 256 320.7 / 159.5; ragged e4m3 d = 64 48 39.9 / 48.3, 128 93.0 / 63.4; bf16 d = 128 16 34.2 / 35.1,
    // 24 38.7 / 37.0, 64 85.2 / 56.8, d = 64 24 26.3 / 30.0, 48 43.4 / 39.1; 64 sequences, d = 64, 24 rows 94.7 / 78.7.
    const bool bf16 = c->format == PC_KV_BF16;
    const bool many = own ? rows > (!bf16 ? 48 : a->d == 128 || (double)seqs * a->Hkv > 2.0 * sm_count ? 16 : 32) && (!bf16 || !lens)
                          : rows > (a->d == 128 && (bf16 || n <= 16384) ? 16 : 32);
    if (many) {
      ph = wide_plan(seqs, rows, a->Hkv, a->d, n, sm_count);
      p.rows = true;
      p.halves |= !bf16;
      p.mark |= own && lens;
    } else {
      ph = few_plan(seqs, rows, a->Hkv, a->d, c->format, n, !window && (own || a->n_own == 0), sm_count);
    }
    if (seqs * a->Hkv * ph.n_rg * ph.n_split > 0x7FFF0000) return PC_ERR_UNSUPPORTED;      // (a queue's counter goes on by the CTAs)
    if (!ph.finish) p.n_slots += ph.n_split;
    p.finished |= ph.finish;
    // More than a round of CTAs: cheaper than each of them rotating its own.  Measured, us, rotated ahead / by the CTAs, short CTAs of one round:
    // 320 items of 60 entries 10.3 / 8.9, 384 of 16 rows of 1000 43.1 / 41.4.
    if (!ph.wide && (double)seqs * a->Hkv * ph.n_rg * ph.n_split > (ph.brief ? ph.group == 8 ? 4.0 : 3.0 : 2.0) * sm_count) p.rows = true;
  }
  if (window) {
    const int64_t rows = (int64_t)a->w * G;
    PhasePlan& ph = p.window;
    ph.n_split = 1; ph.finish = p.finished = true;
    // Groups of 8 rows, more than a round of them on the short CTAs.  Measured, us, long / short, 16 tokens behind 4000 int8 entries, two sequences
    // 27.0 / 29.7, 16 sequences 65.4 / 55.9 (long ones of 16 rows 63.3, short ones 67.0); 128 tokens 43.3 / 39.2 (42.8, 46.7).
    ph.group = 8;
    ph.n_rg = (int)((rows + 7) / 8);
    ph.brief = (double)a->B * a->Hkv * ph.n_rg > 2.0 * sm_count;
    if ((double)a->B * a->Hkv * ph.n_rg > 4.0 * sm_count) p.rows = true;
  }
  if (p.n_slots == 0 && !p.finished) p.rows = true;
  size_t off = 0;
  p.off_counter = off; off += ALIGN;
  p.off_halves = off; off += p.halves ? align_up((size_t)p.total_rows * a->Hkv * a->d * 2) : 0;
  p.off_scale = off; off += p.halves ? align_up((size_t)p.total_rows * a->Hkv * sizeof(float)) : 0;
  p.off_rows = off; off += align_up((size_t)p.total_rows * a->Hkv * a->d * 2);
  p.off_ml = off; off += align_up((size_t)p.total_rows * a->Hkv * p.n_slots * sizeof(float2));
  p.off_o = off; off += align_up((size_t)p.total_rows * a->Hkv * p.n_slots * a->d * sizeof(float));
  p.total = off;
  return PC_OK;
}

int plan_sms() { const int n = pc::sm100_count(); return n > 0 ? n : 148; }

// tensor maps over the first n entries of a cache, boxes of `keys` entries (8-bit formats: and `cols` columns)
bool cache_maps(const pc_kv_cache* c, int n, int keys, int cols, CUtensorMap* tm_k, CUtensorMap* tm_v) {
  const uint64_t d = (uint64_t)c->d, cap = (uint64_t)c->capacity;
  const uint64_t dims[4] = {d, (uint64_t)n, (uint64_t)c->Hkv, (uint64_t)c->B}, str[3] = {d, cap * d, (uint64_t)c->Hkv * cap * d};
  if (c->format == PC_KV_BF16) {
    const uint32_t box[4] = {64, (uint32_t)keys, 1, 1};
    return pc::make_tmap_bf16_4d(tm_k, c->k, dims, str, box) && pc::make_tmap_bf16_4d(tm_v, c->v, dims, str, box);
  }
  const uint32_t box[4] = {(uint32_t)cols, (uint32_t)keys, 1, 1};
  return pc::make_tmap_u8_4d(tm_k, c->k, dims, str, box) && pc::make_tmap_u8_4d(tm_v, c->v, dims, str, box);
}

// the same for the new tokens' keys or values
bool window_map(const pc_cache_attn_args* a, const void* x, const long long stride[3], int keys, CUtensorMap* tm) {
  const uint64_t dims[4] = {(uint64_t)a->d, (uint64_t)a->w, (uint64_t)a->Hkv, (uint64_t)a->B};
  const uint64_t size[3] = {(uint64_t)a->B, (uint64_t)a->w, (uint64_t)a->Hkv};
  uint64_t s[3];
  for (int i = 0; i < 3; ++i) s[i] = size[i] > 1 ? (uint64_t)stride[i] : (uint64_t)a->d;          // (of one entry any stride will do)
  const uint64_t str[3] = {s[1], s[2], s[0]};
  const uint32_t box[4] = {64, (uint32_t)keys, 1, 1};
  return pc::make_tmap_bf16_4d(tm, x, dims, str, box);
}

}  // namespace

extern "C" {

size_t pc_cache_attn_workspace_bytes(const pc_cache_attn_args* a) {
  if (a == nullptr) return 0;
  // The most over what the call may come with beside its sizes: new tokens or none (or ones that TMA cannot fetch), lengths or none.  Where either makes no
  // difference it is not asked for: plans are host time of every call.
  const bool windows = a->w > WINDOW_TOKENS,
             lengths = a->n_own > 0 && a->own != nullptr && a->own->format == PC_KV_BF16 && a->Hkv > 0 && (int64_t)a->w * a->Hq / a->Hkv > 16;
  size_t most = 0;
  for (int window = 0; window <= (windows ? 1 : 0); ++window)
    for (int lens = 0; lens <= (lengths ? 1 : 0); ++lens) {
      CachePlan p;
      if (cache_plan(a, window != 0, lens != 0, plan_sms(), p) != PC_OK) return 0;
      if (p.total > most) most = p.total;
    }
  return most;
}

int32_t pc_cache_attn(const pc_cache_attn_args* a, void* stream) {
  if (a == nullptr) return PC_ERR_INVALID_ARG;
  CachePlan plan;
  const int sms = pc::sm100_count();
  if (int32_t rc = cache_plan(a, window_phase(a), a->own_len != nullptr, sms > 0 ? sms : 148, plan); rc != PC_OK) return rc;
  if (!a->q || !a->out || !aligned(a->q, 16) || !aligned(a->out, 16) || (a->k_win == nullptr) != (a->v_win == nullptr)) return PC_ERR_INVALID_ARG;
  if (!aligned(a->k_win, 16) || !aligned(a->v_win, 16) || !aligned(a->workspace, 32)) return PC_ERR_INVALID_ARG;
  if (a->n_prefix == 0 && a->n_own == 0 && a->k_win == nullptr) return PC_ERR_INVALID_ARG;              // nothing to attend to
  if ((a->q_pos == nullptr && a->q_pos0 < 0) || !(a->rope_theta >= 0.0f) || !(a->softmax_scale >= 0.0f)) return PC_ERR_INVALID_ARG;
  pc::CacheRows rows = {};
  pc::CacheMerge merge = {};
  if (!strides(a->q_stride, a->w, a->Hq, a->d, rows.stride) || !strides(a->k_win_stride, a->w, a->Hkv, a->d, merge.k_stride) ||
      !strides(a->v_win_stride, a->w, a->Hkv, a->d, merge.v_stride))
    return PC_ERR_INVALID_ARG;
  if (!a->workspace || a->workspace_bytes < plan.total) return PC_ERR_WORKSPACE;
  if (sms == 0) return PC_ERR_UNSUPPORTED;

  cudaStream_t st = static_cast<cudaStream_t>(stream);
  uint8_t* const ws = static_cast<uint8_t*>(a->workspace);
  rows.q = a->q; rows.B = a->B; rows.w = a->w; rows.Hq = a->Hq; rows.Hkv = a->Hkv; rows.pos0 = a->q_pos0; rows.pos = a->q_pos;
  const double scale = a->softmax_scale > 0.0f ? (double)a->softmax_scale : 1.0 / std::sqrt((double)a->d);
  const float scale_log2 = (float)(scale * 1.4426950408889634);
  rows.theta = a->rope_theta; rows.scale_log2 = scale_log2;
  cudaError_t e = cudaSuccess;
  bool made = plan.rows;                                                         // the rows are in memory
  rows.rows = ws + plan.off_rows;
  if (plan.rows) {
    rows.clear = reinterpret_cast<int*>(ws + plan.off_counter);
    rows.clear_too = a->clear_status ? a->status_word : nullptr;
    if (plan.mark) { rows.part_ml = reinterpret_cast<float2*>(ws + plan.off_ml); rows.n_slots = plan.n_slots; }
    if (plan.halves) { rows.halves = ws + plan.off_halves; rows.half_scale = reinterpret_cast<float*>(ws + plan.off_scale); }
    e = pc::launch_cache_rows(rows, a->d, st);
  } else if (a->clear_status && a->status_word) {
    e = cudaMemsetAsync(a->status_word, 0, sizeof(int), st);
  }
  merge.n_slots = plan.n_slots; merge.total_rows = (int)plan.total_rows;
  merge.part_o = reinterpret_cast<const float*>(ws + plan.off_o);
  merge.part_ml = reinterpret_cast<const float2*>(ws + plan.off_ml);
  merge.q = rows;
  merge.k_win = a->k_win; merge.v_win = a->v_win;
  merge.out = static_cast<__nv_bfloat16*>(a->out); merge.lse = a->lse;
  int slot = 0;
  for (int phase = 0; phase <= 2 && e == cudaSuccess; ++phase) {                 // the prefix, the own caches, the new tokens
    const bool own = phase > 0, window = phase == 2;
    const pc_kv_cache* const c = own ? a->own : a->prefix;
    const int n = window ? a->w : own ? a->n_own : a->n_prefix;
    const PhasePlan& ph = window ? plan.window : own ? plan.own : plan.prefix;
    if (ph.n_split == 0) continue;
    pc::CachePhase p = {};
    p.seqs = own ? a->B : 1;
    p.rows = own ? a->w * (a->Hq / a->Hkv) : (int)plan.total_rows;
    p.Hkv = a->Hkv; p.n_keys = n; p.len = own && !window ? a->own_len : nullptr;
    if (!window) { p.k_scale = c->k_scale; p.v_scale = c->v_scale; p.capacity = c->capacity; }
    p.n_rg = ph.n_rg; p.n_split = ph.n_split; p.slot0 = slot; p.n_slots = plan.n_slots; p.total_rows = (int)plan.total_rows;
    p.causal = window;
    p.q = rows;
    p.rows_made = made;
    p.part_o = reinterpret_cast<float*>(ws + plan.off_o);
    p.part_ml = reinterpret_cast<float2*>(ws + plan.off_ml);
    p.status = a->status_word;
    p.wait_kcycles = pc::wait_limit_kcycles();
    p.skip_final_publication = pc::skip_final_publication();
    CUtensorMap maps[3] = {}, unused;
    bool ok;
    if (ph.wide) {
      pc::WidePhase wp = {};
      wp.c = p; wp.alt = ph.alt;
      wp.half_scale = rows.half_scale;
      wp.counter = rows.clear + phase;
      const uint64_t d = (uint64_t)a->d, R = (uint64_t)plan.total_rows;
      const uint64_t dims[4] = {d, R, (uint64_t)a->Hkv, 1}, str[3] = {d, R * d, R * d * (uint64_t)a->Hkv};
      const uint32_t box[4] = {64, 128, 1, 1};
      ok = pc::make_tmap_bf16_4d(&maps[0], c->format != PC_KV_BF16 ? rows.halves : rows.rows, dims, str, box) &&
           cache_maps(c, n, ph.pair ? 64 : 128, c->d, &maps[1], &unused) && cache_maps(c, n, 128, ph.pair ? 64 : c->d, &unused, &maps[2]);
      if (ok) e = pc::launch_cache_wide(maps, wp, c->format, a->d, ph.pair, sms, st);
    } else {
      const int format = window ? PC_KV_BF16 : c->format, keys = pc::few_keys(format, a->d, ph.brief);
      ok = window ? window_map(a, a->k_win, merge.k_stride, keys, &maps[1]) && window_map(a, a->v_win, merge.v_stride, keys, &maps[2])
                  : cache_maps(c, n, keys, c->d, &maps[1], &maps[2]);
      if (ok) e = pc::launch_cache_few(maps[1], maps[2], p, ph.finish ? &merge : nullptr, ph.group, ph.brief, format, a->d, st);
    }
    if (!ok) { launched(e); return PC_ERR_CUDA; }
    if (!ph.finish) slot += ph.n_split;
    made = true;
  }
  if (e != cudaSuccess || plan.finished) return launched(e);
  return launched(pc::launch_cache_merge(merge, a->d, st));
}

}  // extern "C"
