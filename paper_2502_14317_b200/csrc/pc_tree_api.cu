// C ABI of the paged caches, the attention of drafted tokens over them, and the log probabilities: argument checks, plans, launches.
#include "pc_cache_plan.h"
#include "pc_logprob.h"
#include "pc_tmap.h"
#include "pc_tree.h"

#include <algorithm>

using namespace pc::plan;

namespace {

constexpr int64_t MOST_OF_A_SEQUENCE = 1 << 28;
constexpr int MOST_DRAFTED = 64;
int least_tiles(int64_t seqs) { return seqs > 1 ? 4 : 1; }      // of a piece of a sequence's keys, many rows

// a pool of pages and the sequences' tables
int32_t check_pages(const pc_kv_cache* c, const int32_t* table, int64_t stride, int32_t n_table) {
  if (int32_t rc = check_cache(c, false); rc != PC_OK) return rc;
  if (!table || !aligned(table, 4) || stride < 0 || n_table < 1) return PC_ERR_INVALID_ARG;
  if (n_table > 1 && c->capacity % 16 != 0) return PC_ERR_UNSUPPORTED;                  // (the kernels take 16 entries at a time)
  if (c->capacity * n_table > MOST_OF_A_SEQUENCE) return PC_ERR_UNSUPPORTED;
  return PC_OK;
}
pc::Pages pages_of(const pc_kv_cache* c, const int32_t* table, int64_t stride, int32_t n_table) {
  pc::Pages p = {table, stride, n_table, (int)c->capacity, c->B, 0, 0};
  unsigned bits = 0;                             // 2^bits >= page: with 2^(28 + bits) / page rounded up the product is off by less than 1 / page for e < 2^28
  while ((1ll << bits) < c->capacity) ++bits;
  p.shift = 28 + bits;
  p.mul = (unsigned)(((1ull << p.shift) + (uint64_t)c->capacity - 1) / (uint64_t)c->capacity);
  return p;
}

// theta^(-2t/d) / (2 pi) as products of two: off by some 2^-51 of themselves, and sixteen powers make all
void turns_of(float theta, int d, pc::Turns& out) {
  const double step = -2.0 / d, turn = 0.15915494309189535;
  for (int i = 0; i < 8; ++i) {
    out.fine[i] = std::pow((double)theta, step * i);
    out.coarse[i] = std::pow((double)theta, step * 8 * i) * turn;
  }
}
bool good_theta(float theta) { return theta >= 0.0f && std::isfinite(theta); }

}  // namespace

extern "C" {

int32_t pc_page_append(const pc_page_append_args* a, void* stream) {
  if (a == nullptr) return PC_ERR_INVALID_ARG;
  if (int32_t rc = check_pages(a->pages, a->table, a->table_stride, a->n_table); rc != PC_OK) return rc;
  if (a->B < 1 || a->n < 1 || !a->k || !a->v || !aligned(a->k, 16) || !aligned(a->v, 16) || !good_theta(a->rope_theta)) return PC_ERR_INVALID_ARG;
  if (a->at == nullptr && (a->at0 < 0 || (int64_t)a->at0 + a->n > a->pages->capacity * a->n_table)) return PC_ERR_INVALID_ARG;
  if ((a->pick != nullptr && (a->parents != nullptr || a->n_src < 1 || a->pick_stride < 0)) || (a->parents != nullptr && a->parents_stride < 0)) return PC_ERR_INVALID_ARG;
  if (a->n > MOST_OF_A_SEQUENCE || (a->parents != nullptr && a->n > MOST_DRAFTED) || a->B > (1 << 24) || a->pages->Hkv > (1 << 18) - 4)
    return PC_ERR_UNSUPPORTED;
  const pc_kv_cache* const c = a->pages;
  pc::PageWrite w = {};
  const int n_src = a->pick != nullptr ? a->n_src : a->n;
  if (!strides(a->k_stride, n_src, c->Hkv, c->d, w.k_stride) || !strides(a->v_stride, n_src, c->Hkv, c->d, w.v_stride)) return PC_ERR_INVALID_ARG;
  if (pc::sm100_count() == 0) return PC_ERR_UNSUPPORTED;
  w.k_src = a->k; w.v_src = a->v;
  w.k = static_cast<uint8_t*>(c->k); w.v = static_cast<uint8_t*>(c->v);
  w.k_scale = c->k_scale; w.v_scale = c->v_scale;
  w.pages = pages_of(c, a->table, a->table_stride, a->n_table);
  w.B = a->B; w.Hkv = c->Hkv; w.n = a->n; w.n_src = n_src;
  w.at0 = a->at0; w.pos0 = a->pos0; w.at = a->at; w.pos = a->pos; w.count = a->count; w.pick = a->pick; w.parents = a->parents;
  w.pick_stride = a->pick_stride; w.parent_stride = a->parents_stride;
  w.turn = a->rope_theta > 0.0f;
  if (w.turn) turns_of(a->rope_theta, c->d, w.turns);
  w.status = a->status_word;
  return launched(pc::launch_page_append(w, c->format, c->d, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"

// ------------------------------------------------------------------------------------ attention of drafted tokens
namespace {

struct TreePlan {
  PhasePlan phase;
  int n_slots;                                   // results of a row in memory
  int64_t total_rows;
  bool rows, halves;                             // a launch for the rows; as halves as well (many rows over 8-bit codes)
  size_t off_counter, off_sees, off_halves, off_scale, off_rows, off_ml, off_o, total;
};

// Few rows: splits of the keys, as few_plan() but for sequences whose lengths may differ and whose copies go by pages.  Least time by a model in us, fitted to 2458 measured times (1 to 64
// sequences of 1500 to 120000 entries, 4 to 48 rows of 2 and 8 kv-heads, 1 to 64 splits; off by 8 % on average, and the splits that it chooses by 0.7 % of the best): 6.7 for a CTA's start and
// join, 2 more for 16 rows; its tiles, at what a unit of 16 keys takes a warp of a CTA alone on an SM or beside another, or at the memory's rate (of several sequences, whose lengths the
// host does not see, as if they had 0.53 of the longest's); beyond a round of the GPU the launch for the rows, what all have to read, 5 to 6 a round and a third of a longest piece for
// the end, where only the longest sequences are left; slots 1.25 + 0.03 a split.
PhasePlan tree_few_plan(int64_t seqs, int64_t rows, int Hkv, int d, int format, int n_keys, int sm_count, double& least) {
  PhasePlan p = few_plan(seqs, rows, Hkv, d, format, n_keys, true, sm_count);
  least = -1.0;
  if (p.brief) return p;
  const bool bf16 = format == PC_KV_BF16;
  const int keys = pc::few_keys(format, d, false), tiles = (n_keys + keys - 1) / keys;
  static const double unit_us[2][2][2][2] = {{{{0.47, 0.53}, {0.71, 0.85}}, {{1.03, 1.52}, {0.86, 1.18}}},            // 8 rows, head size 64: bf16, codes; 128
                                             {{{0.50, 0.66}, {0.78, 1.14}}, {{1.09, 1.19}, {1.10, 1.25}}}};           // 16
  const auto& us = unit_us[p.group == 16][d == 128][!bf16];
  const double units = keys / 16 / (p.group == 8 || d == 64 ? 7.0 : 5.0), alone = us[0] * units, beside = us[1] * units;
  const double items = (double)seqs * Hkv * p.n_rg, bytes = 2.0 * keys * (bf16 ? 2 * d : d + 4) / 7.3e6 / p.n_rg;           // of a tile, us (row groups share it)
  const double part = seqs > 1 ? 0.53 : 1.0, round_us = bf16 ? 4.6 : 6.0, start = p.group == 8 ? 6.7 : 8.7;
  auto look = [&](int s, bool finish) {
    const double fit = 2.0 * sm_count, ctas = items * s, most = std::ceil((double)tiles / s), mean = (double)tiles / s;
    const double per = seqs > 1 ? 0.2 * most + 0.8 * mean : most;
    double t = start + (finish ? 0.0 : 1.25 + 0.03 * s);
    if (ctas <= fit) {
      const double work = per * (ctas <= sm_count ? alone : beside), read = (seqs > 1 ? per : mean) * part * bytes * ctas;
      t += work > read ? work : read;
    } else {
      const double tile = beside > bytes * fit ? beside : bytes * fit;
      t += 7.9 + part * items * tiles * tile / fit + round_us * (ctas / fit - 1.0) + 0.3 * per * beside;
    }
    if (least < 0.0 || t < least) { least = t; p.n_split = s; p.finish = finish; }
  };
  for (int s = 1; s <= 64 && s <= tiles; ++s) {
    if (s == 1 || (s <= 8 && items <= few_fit(s))) look(s, true);
    look(s, false);
  }
  return p;
}

// Many rows, on single CTAs: blocks of 128 rows, two of them to an item, or one whose key tiles go to either half of the CTA (alt), and pieces of the keys that are drawn
// from a queue.  Least time by a model in us: a tile of two blocks 2.1 (head size 64: 1.55), of one 1.4 (1.1, the memory's rate), a tile more for each piece, the results of the
// pieces through memory; of several sequences, whose lengths the host does not see, 0.6 of the longest's work and half of a piece for the end.  Measured, one sequence, 256 rows, 32768
// entries, 18 pieces of two blocks / 9 of one: pages of 128 53.5 / 56.2, of 16 59.6 / 83.7, head size 64 46.3 / 51.9.
PhasePlan tree_wide_plan(int64_t seqs, int64_t rows, int Hkv, int d, int n_keys, int sm_count, double& least) {
  PhasePlan p = {};
  p.wide = true;
  const int64_t blocks = (rows + 127) / 128;
  const int tiles = (n_keys + 127) / 128, most = (tiles + least_tiles(seqs) - 1) / least_tiles(seqs);
  const double part = seqs > 1 ? 0.6 : 1.0;
  least = -1.0;
  for (int alt = blocks == 1 ? 1 : 0; alt <= 1; ++alt) {
    const int64_t n_rg = alt ? blocks : (blocks + 1) / 2;
    const double items = (double)seqs * Hkv * n_rg, tile = alt ? (d == 64 ? 1.1 : 1.4) : (d == 64 ? 1.55 : 2.1);
    for (int s = 1; s <= most && s <= 64; ++s) {
      const double rounds = items * s / sm_count, per = std::ceil((double)tiles / s);
      double t = (double)seqs * rows * Hkv * s * part * d * 8.0 / 4.0e6;
      if (rounds <= 1.0 || seqs == 1) t += std::ceil(rounds) * (per + 1.0) * tile;
      else t += part * rounds * (per + 1.0) * tile + 0.5 * per * tile;
      if (least < 0.0 || t < least) { least = t; p.alt = alt; p.n_rg = (int)n_rg; p.n_split = s; }
    }
  }
  return p;
}

int32_t tree_plan(const pc_tree_attn_args* a, int sm_count, TreePlan& p) {
  if (a->B < 1 || a->w < 1 || a->Hq < 1 || a->max_len < 0) return PC_ERR_INVALID_ARG;
  if (int32_t rc = check_cache(a->pages, false); rc != PC_OK) return rc;
  const pc_kv_cache* const c = a->pages;
  if (a->Hq % c->Hkv != 0) return PC_ERR_INVALID_ARG;
  if (a->w > MOST_DRAFTED || a->Hq > (1 << 18) || (int64_t)a->B * a->w * a->Hq > (1 << 24) || a->max_len > MOST_OF_A_SEQUENCE) return PC_ERR_UNSUPPORTED;
  const int G = a->Hq / c->Hkv;
  p.total_rows = (int64_t)a->B * a->w * G;
  const int64_t rows = (int64_t)a->w * G;
  const bool bf16 = c->format == PC_KV_BF16;
  const int n_keys = a->max_len + a->w;
  double few_us;
  p.phase = tree_few_plan(a->B, rows, c->Hkv, c->d, c->format, n_keys, sm_count, few_us);
  double wide_us;
  const PhasePlan many = tree_wide_plan(a->B, rows, c->Hkv, c->d, n_keys, sm_count, wide_us);
  // Many rows on the kernel for many where it takes less time: its launches and start some 10, and what the plan's tiles take beside 16 to 48 rows of which a block has 128 (over codes
  // conversions bound a tile); by short CTAs as pc_cache_attn.  Measured, few / many, 16 rows: one sequence of 120000 bf16 entries, head size 64, 22 / 33, 64 of up to 6000 31 / 58; 48 rows: 16 of
  // up to 6000, head size 128, 98 / 63, int8 105 / 97.
  wide_us = c->d == 128 ? (bf16 ? 12.0 + 1.1 * wide_us : 9.5 + 1.85 * wide_us) : (bf16 ? 10.5 + 1.3 * wide_us : 9.5 + 1.75 * wide_us);
  bool wide = p.phase.brief ? rows > (!bf16 ? 48 : c->d == 128 || (double)a->B * c->Hkv > 2.0 * sm_count ? 16 : 32) : rows > 8 && wide_us < few_us;
  if (wide) p.phase = many;
  p.halves = wide && !bf16;
  if ((int64_t)a->B * c->Hkv * p.phase.n_rg * p.phase.n_split > 0x7FFF0000) return PC_ERR_UNSUPPORTED;
  p.n_slots = p.phase.finish ? 0 : p.phase.n_split;
  // more than a round of CTAs: cheaper than each of them rotating its own (as in pc_cache_attn)
  p.rows = p.phase.wide || (double)a->B * c->Hkv * p.phase.n_rg * p.phase.n_split > (p.phase.brief ? p.phase.group == 8 ? 4.0 : 3.0 : 2.0) * sm_count;
  size_t off = 0;
  p.off_counter = off; off += ALIGN;
  p.off_sees = off; off += align_up((size_t)a->B * a->w * 8);
  p.off_halves = off; off += p.halves ? align_up((size_t)p.total_rows * c->Hkv * c->d * 2) : 0;
  p.off_scale = off; off += p.halves ? align_up((size_t)p.total_rows * c->Hkv * sizeof(float)) : 0;
  p.off_rows = off; off += align_up((size_t)p.total_rows * c->Hkv * c->d * 2);
  p.off_ml = off; off += align_up((size_t)p.total_rows * c->Hkv * p.n_slots * sizeof(float2));
  p.off_o = off; off += align_up((size_t)p.total_rows * c->Hkv * p.n_slots * c->d * sizeof(float));
  p.total = off;
  return PC_OK;
}

// tensor maps of the pool's keys and values, boxes of `rows` entries (8-bit formats: whole rows; bf16: 64 columns)
bool page_maps(const pc_kv_cache* c, int rows, CUtensorMap* tm_k, CUtensorMap* tm_v) {
  const uint64_t d = (uint64_t)c->d, page = (uint64_t)c->capacity;
  const uint64_t dims[4] = {d, page, (uint64_t)c->Hkv, (uint64_t)c->B}, str[3] = {d, page * d, (uint64_t)c->Hkv * page * d};
  const uint32_t box[4] = {c->format == PC_KV_BF16 ? 64u : (uint32_t)c->d, (uint32_t)rows, 1, 1};
  if (c->format == PC_KV_BF16) return pc::make_tmap_bf16_4d(tm_k, c->k, dims, str, box) && pc::make_tmap_bf16_4d(tm_v, c->v, dims, str, box);
  return pc::make_tmap_u8_4d(tm_k, c->k, dims, str, box) && pc::make_tmap_u8_4d(tm_v, c->v, dims, str, box);
}
// entries of a box of copies: the largest power of two that divides a page, up to a tile; of pages that have no multiple of 16, one for each sequence, a tile
int box_of(int64_t page, int tile) {
  if (page % 16 != 0) return tile;
  int box = 16;
  while (box < tile && page % (2 * box) == 0) box *= 2;
  return box;
}

}  // namespace

extern "C" {

size_t pc_tree_attn_workspace_bytes(const pc_tree_attn_args* a) {
  if (a == nullptr) return 0;
  TreePlan p;
  const int sms = pc::sm100_count();
  return tree_plan(a, sms > 0 ? sms : 148, p) == PC_OK ? p.total : 0;
}

int32_t pc_tree_attn(const pc_tree_attn_args* a, void* stream) {
  if (a == nullptr) return PC_ERR_INVALID_ARG;
  TreePlan plan;
  const int sms = pc::sm100_count();
  if (int32_t rc = tree_plan(a, sms > 0 ? sms : 148, plan); rc != PC_OK) return rc;
  if (int32_t rc = check_pages(a->pages, a->table, a->table_stride, a->n_table); rc != PC_OK) return rc;
  const pc_kv_cache* const c = a->pages;
  if (!a->q || !a->out || !a->lens || !aligned(a->q, 16) || !aligned(a->out, 16) || !aligned(a->workspace, 32)) return PC_ERR_INVALID_ARG;
  if ((int64_t)a->max_len + a->w > c->capacity * a->n_table || a->parents_stride < 0) return PC_ERR_INVALID_ARG;
  if (!good_theta(a->rope_theta) || !(a->softmax_scale >= 0.0f) || !std::isfinite(a->softmax_scale)) return PC_ERR_INVALID_ARG;
  pc::CacheRows rows = {};
  if (!strides(a->q_stride, a->w, a->Hq, c->d, rows.stride)) return PC_ERR_INVALID_ARG;
  if (!a->workspace || a->workspace_bytes < plan.total) return PC_ERR_WORKSPACE;
  if (sms == 0) return PC_ERR_UNSUPPORTED;

  cudaStream_t st = static_cast<cudaStream_t>(stream);
  uint8_t* const ws = static_cast<uint8_t*>(a->workspace);
  const PhasePlan& ph = plan.phase;
  rows.q = a->q; rows.B = a->B; rows.w = a->w; rows.Hq = a->Hq; rows.Hkv = c->Hkv; rows.pos0 = a->pos0; rows.pos = a->pos;
  const double scale = a->softmax_scale > 0.0f ? (double)a->softmax_scale : 1.0 / std::sqrt((double)c->d);
  rows.scale_log2 = (float)(scale * 1.4426950408889634);
  rows.rows = ws + plan.off_rows;
  pc::TreePhase tree = {};
  tree.pages = pages_of(c, a->table, a->table_stride, a->n_table);
  tree.lens = a->lens; tree.parents = a->parents; tree.parent_stride = a->parents_stride;
  tree.max_len = a->max_len;
  tree.least_tiles = least_tiles(a->B);
  tree.turn = a->rope_theta > 0.0f;
  if (tree.turn) turns_of(a->rope_theta, c->d, tree.turns);
  tree.k = static_cast<const uint8_t*>(c->k); tree.v = static_cast<const uint8_t*>(c->v);
  tree.sees = reinterpret_cast<unsigned long long*>(ws + plan.off_sees);
  cudaError_t e = cudaSuccess;
  if (plan.rows) {
    rows.clear = reinterpret_cast<int*>(ws + plan.off_counter);
    rows.clear_too = a->clear_status ? a->status_word : nullptr;
    if (ph.wide) { rows.part_ml = reinterpret_cast<float2*>(ws + plan.off_ml); rows.n_slots = plan.n_slots; }      // (items without keys are left out)
    if (plan.halves) { rows.halves = ws + plan.off_halves; rows.half_scale = reinterpret_cast<float*>(ws + plan.off_scale); }
    e = pc::launch_tree_rows(rows, tree, c->d, st);
  } else if (a->clear_status && a->status_word) {
    e = cudaMemsetAsync(a->status_word, 0, sizeof(int), st);
  }
  pc::CacheMerge merge = {};
  merge.n_slots = plan.n_slots; merge.total_rows = (int)plan.total_rows;
  merge.part_o = reinterpret_cast<const float*>(ws + plan.off_o);
  merge.part_ml = reinterpret_cast<const float2*>(ws + plan.off_ml);
  merge.q = rows;
  merge.out = static_cast<__nv_bfloat16*>(a->out); merge.lse = a->lse;
  pc::CachePhase p = {};
  p.seqs = a->B;
  p.rows = a->w * (a->Hq / c->Hkv);
  p.Hkv = c->Hkv; p.n_keys = a->max_len + a->w; p.len = a->lens;
  p.k_scale = c->k_scale; p.v_scale = c->v_scale; p.capacity = c->capacity;
  p.n_rg = ph.n_rg; p.n_split = ph.n_split; p.n_slots = plan.n_slots; p.total_rows = (int)plan.total_rows;
  p.q = rows;
  p.rows_made = plan.rows;
  p.part_o = reinterpret_cast<float*>(ws + plan.off_o);
  p.part_ml = reinterpret_cast<float2*>(ws + plan.off_ml);
  p.status = a->status_word;
  p.wait_kcycles = pc::wait_limit_kcycles();
  p.skip_final_publication = pc::skip_final_publication();
  CUtensorMap maps[3];
  if (e == cudaSuccess) {
    const int box = box_of(c->capacity, ph.wide ? 128 : pc::few_keys(c->format, c->d, ph.brief));
    while ((1 << tree.log_box) < box) ++tree.log_box;
    tree.scales_by_four = c->capacity % 16 == 0 && aligned(c->k_scale, 16) && aligned(c->v_scale, 16);
    if (!page_maps(c, box, &maps[1], &maps[2])) { launched(e); return PC_ERR_CUDA; }
    if (ph.wide) {
      pc::WidePhase wp = {};
      wp.c = p; wp.alt = ph.alt;
      wp.half_scale = rows.half_scale;
      wp.counter = rows.clear;
      const uint64_t d = (uint64_t)c->d, R = (uint64_t)plan.total_rows;
      const uint64_t dims[4] = {d, R, (uint64_t)c->Hkv, 1}, str[3] = {d, R * d, R * d * (uint64_t)c->Hkv};
      const uint32_t row_box[4] = {64, 128, 1, 1};
      if (!pc::make_tmap_bf16_4d(&maps[0], plan.halves ? rows.halves : rows.rows, dims, str, row_box)) { launched(e); return PC_ERR_CUDA; }
      e = pc::launch_tree_wide(maps, wp, tree, c->format, c->d, sms, st);
    } else {
      e = pc::launch_tree_few(maps[1], maps[2], p, tree, ph.finish ? &merge : nullptr, ph.group, ph.brief, c->format, c->d, st);
    }
  }
  if (e != cudaSuccess || ph.finish) return launched(e);
  return launched(pc::launch_tree_merge(merge, c->d, sms, st));
}

int32_t pc_token_logprobs(const pc_token_logprobs_args* a, void* stream) {
  if (a == nullptr || a->type < PC_LOGITS_F32 || a->type > PC_LOGITS_F16) return PC_ERR_INVALID_ARG;
  const int bytes = a->type == PC_LOGITS_F32 ? 4 : 2;
  if (a->N < 1 || a->V < 1 || a->top < 0 || a->top > a->V || a->group < 0 || !a->logits || !aligned(a->logits, bytes) || a->stride < 0) return PC_ERR_INVALID_ARG;
  if (!(a->scale >= 7.8886091e-31f) || a->scale > 1.2676506e30f || (a->logprob != nullptr) != (a->tokens != nullptr)) return PC_ERR_INVALID_ARG;
  if ((a->top > 0 && (!a->top_logprob || !a->top_id)) || (a->top == 0 && !a->logprob && !a->entropy)) return PC_ERR_INVALID_ARG;
  if (a->nll != nullptr && (a->group < 1 || a->N % a->group != 0 || !a->logprob)) return PC_ERR_INVALID_ARG;
  if (a->top > PC_MOST_ALTERNATIVES || a->V > (1 << 28) || a->N > (1 << 27)) return PC_ERR_UNSUPPORTED;
  const int sms = pc::sm100_count();
  if (sms == 0) return PC_ERR_UNSUPPORTED;
  const pc::LogProb p = {a->logits, a->stride, a->N, a->V, a->top, a->group, a->scale, a->tokens, a->logprob, a->entropy, a->top_logprob, a->top_id, a->nll};
  return launched(pc::launch_token_logprobs(p, a->type, sms, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
