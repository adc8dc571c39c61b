// Parameter blocks and launchers of the paged caches, the attention of drafted tokens over them, and the log probabilities (internal).
#pragma once
#include "pc_cache.h"

namespace pc {

// A position turns pair t by theta^(-2t/d) / (2 pi) = coarse[t / 8] * fine[t % 8] of a full turn; the host computes these in fp64.
struct Turns { double coarse[8], fine[8]; };

// Pages of the sequences: entry e of sequence b is entry e % page of page table[b * stride + e / page].
struct Pages {
  const int* table;
  long long stride;
  int n_table, page, n_pages;                    // pages of a sequence, entries of a page, pages of the pool
  unsigned mul, shift;                           // e / page = e * mul >> shift for 0 <= e < 2^28
};

// New rows into pages (pc_page_append.cu).
struct PageWrite {
  const void *k_src, *v_src;
  long long k_stride[3], v_stride[3];            // elements: sequence, token, head
  uint8_t *k, *v;
  float *k_scale, *v_scale;
  Pages pages;
  int B, Hkv, n, n_src;                          // sequences, kv-heads, entries to be written of each, tokens of the source
  int at0, pos0;
  const int *at, *pos, *count, *pick, *parents;  // each [B] or null; pick, parents [B,n] through a stride
  long long pick_stride, parent_stride;
  int turn;                                      // 0: keys as they are
  Turns turns;
  int* status;
};
cudaError_t launch_page_append(const PageWrite& w, int format, int d, cudaStream_t st);

// What the attention of drafted tokens needs beside a phase of pc_cache_attn: its caches are pages, and the last w entries of a
// sequence are the new tokens, each of which sees its ancestors.
struct TreePhase {
  Pages pages;
  const int* lens;                               // [B] entries before the new tokens; negative: no such sequence
  const int* parents;                            // [B,w] through a stride, or null: each token the child of the one before
  long long parent_stride;
  int max_len;                                   // of lens
  int log_box;                                   // of the entries of a tensor map's box: a divisor of a page; of a page that has no multiple of 16 entries a tile
  int scales_by_four;                           // 8-bit formats: four scales of a page are 16 bytes at a multiple of 16
  int least_tiles;                               // many rows: of a piece of a sequence's keys
  int turn;                                      // 0: queries as they are
  Turns turns;
  const uint8_t *k, *v;                          // the pool
  unsigned long long* sees;                      // [B,w], written by the launch for the rows: bit j: token j is seen; 0: the token is not there
};
// The kernel for few rows (pc_tree_few.cu): as launch_cache_few(), p.len the entries before the new tokens, maps of the pool with boxes of 2^t.log_box entries.
cudaError_t launch_tree_few(const CUtensorMap& tm_k, const CUtensorMap& tm_v, const CachePhase& p, const TreePhase& t, const CacheMerge* finish, int group,
                            bool brief, int format, int d, cudaStream_t st);
// The kernel for many rows (pc_tree_wide.cu): as launch_cache_wide() on single CTAs.
cudaError_t launch_tree_wide(const CUtensorMap* maps, const WidePhase& p, const TreePhase& t, int format, int d, int sm_count, cudaStream_t st);
// Joins the slots of a row (pc_tree_prepare.cu).
cudaError_t launch_tree_merge(const CacheMerge& p, int d, int sm_count, cudaStream_t st);
// Rows into memory, rotated, and t.sees; clears as cache_rows_kernel does (pc_tree_prepare.cu).
cudaError_t launch_tree_rows(const CacheRows& p, const TreePhase& t, int d, cudaStream_t st);

}  // namespace pc
