// Parameter blocks and launchers of the 8-bit caches and of the attention over shared and own caches (internal).
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>

namespace pc {

// Rows that go into an 8-bit cache (pc_kv_quant.cu).
struct KvWrite {
  const void *k_src, *v_src;
  long long k_stride[3], v_stride[3];            // elements: sequence (chunk), token, head
  uint8_t *k, *v;
  float *k_scale, *v_scale;
  long long capacity;
  int B, Hkv, n;                                 // append: sequences, kv-heads, tokens; gather: 1, kv-heads, entries m * k
  int at0;
  const int* at;                                 // append: [B] or null
  const int *kept, *idx;                         // gather: chunk ids [m], positions [m,Hkv,per_chunk]
  int per_chunk;
  unsigned chunk_mul, chunk_shift;               // e / per_chunk = e * chunk_mul >> chunk_shift for e < 2^28
  int* pos_out;                                  // gather: [Hkv,n] or null
  int* status;
};
cudaError_t launch_kv_quantize(const KvWrite& w, int format, int d, bool gather, cudaStream_t st);

struct KvRead {
  const uint8_t *k, *v;
  const float *k_scale, *v_scale;
  long long capacity;
  int B, Hkv, n, at0;
  const int* at;
  void *k_out, *v_out;
  bool sectors;                                  // both aligned to 32 bytes
};
cudaError_t launch_kv_dequantize(const KvRead& r, int format, int d, cudaStream_t st);

// Queries of pc_cache_attn as rows of a kv-head: row (b * w + i) * G + g is q[b, i, hkv * G + g, :], rotated and rounded to bf16
// (theta 0: as it is), in memory as rows[hkv][row][d].  The kernel for few rows makes them where it needs them and leaves them
// there for those behind it; ahead of the one for many rows a launch of its own does, and, for 8-bit codes, leaves halves: the same times a power of
// two of each row as numbers of half precision, whose inverse times scale_log2 is in half_scale.
struct CacheRows {
  const void* q;
  long long stride[3];
  int B, w, Hq, Hkv, pos0;
  const int* pos;
  float theta, scale_log2;
  void *rows, *halves;           // halves: or null
  float* half_scale;             // [Hkv,B*w*G]
  int *clear, *clear_too;        // two words and one that are set to 0, or null
  float2* part_ml;               // slots of the rows, n_slots each, that are marked as empty, or null (a phase for many rows leaves out items without keys)
  int n_slots;
};
cudaError_t launch_cache_rows(const CacheRows& p, int d, cudaStream_t st);

// What a row's result is joined from beside the caches' results that a kernel has itself: slots in memory and the new tokens' own keys.
struct CacheMerge {
  int n_slots, total_rows;
  const float* part_o;
  const float2* part_ml;
  CacheRows q;                                   // (rows in memory)
  const void *k_win, *v_win;                     // or null
  long long k_stride[3], v_stride[3];
  __nv_bfloat16* out;
  float* lse;
};
// One phase of pc_cache_attn: the rows of each of `seqs` sequences (prefix: one, all rows; own caches: B, w * G rows) over a cache.
// A split's result of a row goes to slot slot0 + split of its n_slots: the unnormalised output, and (maximum in log2 units,
// sum); a split without keys leaves (-inf, 0) and no output.
struct CachePhase {
  int seqs, rows, Hkv, n_keys;                   // n_keys: entries, or their most
  const int* len;                                // [seqs] or null: n_keys each
  const float *k_scale, *v_scale;                // [seqs,Hkv,capacity] (8-bit formats)
  long long capacity;
  int n_rg, n_split, slot0, n_slots, total_rows; // row groups of a sequence, key splits; total_rows = rows of a kv-head over all sequences
  int causal;                                    // 1 (few rows in groups of 8, bf16, one split): the entries are the new tokens themselves, token i sees 0 .. i
  CacheRows q;
  int rows_made;                                 // 1: the rows are in memory; 0: this launch makes them
  float* part_o;                                 // [Hkv,total_rows,n_slots,d]
  float2* part_ml;                               // [Hkv,total_rows,n_slots]
  int* status;
  int wait_kcycles;
  int skip_final_publication;                    // test hook of the bounded waits (see pc_debug_bounded_wait_test in pc.h)
};
// Few rows (pc_cache_few.cu), groups of 8 or 16.  finish null: every split leaves its slot.  Else the splits of a (sequence, kv-head, row
// group) are the CTAs of a cluster, and the kernel finishes its rows: its splits' results, finish's slots and the new tokens' keys.
// group: 8 or 16 rows; brief: the build for many sequences with few entries.
// maps of the cache's keys and values: boxes of few_keys() entries
int few_keys(int format, int d, bool brief);     // keys of a stage
int few_clusters(int n);                         // clusters of n CTAs that the current device runs at a time (not brief)
cudaError_t launch_cache_few(const CUtensorMap& tm_k, const CUtensorMap& tm_v, const CachePhase& p, const CacheMerge* finish, int group, bool brief,
                             int format, int d, cudaStream_t st);

// The same phase for many rows of a sequence (pc_cache_wide.cu), blocks of 128 rows.  With len, which bf16 caches do not have here, the slots are marked
// as empty ahead.
struct WidePhase {
  CachePhase c;                  // n_rg, n_split: of the blocks below
  int alt;                       // 1: the two blocks of a CTA hold the same rows and take alternate key tiles; 0: different rows
  const float* half_scale;       // [Hkv,total_rows] (8-bit formats)
  int* counter;                  // work queue, zeroed
};
// maps: rows of queries (box 64 x 128 rows; halves for 8-bit formats), keys (128, of a pair 64 entries) and values (128)
cudaError_t launch_cache_wide(const CUtensorMap* maps, const WidePhase& p, int format, int d, bool pair, int sm_count, cudaStream_t st);

// Joins the slots of a row and the new tokens' own keys.
cudaError_t launch_cache_merge(const CacheMerge& p, int d, cudaStream_t st);

}  // namespace pc
