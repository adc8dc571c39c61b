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
#include "pc_wide.cuh"

namespace pc {

template <int D, int FMT, bool PAIR>
__global__ void __launch_bounds__(flash::NT2, 1)
cache_wide_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                  const __grid_constant__ WidePhase prm) {
  wide::wide_body<D, FMT, PAIR>(tm_q, tm_k, tm_v, prm, wide::NoTree{});
}

namespace {

template <int D, int FMT, bool PAIR>
cudaError_t wide_t(const CUtensorMap* maps, const WidePhase& p, int sm_count, cudaStream_t st) {
  using C = flash::Cfg<D, PAIR>;
  constexpr int SMEM = wide::smem_bytes<D, FMT, PAIR, wide::NoTree>();
  if (cudaError_t e = cudaFuncSetAttribute(cache_wide_kernel<D, FMT, PAIR>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM); e != cudaSuccess) return e;
  const long long n_items = (long long)p.c.seqs * p.c.Hkv * p.c.n_rg * p.c.n_split;
  const int units = sm_count / C::NCTA;
  if (units < 1) return cudaErrorInvalidConfiguration;
  return launch_chained(cache_wide_kernel<D, FMT, PAIR>, dim3((unsigned)((n_items < units ? (int)n_items : units) * C::NCTA)), dim3(flash::NT2), SMEM, st, C::NCTA,
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
