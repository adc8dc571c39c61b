// Attention of few query rows over a cache in bf16 or 8 bits (pc_cache_attn): up to 16 rows of a kv-head at a time.
//
// With keys, then head-dim columns, as the 16 rows of a product and the query rows as its 8 columns,
//     S^T [16 keys x 8 rows] = K Q^T,      O^T [16 of d x 8 rows] += V^T P^T,
// a step computes what its rows need (8 or 16 of them) and no more, and the codes of a cache go from shared memory into
// the operands' registers on their way: the operand layout asks a thread for 4 consecutive elements of a key at a time (for V: of
// 4 keys at a time, so that bytes of two keys are interleaved), and which elements of d they are is free as long as Q has
// them in the same order.  int8 and e4m3 become half precision exactly; the scale of a key multiplies its row of S^T, the scale
// of a value its probability, so nothing that a cache holds is rounded.  Queries are bf16 numbers; times a power of two of their row
// they are halves too (elements 2^-22 below the row's largest lose bits).  Probabilities are rounded to half precision (11 bits,
// bf16 caches: bf16, 8 bits) beside sums and accumulators in fp32; half precision has a short range, so they are held relative to the
// largest product of probability and scale of their row (cw below), raised together with the reference maximum.
//
// Bound by reading the cache, and, with 16 rows of 8-bit codes, by the instructions that make operands of them.  A warp takes 16 keys (a
// unit) at a time on its own, with its own maximum, sum and accumulators, and waits for nobody but the copies; a producer warp keeps
// the ring full.  The maximum is looked at with one vote per 8 rows and raised only where a logit exceeds it by 2^8.  The warps'
// results are added in shared memory, the splits' through distributed shared memory or by the merge kernel.
// Measured, 32/8 heads of 128: 64 sequences over 16384 int8 entries each, 2.2 GB, 340 us = 6.5 TB/s, in a loop at the power cap (1.56 GHz) 386 = 5.7 TB/s;
// one sequence 15.3 (splits as slots; rows, first copies, a tile, join and merge: latency); 16 rows a kv-head over 8000 entries 251 us, bf16 312 =
// 6.7 TB/s.  28 rows, two groups, of codes at head size 64 (23 sequences of 4 tokens, up to 5000 e4m3 entries) 22: chains of dependent
// instructions of few warps.
#include "pc_few.cuh"

namespace pc {

template <class C>
__global__ void __launch_bounds__(C::THREADS, C::CTAS)
cache_few_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CachePhase prm,
                 const __grid_constant__ CacheMerge fin, const int finish) {
  few::few_body<C>(tm_k, tm_v, prm, fin, finish, few::NoTree{});
}

namespace {

using few::Few;

template <class C>
cudaError_t few_t(const CUtensorMap& tm_k, const CUtensorMap& tm_v, const CachePhase& p, const CacheMerge* finish, cudaStream_t st) {
  constexpr int SMEM = few::smem_bytes<C>();
  static_assert(C::CTAS * (SMEM + 1024) <= 233472, "CTAs per SM");
  if (cudaError_t e = cudaFuncSetAttribute(cache_few_kernel<C>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM); e != cudaSuccess) return e;
  return launch_chained(cache_few_kernel<C>, dim3((unsigned)((long long)p.seqs * p.Hkv * p.n_rg * p.n_split)), dim3(C::THREADS), SMEM, st,
                        finish ? p.n_split : 1, tm_k, tm_v, p, finish ? *finish : CacheMerge{}, finish != nullptr ? 1 : 0);
}
template <int D, int FMT>
cudaError_t few_n(const CUtensorMap& tm_k, const CUtensorMap& tm_v, const CachePhase& p, const CacheMerge* finish, int group, bool brief, cudaStream_t st) {
  if (group == 8)
    return brief ? few_t<Few<D, FMT, 1, true>>(tm_k, tm_v, p, finish, st) : few_t<Few<D, FMT, 1, false>>(tm_k, tm_v, p, finish, st);
  return brief ? few_t<Few<D, FMT, 2, true>>(tm_k, tm_v, p, finish, st) : few_t<Few<D, FMT, 2, false>>(tm_k, tm_v, p, finish, st);
}
template <int D>
cudaError_t few_causal(const CUtensorMap& tm_k, const CUtensorMap& tm_v, const CachePhase& p, const CacheMerge* finish, bool brief, cudaStream_t st) {
  return brief ? few_t<Few<D, FMT_BF16, 1, true, true>>(tm_k, tm_v, p, finish, st) : few_t<Few<D, FMT_BF16, 1, false, true>>(tm_k, tm_v, p, finish, st);
}
template <int D>
cudaError_t few_d(const CUtensorMap& tm_k, const CUtensorMap& tm_v, const CachePhase& p, const CacheMerge* finish, int group, bool brief, int format,
                  cudaStream_t st) {
  if (p.causal) return few_causal<D>(tm_k, tm_v, p, finish, brief, st);
  return format == FMT_INT8   ? few_n<D, FMT_INT8>(tm_k, tm_v, p, finish, group, brief, st)
         : format == FMT_E4M3 ? few_n<D, FMT_E4M3>(tm_k, tm_v, p, finish, group, brief, st)
                              : few_n<D, FMT_BF16>(tm_k, tm_v, p, finish, group, brief, st);
}
template <class C>
int clusters_t(int n) {
  constexpr int SMEM = few::smem_bytes<C>();
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)n);
  cfg.blockDim = dim3(C::THREADS);
  cfg.dynamicSmemBytes = SMEM;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim = {(unsigned)n, 1, 1};
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int fit = 0;
  if (cudaFuncSetAttribute(cache_few_kernel<C>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM) != cudaSuccess ||
      cudaOccupancyMaxActiveClusters(&fit, cache_few_kernel<C>, &cfg) != cudaSuccess) {
    cudaGetLastError();
    return 0;
  }
  return fit;
}
template <bool SHORT>
int keys_t(int format, int d) {
  if (format == FMT_BF16) return d == 128 ? Few<128, FMT_BF16, 1, SHORT>::KEYS : Few<64, FMT_BF16, 1, SHORT>::KEYS;
  return d == 128 ? Few<128, FMT_INT8, 1, SHORT>::KEYS : Few<64, FMT_INT8, 1, SHORT>::KEYS;
}

}  // namespace

int few_clusters(int n) { return clusters_t<Few<128, FMT_INT8, 2, false>>(n); }      // (all builds take half an SM's shared memory)
int few_keys(int format, int d, bool brief) { return brief ? keys_t<true>(format, d) : keys_t<false>(format, d); }
cudaError_t launch_cache_few(const CUtensorMap& tm_k, const CUtensorMap& tm_v, const CachePhase& p, const CacheMerge* finish, int group, bool brief,
                             int format, int d, cudaStream_t st) {
  return d == 128 ? few_d<128>(tm_k, tm_v, p, finish, group, brief, format, st) : few_d<64>(tm_k, tm_v, p, finish, group, brief, format, st);
}

}  // namespace pc
