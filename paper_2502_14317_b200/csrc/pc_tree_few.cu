// Attention of few query rows of drafted tokens over pages (pc_tree_attn): the body of pc_cache_few.cu, up to 16 rows of a kv-head at a time.
//
// A box of the producer's copies is a page, or as much of one as a tile has: a lane issues each.  The ids of 64 pages lie in its warp's registers; looked up tile by tile,
// a load that the copies wait for, 64 sequences of up to 16384 int8 entries took 1.7 times as long.  Small boxes are slower than whole tiles: over 16400 bf16
// entries 25.5 us with pages of 16, 20.9 with pages of 64 (cp.async of 16 bytes in place of the boxes 30.2).  The last w entries of a sequence are its new tokens;
// a unit that holds any is masked by the rows' words of ancestors, which every CTA makes itself from the parents (some 400 cycles, under the first copies).
//
// Bound by reading the pages, with few sequences by latencies: 64 sequences of up to 16384 int8 entries, 8145 on average (1.1 GB), 32/8 heads of 128, 214 to 230 us = 5.1 to 4.8 TB/s (the
// copies' conversions and an end in which only the longest sequences are left); one sequence of 16400 bf16 entries (67 MB) 20 us: some 8 for the start, rows
// and join, then a tile at a time.
#include "pc_few.cuh"

namespace pc {

template <class C>
__global__ void __launch_bounds__(C::THREADS, C::CTAS)
tree_few_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CachePhase prm,
                const __grid_constant__ CacheMerge fin, const int finish, const __grid_constant__ TreePhase tree) {
  few::few_body<C>(tm_k, tm_v, prm, fin, finish, tree);
}

namespace {

template <class C>
cudaError_t few_t(const CUtensorMap& tm_k, const CUtensorMap& tm_v, const CachePhase& p, const TreePhase& t, const CacheMerge* finish, cudaStream_t st) {
  constexpr int SMEM = few::smem_bytes<C>();
  static_assert(C::CTAS * (SMEM + 1024) <= 233472, "CTAs per SM");
  if (cudaError_t e = cudaFuncSetAttribute(tree_few_kernel<C>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM); e != cudaSuccess) return e;
  return launch_chained(tree_few_kernel<C>, dim3((unsigned)((long long)p.seqs * p.Hkv * p.n_rg * p.n_split)), dim3(C::THREADS), SMEM, st,
                        finish ? p.n_split : 1, tm_k, tm_v, p, finish ? *finish : CacheMerge{}, finish != nullptr ? 1 : 0, t);
}
template <int D, int FMT>
cudaError_t few_n(const CUtensorMap& tm_k, const CUtensorMap& tm_v, const CachePhase& p, const TreePhase& t, const CacheMerge* finish, int group, bool brief,
                  cudaStream_t st) {
  if (group == 8)
    return brief ? few_t<few::Few<D, FMT, 1, true, false, true>>(tm_k, tm_v, p, t, finish, st)
                 : few_t<few::Few<D, FMT, 1, false, false, true>>(tm_k, tm_v, p, t, finish, st);
  return brief ? few_t<few::Few<D, FMT, 2, true, false, true>>(tm_k, tm_v, p, t, finish, st)
               : few_t<few::Few<D, FMT, 2, false, false, true>>(tm_k, tm_v, p, t, finish, st);
}
template <int D>
cudaError_t few_d(const CUtensorMap& tm_k, const CUtensorMap& tm_v, const CachePhase& p, const TreePhase& t, const CacheMerge* finish, int group, bool brief,
                  int format, cudaStream_t st) {
  return format == FMT_INT8   ? few_n<D, FMT_INT8>(tm_k, tm_v, p, t, finish, group, brief, st)
         : format == FMT_E4M3 ? few_n<D, FMT_E4M3>(tm_k, tm_v, p, t, finish, group, brief, st)
                              : few_n<D, FMT_BF16>(tm_k, tm_v, p, t, finish, group, brief, st);
}

}  // namespace

cudaError_t launch_tree_few(const CUtensorMap& tm_k, const CUtensorMap& tm_v, const CachePhase& p, const TreePhase& t, const CacheMerge* finish, int group,
                            bool brief, int format, int d, cudaStream_t st) {
  return d == 128 ? few_d<128>(tm_k, tm_v, p, t, finish, group, brief, format, st) : few_d<64>(tm_k, tm_v, p, t, finish, group, brief, format, st);
}

}  // namespace pc
