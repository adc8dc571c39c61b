// Attention of many query rows of drafted tokens over pages (pc_tree_attn): the body of pc_cache_wide.cu on single CTAs.
//
// out = softmax over {e < len} and the ancestors of (R(p) q . k_e) scale, times v: 128 rows of a kv-head a block, two blocks an item, so that 256 rows read a page once.
// The tile that holds new tokens is masked by the rows' words of ancestors; values behind a sequence's end, which may be NaN in memory, are set to zero in
// shared memory before the product takes them.  Single CTAs, not pairs: what the pair shares is the keys, which the two blocks of an item share already.
// A tile of 128 keys takes 2.05 to 2.35 us of two blocks, the softmax of 256 rows and the matrix products one behind the other, and 1.4 of one block, the rate at
// which its copies come.  Around it 20 us that do not depend on the keys: rows kernel 5, the CTA's start, slots and their join 6 to 10.
// Measured, 32/8 heads of 128, bf16: 64 tokens of one sequence over 32768 entries (134 MB) 51 to 57 us; 40 tokens of each of 16 sequences of up to 12000 entries
// 134 to 152 (160 rows cost what 256 do).  Codes: one stage of converted keys, 4 to 5 us a tile.
#include "pc_wide.cuh"

namespace pc {

template <int D, int FMT>
__global__ void __launch_bounds__(flash::NT2, 1)
tree_wide_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                 const __grid_constant__ WidePhase prm, const __grid_constant__ TreePhase tree) {
  wide::wide_body<D, FMT, false>(tm_q, tm_k, tm_v, prm, tree);
}

namespace {

template <int D, int FMT>
cudaError_t wide_t(const CUtensorMap* maps, const WidePhase& p, const TreePhase& t, int sm_count, cudaStream_t st) {
  constexpr int SMEM = wide::smem_bytes<D, FMT, false, TreePhase>();
  static_assert(SMEM <= 232448, "shared memory of a CTA");
  if (cudaError_t e = cudaFuncSetAttribute(tree_wide_kernel<D, FMT>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM); e != cudaSuccess) return e;
  const long long n_items = (long long)p.c.seqs * p.c.Hkv * p.c.n_rg * p.c.n_split;
  return launch_chained(tree_wide_kernel<D, FMT>, dim3((unsigned)(n_items < sm_count ? n_items : sm_count)), dim3(flash::NT2), SMEM, st, 1, maps[0], maps[1], maps[2],
                        p, t);
}
template <int D>
cudaError_t wide_d(const CUtensorMap* maps, const WidePhase& p, const TreePhase& t, int format, int sm_count, cudaStream_t st) {
  return format == FMT_BF16   ? wide_t<D, FMT_BF16>(maps, p, t, sm_count, st)
         : format == FMT_INT8 ? wide_t<D, FMT_INT8>(maps, p, t, sm_count, st)
                              : wide_t<D, FMT_E4M3>(maps, p, t, sm_count, st);
}

}  // namespace

cudaError_t launch_tree_wide(const CUtensorMap* maps, const WidePhase& p, const TreePhase& t, int format, int d, int sm_count, cudaStream_t st) {
  return d == 128 ? wide_d<128>(maps, p, t, format, sm_count, st) : wide_d<64>(maps, p, t, format, sm_count, st);
}

}  // namespace pc
