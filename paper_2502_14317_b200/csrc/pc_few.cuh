// The body of the kernels for few query rows over a cache in bf16 or 8 bits: pc_cache_few.cu (caches of pc_cache_attn) and pc_tree_few.cu (pages, drafted
// tokens).  What it does and what bounds it: pc_cache_few.cu.
#pragma once
#include "pc_cache_finish.cuh"
#include "pc_cache_rows.cuh"
#include "pc_kernels.h"
#include "pc_kv8.cuh"
#include "pc_tree_rows.cuh"
#include <cfloat>

namespace pc {
namespace few {

// CAUSAL: the entries are the new tokens themselves, token i sees 0 .. i.
// TREE: the cache is pages, the last w entries of a sequence are its new tokens, each of which sees its ancestors.
// SHORT: for many sequences with few entries, four CTAs per SM (16 rows: three) instead of two, with half the ring: three consumer warps (16 rows at head
// size 64: four) instead of seven (16 rows at 128: five), stages of half the size (codes at head size 64, 16 KB: the same, and half as many).
template <int D_, int FMT_, int NT8_, bool SHORT_, bool CAUSAL_ = false, bool TREE_ = false>
struct Few {
  static constexpr int D = D_, FMT = FMT_, NT8 = NT8_;
  static constexpr bool CAUSAL = CAUSAL_, TREE = TREE_;
  static constexpr int EB = FMT == FMT_BF16 ? 2 : 1;            // bytes of an element
  static constexpr int ROWB = D * EB, BOXES = ROWB > 128 ? 2 : 1, BOXB = ROWB / BOXES, EPB = BOXB / EB;
  // Consumer warps: with the producers 16 warps an SM (15 of the short build for 16 rows), 128 registers a thread, or for 16 rows at head size 128 12 and 168.  (16 rows at head size 64, 12 / 16
  // warps, us: 64 sequences of 2000 e4m3 entries, 8 kv-heads 60.5 / 55.2, of 8000 146.7 / 133.8, int8 164.2 / 150.8, bf16 167.5 / 165.2; 23 of up to 5000 22.4 / 21.4.)
  static constexpr int CTAS = SHORT_ ? (NT8 == 1 ? 4 : 3) : 2, WARPS = (NT8 == 1 || D == 64 ? 16 : 12) / CTAS - 1;
  static constexpr int UNITS = (ROWB == 256 ? 4 : 8) / (SHORT_ && ROWB != 64 ? 2 : 1);             // of a stage
  static constexpr int KEYS = 16 * UNITS, HALF_BYTES = KEYS * ROWB, STAGE_BYTES = 2 * HALF_BYTES;
  static constexpr int NS = (SHORT_ ? 49152 : 98304) / STAGE_BYTES;
  static constexpr int N = 8 * NT8, KST = D / 16, MT = D / 16;
  static constexpr int THREADS = 32 * (WARPS + 1);
  static constexpr int OFF_SCALE = NS * STAGE_BYTES, OFF_Q = OFF_SCALE + (EB == 1 ? NS * 2 * KEYS * 4 : 0), OFF_ROWS = OFF_Q + KST * NT8 * 256,
                       OFF_MISC = OFF_ROWS + N * D * 2;
  static constexpr int CPT = BOXB / 64, EPC = 16 / EB, KPC = EPC / 4;      // 16-byte chunks of a thread in a box row, their elements and k-steps
  static_assert(WARPS * N * D * 4 <= OFF_SCALE, "partial results of the warps go into the ring");
};
template <class C>
struct __align__(16) FewMisc {
  uint64_t full[C::NS], empty[C::NS];
  int abort_flag;                                               // these two words stay adjacent (bounded waits)
  int wait_kcycles;
  int odd;                                                      // causal: a value that is no number
  float qs[C::N];                                               // scale of a row's logits, in log2 units
  float2 ml[C::WARPS][C::N], all[C::N];                         // maximum and sum of a row: of a warp, of the CTA
};
// TREE: beside it
template <class C>
struct __align__(16) TreeMisc {
  unsigned long long sees[C::N];                                // the new tokens that a row sees, 0: the row is not there
  unsigned long long odd;                                       // new tokens with a value that is no number
};
struct NoTree {};                                              // in the place of TreePhase
template <class C>
constexpr int smem_bytes() { return C::OFF_MISC + (int)sizeof(FewMisc<C>) + (C::TREE ? (int)sizeof(TreeMisc<C>) : 0); }
enum { WF_FULL = 411, WF_EMPTY };

__device__ __forceinline__ uint32_t full_par(uint32_t n) { return n & 1u; }
__device__ __forceinline__ uint32_t free_par(uint32_t n) { return (n & 1u) ^ 1u; }

template <int FMT>
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (FMT == FMT_BF16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
template <int FMT>
__device__ __forceinline__ uint32_t pack_p(float lo, float hi) {
  if constexpr (FMT == FMT_BF16) return pack_bf16x2(lo, hi);
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float max_over_keys(float x) {
#pragma unroll
  for (int o = 4; o < 32; o <<= 1) x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
  return x;
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const float* src, bool there) {      // zero where there is no entry
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_arrive(uint64_t* bar) {                             // once this thread's copies have landed
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
template <int E>
__device__ __forceinline__ void ld_cluster(uint32_t addr, float (&x)[E]) {
  if constexpr (E == 4)
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]) : "r"(addr) : "memory");
  else
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(x[0]), "=f"(x[1]) : "r"(addr) : "memory");
}
// A wait that gives up pauses first: the warps are about to leave their results in the ring, into which copies may still be on their way.  (A warp
// that has seen all its tiles has seen every copy land.)
static __device__ __noinline__ bool wait_over(long long t0, volatile int* abort_flag, int* status, int where) {
  if (!mbar_wait_over(t0, abort_flag, status, where)) return false;
  abort_grace_pause(abort_flag);
  return true;
}
__device__ __forceinline__ bool ring_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag, int* status, int where) {
  return mbar_wait_ns<SPIN_BACKOFF_NS, wait_over>(bar, parity, abort_flag, status, where);
}

template <class C, class T>
__device__ __forceinline__ void few_body(const CUtensorMap& tm_k, const CUtensorMap& tm_v, const CachePhase& prm, const CacheMerge& fin, const int finish,
                                         [[maybe_unused]] const T& tr) {
  constexpr int D = C::D, FMT = C::FMT, NT8 = C::NT8, N = C::N, KEYS = C::KEYS, NS = C::NS, E = D / 32;
  constexpr bool Q8 = FMT != FMT_BF16;
  extern __shared__ __align__(1024) uint8_t smem[];
  FewMisc<C>& mi = *reinterpret_cast<FewMisc<C>*>(smem + C::OFF_MISC);
  [[maybe_unused]] TreeMisc<C>& tm = *reinterpret_cast<TreeMisc<C>*>(smem + C::OFF_MISC + sizeof(FewMisc<C>));
  volatile int* const abort_flag = &mi.abort_flag;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  int x = blockIdx.x;
  const int split = x % prm.n_split; x /= prm.n_split;          // (finish: the rank in the cluster)
  const int rg = x % prm.n_rg; x /= prm.n_rg;
  const int hkv = x % prm.Hkv, seq = x / prm.Hkv;

  if (tid == C::WARPS * 32) {
    const int hook = prm.skip_final_publication != 0 ? 1 : 0;    // test hook: an arrival that nobody makes, so that the waits for copies run out
    for (int i = 0; i < NS; ++i) { mbar_init(&mi.full[i], (Q8 ? 33 : 1) + hook); mbar_init(&mi.empty[i], C::WARPS); }
    mi.abort_flag = 0;
    mi.wait_kcycles = prm.wait_kcycles;
    mi.odd = 0;
    if constexpr (C::TREE) tm.odd = 0;
    fence_mbar_init();
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
  }
  auto turner = [&]() {
    if constexpr (C::TREE) return TreeTurner<D>(tr, lane);
    else return RowTurner<D>(prm.rows_made ? 0.0f : prm.q.theta, lane);
  }();
  __syncthreads();
  chain();
  const int entries = prm.len != nullptr ? __ldg(prm.len + seq) : prm.n_keys;          // TREE: before the new tokens
  const int row0 = seq * prm.rows + rg * N, n_rows = prm.rows - rg * N < N ? prm.rows - rg * N : N;      // rows of the kv-head
  const size_t part0 = ((size_t)hkv * prm.total_rows + row0) * prm.n_slots + prm.slot0 + split;

  int n, j0, nt;                                                 // entries of this sequence; tiles j0 .. j0 + nt - 1 of this split
  auto share = [&]() {
    if constexpr (C::TREE) {
      n = tree_entries(tr, prm.q.w, entries);
      if (tid == 0 && n < 0) { if (prm.status) atomicCAS(prm.status, 0, 422); }
      n = n < 0 ? 0 : n;
    } else {
      n = entries < 0 ? 0 : entries > prm.n_keys ? prm.n_keys : entries;
    }
    const int n_all = (n + KEYS - 1) / KEYS;
    j0 = (int)((long long)n_all * split / prm.n_split);
    nt = (int)((long long)n_all * (split + 1) / prm.n_split) - j0;
  };
  // TREE: a lane of the producer warp has a box of a tile's copies: which of the keys' or the values', or none (KEYS)
  [[maybe_unused]] int lane_box = C::KEYS, lane_values = 0, lane_col = 0, lane_to = 0;
  if constexpr (C::TREE) {
    const int part = lane * (1 << tr.log_box) / KEYS;            // columns of the keys, columns of the values
    if (part < 2 * C::BOXES) {
      lane_box = lane - part * (KEYS >> tr.log_box);
      lane_values = part / C::BOXES;
      lane_col = part % C::BOXES * C::EPB;
      lane_to = lane_values * C::HALF_BYTES + (part % C::BOXES * KEYS + (lane_box << tr.log_box)) * C::BOXB;
    }
  }
  // pages of the table, 64 at a time in the producer warp's registers, the second half on its way while the first is used
  [[maybe_unused]] int ids = -1, ids_next = -1, ids_first = 0;
  [[maybe_unused]] auto ids_at = [&](int first) {
    if constexpr (C::TREE) {
      const int which = first + lane;
      return n > 0 && which <= page_of(tr.pages, n - 1) ? __ldg(tr.pages.table + seq * tr.pages.stride + which) : -1;
    }
    return -1;
  };
  [[maybe_unused]] auto id_of = [&](int which) {                // of a page of the present tile; the whole warp calls
    const int at = which - ids_first, x = __shfl_sync(0xFFFFFFFFu, ids, at & 31);
    if (!__any_sync(0xFFFFFFFFu, at >= 32)) return x;             // (does not wait for what is still on its way)
    const int y = __shfl_sync(0xFFFFFFFFu, ids_next, at & 31);
    return at < 32 ? x : y;
  };
  // copies of tile i into its stage; the whole producer warp calls
  auto load = [&](int i) {
    const int st = i % NS, key = (j0 + i) * KEYS;
    if constexpr (C::TREE) {
      const int box = 1 << tr.log_box, some = (n - key + box - 1) >> tr.log_box, boxes = some < KEYS >> tr.log_box ? some : KEYS >> tr.log_box;   // with entries
      const int first = page_of(tr.pages, key);
      if (first - ids_first >= 32) {
        ids_first += 32;
        ids = ids_next;
        ids_next = ids_at(ids_first + 32);
      }
      const int e = key + (lane_box << tr.log_box), which = lane_box < boxes ? page_of(tr.pages, e) : first, id = id_of(which);
      if (lane == 0) mbar_arrive_expect_tx(&mi.full[st], 2 * C::ROWB * boxes << tr.log_box);
      __syncwarp();
      if (lane_box < boxes)
        tma_load_4d(smem + st * C::STAGE_BYTES + lane_to, lane_values ? &tm_v : &tm_k, &mi.full[st], lane_col, e - which * tr.pages.page, hkv,
                    page_checked(tr.pages, id, prm.status));
    } else if (lane == 0) {
      mbar_arrive_expect_tx(&mi.full[st], C::STAGE_BYTES);
#pragma unroll
      for (int b = 0; b < C::BOXES; ++b) {
        tma_load_4d(smem + st * C::STAGE_BYTES + b * KEYS * C::BOXB, &tm_k, &mi.full[st], b * C::EPB, key, hkv, seq);
        tma_load_4d(smem + st * C::STAGE_BYTES + C::HALF_BYTES + b * KEYS * C::BOXB, &tm_v, &mi.full[st], b * C::EPB, key, hkv, seq);
      }
    }
    if constexpr (Q8) {
      const uint32_t dst = smem_u32(smem + C::OFF_SCALE) + st * (2 * KEYS * 4);
      if constexpr (C::TREE) {
        if (tr.scales_by_four) {                                 // (four entries lie in one page)
          const int e = key + 4 * lane, which = page_of(tr.pages, e < n ? e : key), id = id_of(which);
          const bool there = e < n && id >= 0 && id < tr.pages.n_pages;
          if (4 * lane < KEYS) {
            const size_t from = there ? ((size_t)id * prm.Hkv + hkv) * tr.pages.page + (e - which * tr.pages.page) : 0;
            cp_async16(dst + lane * 16, prm.k_scale + from, there);
            cp_async16(dst + KEYS * 4 + lane * 16, prm.v_scale + from, there);
          }
          cp_async_arrive(&mi.full[st]);
          __syncwarp();
          return;
        }
      }
      const size_t at = ((size_t)seq * prm.Hkv + hkv) * prm.capacity;
      for (int k = lane; k < KEYS; k += 32) {
        bool there = key + k < n;
        size_t e = at + (there ? key + k : 0);
        if constexpr (C::TREE) {
          const int which = there ? page_of(tr.pages, key + k) : 0, id = there ? __ldg(tr.pages.table + seq * tr.pages.stride + which) : -1;
          there = id >= 0 && id < tr.pages.n_pages;
          e = there ? ((size_t)id * prm.Hkv + hkv) * tr.pages.page + (key + k - which * tr.pages.page) : 0;
        }
        cp_async4(dst + k * 4, prm.k_scale + e, there);
        cp_async4(dst + (KEYS + k) * 4, prm.v_scale + e, there);
      }
      cp_async_arrive(&mi.full[st]);
    }
    __syncwarp();
  };

  if (warp == C::WARPS) {
    share();
    if constexpr (C::TREE) {
      ids_first = page_of(tr.pages, j0 * KEYS);
      ids = ids_at(ids_first);
      ids_next = ids_at(ids_first + 32);
    }
    for (int i = 0; i < NS && i < nt; ++i) load(i);
  } else {
    // ---- the rows' queries: as they are, and as operands in the order in which the threads hold their keys
    [[maybe_unused]] Seen seen;
    if constexpr (C::TREE) seen = tree_seen(tr.parents == nullptr ? nullptr : tr.parents + seq * tr.parent_stride, prm.q.w, lane);
    for (int r = warp; r < N; r += C::WARPS) {
      uint32_t q[E / 2] = {};
      if constexpr (C::TREE) {
        const unsigned long long sees = r < n_rows ? seen.of((row0 + r) / (prm.q.Hq / prm.q.Hkv) % prm.q.w) : 0;
        if (lane == 0) tm.sees[r] = sees;
        turner.place(prm.q, seq, entries, __popcll(sees));
      }
      if (r < n_rows) {
        turner.row(prm.q, prm.rows_made != 0, hkv, row0 + r, lane, q);
        if (finish) RowTurner<D>::store(smem + C::OFF_ROWS, r, lane, q);
        else if (split == 0 && !prm.rows_made) RowTurner<D>::store(prm.q.rows, (size_t)hkv * prm.total_rows + row0 + r, lane, q);
      }
      float qs = prm.q.scale_log2;
      if constexpr (Q8) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < E / 2; ++i) m = __vmaxu2(m, q[i] & 0x7FFF7FFFu);
        float inv;
        const float f = row_factor(__reduce_max_sync(0xFFFFFFFFu, max(m & 0xFFFFu, m >> 16)), inv);
        qs *= inv;
#pragma unroll
        for (int i = 0; i < E / 2; ++i) q[i] = pack_p<FMT>(__uint_as_float(q[i] << 16) * f, __uint_as_float(q[i] & 0xFFFF0000u) * f);
      }
#pragma unroll
      for (int i = 0; i < E / 2; ++i) {
        const int d = E * lane + 2 * i, b = d / C::EPB, in = d % C::EPB, chunk = in / C::EPC, t = in % C::EPC / 4;
        const int ks = (b * C::CPT + chunk % C::CPT) * C::KPC + t, a = chunk / C::CPT;
        reinterpret_cast<uint32_t*>(smem + C::OFF_Q)[2 * ((ks * NT8 + r / 8) * 32 + (r % 8) * 4 + a) + (d % 4) / 2] = q[i];
      }
      if (lane == 0) mi.qs[r] = r < n_rows ? qs : 0.0f;
    }
    share();
  }
  if (nt == 0) {                                                 // nothing for this split
    if (!finish) {
      if (tid < n_rows) prm.part_ml[part0 + (size_t)tid * prm.n_slots] = make_float2(-INFINITY, 0.0f);
      return;
    }
    if (tid < N) mi.all[tid] = make_float2(-INFINITY, 0.0f);
  } else {
  __syncthreads();

  if (warp == C::WARPS) {
    int i = NS < nt ? NS : nt;
    for (; i < nt && !*abort_flag; ++i) {
      if (!ring_wait(&mi.empty[i % NS], free_par(i / NS), abort_flag, prm.status, WF_EMPTY)) break;
      load(i);
    }
    for (int k = i > NS ? i - NS : 0; k < i; ++k) mbar_wait_drain(&mi.full[k % NS], full_par(k / NS), abort_flag);   // every copy has landed before exit
  } else {
    // ================================================================ a warp: 16 keys at a time
    const int g = lane >> 2, a = lane & 3;
    uint2 qf[C::KST][NT8];
#pragma unroll
    for (int ks = 0; ks < C::KST; ++ks)
#pragma unroll
      for (int t = 0; t < NT8; ++t) qf[ks][t] = reinterpret_cast<const uint2*>(smem + C::OFF_Q)[(ks * NT8 + t) * 32 + lane];
    // per row pair (2 a, 2 a + 1) of each 8 rows: reference maximum (log2 units), sum over this thread's keys, scale of the weights
    float m[NT8][2], l[NT8][2], cw[NT8][2], qs[NT8][2], acc[C::MT][NT8][4];
#pragma unroll
    for (int t = 0; t < NT8; ++t)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        m[t][e] = -FLT_MAX; l[t][e] = 0.0f; cw[t][e] = 0x1p110f; qs[t][e] = mi.qs[8 * t + 2 * a + e];
      }
#pragma unroll
    for (int j = 0; j < C::MT; ++j)
#pragma unroll
      for (int t = 0; t < NT8; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][t][e] = 0.0f;
    // causal: a row sees the new tokens up to its own
    [[maybe_unused]] int own[NT8][2];
    if constexpr (C::CAUSAL) {
      const int G = prm.q.Hq / prm.q.Hkv;
#pragma unroll
      for (int t = 0; t < NT8; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e) own[t][e] = (row0 + 8 * t + 2 * a + e) / G % prm.q.w;
    }
    // Places of this thread's chunks in a unit, whose rows begin at a multiple of 16: the swizzle of a row goes by its last bits.
    // K: chunk a CPT + h of keys g and g + 8;  V: chunk g of keys 2 a + e and 2 a + e + 8.
    uint32_t k_at[C::CPT], v_at[2];
#pragma unroll
    for (int h = 0; h < C::CPT; ++h) k_at[h] = g * C::BOXB + (((a * C::CPT + h) * 16) ^ ((C::BOXB == 128 ? g : (g >> 1) & 3) << 4));
#pragma unroll
    for (int e = 0; e < 2; ++e) v_at[e] = C::HALF_BYTES + (2 * a + e) * C::BOXB + ((g * (C::BOXB / 8)) ^ ((C::BOXB == 128 ? 2 * a + e : a) << 4));

    // The units go round among the warps.  A warp waits for every tile and leaves every tile, with a unit of its own there or not: copies may
    // land out of order, and the parity of a barrier tells a lap of the ring only from the one before it.
    int st = 0, u = warp;
    uint32_t lap = 0;
    for (int i = 0; i < nt; ++i) {
      if (!ring_wait(&mi.full[st], lap & 1u, abort_flag, prm.status, WF_FULL)) break;
      for (; u < (i + 1) * C::UNITS; u += C::WARPS) {
        const int r0 = (u - i * C::UNITS) * 16, key0 = (j0 + i) * KEYS + r0;
        if (key0 >= n) continue;
        const uint8_t* const unit = smem + st * C::STAGE_BYTES + r0 * C::BOXB;
        const int left = n - key0;                               // entries of the unit, 16 or more: all
        float sk0 = 1.0f, sk1 = 1.0f, sv0 = 1.0f, sv1 = 1.0f;
        if constexpr (Q8) {
          const float* const sc = reinterpret_cast<const float*>(smem + C::OFF_SCALE) + st * 2 * KEYS + r0 + g;
          sk0 = sc[0]; sk1 = sc[8]; sv0 = sc[KEYS]; sv1 = sc[KEYS + 8];
        }
        // ---- S^T, in two chains of products
        constexpr int CH = NT8 == 1 ? 2 : 1;
        float s[CH][NT8][4];
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int t = 0; t < NT8; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[c][t][e] = 0.0f;
#pragma unroll
        for (int b = 0; b < C::BOXES; ++b)
#pragma unroll
          for (int h = 0; h < C::CPT; ++h) {
            const uint4 y0 = *reinterpret_cast<const uint4*>(unit + b * KEYS * C::BOXB + k_at[h]),
                        y1 = *reinterpret_cast<const uint4*>(unit + b * KEYS * C::BOXB + k_at[h] + 8 * C::BOXB);
            const uint32_t x0[4] = {y0.x, y0.y, y0.z, y0.w}, x1[4] = {y1.x, y1.y, y1.z, y1.w};
#pragma unroll
            for (int t = 0; t < C::KPC; ++t) {
              const int ks = (b * C::CPT + h) * C::KPC + t;
              uint32_t a0, a1, a2, a3;
              if constexpr (Q8) {
                const uint32_t z0 = flip_signs<FMT>(x0[t]), z1 = flip_signs<FMT>(x1[t]);
                a0 = codes_to_half2<FMT, 0>(z0); a2 = codes_to_half2<FMT, 1>(z0);
                a1 = codes_to_half2<FMT, 0>(z1); a3 = codes_to_half2<FMT, 1>(z1);
              } else {
                a0 = x0[2 * t]; a2 = x0[2 * t + 1]; a1 = x1[2 * t]; a3 = x1[2 * t + 1];
              }
#pragma unroll
              for (int c = 0; c < NT8; ++c) mma16816<FMT>(s[ks % CH][c], a0, a1, a2, a3, qf[ks][c].x, qf[ks][c].y);
            }
          }
        // ---- V of this thread: 4 keys (positions 2 a, 2 a + 1, 2 a + 8, 2 a + 9 of the 16)
        uint32_t v[C::BOXES][4][C::BOXB / 32];
#pragma unroll
        for (int b = 0; b < C::BOXES; ++b)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint8_t* const from = unit + b * KEYS * C::BOXB + v_at[k & 1] + (k >> 1) * 8 * C::BOXB;
            if constexpr (C::BOXB == 128) {
              const uint4 y = *reinterpret_cast<const uint4*>(from);
              v[b][k][0] = y.x; v[b][k][1] = y.y; v[b][k][2] = y.z; v[b][k][3] = y.w;
            } else {
              const uint2 y = *reinterpret_cast<const uint2*>(from);
              v[b][k][0] = y.x; v[b][k][1] = y.y;
            }
          }
        // ---- logits; the last unit ends before its 16th key: whatever stands behind it, NaN included, must not count
        float z[NT8][4];
#pragma unroll
        for (int t = 0; t < NT8; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) z[t][e] = (CH == 2 ? s[0][t][e] + s[CH - 1][t][e] : s[0][t][e]) * ((e < 2 ? sk0 : sk1) * qs[t][e & 1]);
        if (left < 16) {
#pragma unroll
          for (int t = 0; t < NT8; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (g + (e < 2 ? 0 : 8) >= left) z[t][e] = -INFINITY;
          if (g >= left) sv0 = 0.0f;
          if (g + 8 >= left) sv1 = 0.0f;
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (2 * a + (k & 1) + 8 * (k >> 1) >= left)
#pragma unroll
              for (int b = 0; b < C::BOXES; ++b)
#pragma unroll
                for (int y = 0; y < C::BOXB / 32; ++y) v[b][k][y] = 0;
        }
        if constexpr (C::TREE) {
          const int mine = entries - key0;                       // position of the first new token in the unit
          if (mine < 16) {
#pragma unroll
            for (int t = 0; t < NT8; ++t)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int token = g + (e < 2 ? 0 : 8) - mine;
                if (token >= 0 && !(token < 64 && (tm.sees[8 * t + 2 * a + (e & 1)] >> token & 1))) z[t][e] = -INFINITY;
              }
            // A new token's value that is no number would reach the rows that do not see it, times their zero: it is left out here and counted behind the
            // sums, for the rows that do.
            unsigned long long odd = 0;
            auto out = [&](int key) { if (key >= mine && key < left) odd |= 1ull << (key - mine); };
            if constexpr (Q8) {
              if (g >= mine && !(fabsf(sv0) < INFINITY)) { out(g); sv0 = 0.0f; }
              if (g + 8 >= mine && !(fabsf(sv1) < INFINITY)) { out(g + 8); sv1 = 0.0f; }
            }
            if constexpr (FMT != FMT_INT8) {
#pragma unroll
              for (int b = 0; b < C::BOXES; ++b)
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                  for (int y = 0; y < C::BOXB / 32; ++y) {
                    const uint32_t numbers = finite_parts<FMT>(v[b][k][y]);
                    const int key = 2 * a + (k & 1) + 8 * (k >> 1);
                    if (numbers != 0xFFFFFFFFu && key >= mine) { out(key); v[b][k][y] &= numbers; }
                  }
            }
            if (odd) atomicOr(&tm.odd, odd);
          }
        }
        if constexpr (C::CAUSAL) {
#pragma unroll
          for (int t = 0; t < NT8; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (key0 + g + (e < 2 ? 0 : 8) > own[t][e & 1]) z[t][e] = -INFINITY;
          // A value that is no number would reach the rows that do not see it, times their zero: then the rows take these keys one by one.
          {
            bool odd = false;
#pragma unroll
            for (int b = 0; b < C::BOXES; ++b)
#pragma unroll
              for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int y = 0; y < C::BOXB / 32; ++y) odd |= (v[b][k][y] & 0x7F80u) == 0x7F80u || (v[b][k][y] & 0x7F800000u) == 0x7F800000u;
            if (odd) mi.odd = 1;
          }
        }
        // ---- probabilities
        uint32_t pb[NT8][2];
#pragma unroll
        for (int t = 0; t < NT8; ++t) {
          float p[4], w[4], over = -INFINITY, heavy = 0.0f;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float above = z[t][e] - m[t][e & 1];
            over = fmaxf(over, above);
            p[e] = fast_exp2(above);
            w[e] = p[e];
            if constexpr (Q8) {                                  // (scale times cw may be infinite where p is 0)
              w[e] = p[e] * (e < 2 ? sv0 : sv1) * cw[t][e & 1];
              heavy = fmaxf(heavy, w[e]);
            }
          }
          if (__any_sync(0xFFFFFFFFu, over > 8.0f || heavy > 32768.0f)) {          // rare after the first keys
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float top = fmaxf(m[t][e], max_over_keys(fmaxf(z[t][e], z[t][2 + e])));
              float f = fast_exp2(m[t][e] - top);
              m[t][e] = top;
              l[t][e] *= f;
              p[e] = fast_exp2(z[t][e] - top);
              p[2 + e] = fast_exp2(z[t][2 + e] - top);
              w[e] = p[e]; w[2 + e] = p[2 + e];
              if constexpr (Q8) {                                // cw = 1024 / (largest weight so far)
                const float before = f * (1024.0f / cw[t][e]);
                const float most = fmaxf(fmaxf(before, max_over_keys(fmaxf(p[e] * sv0, p[2 + e] * sv1))), 0x1p-100f);
                cw[t][e] = 1024.0f / most;
                f = before / most;
                w[e] = p[e] * sv0 * cw[t][e];
                w[2 + e] = p[2 + e] * sv1 * cw[t][e];
              }
#pragma unroll
              for (int j = 0; j < C::MT; ++j) { acc[j][t][e] *= f; acc[j][t][2 + e] *= f; }
            }
          }
          l[t][0] += p[0] + p[2];
          l[t][1] += p[1] + p[3];
          pb[t][0] = transpose8x8(pack_p<FMT>(w[0], w[1]));
          pb[t][1] = transpose8x8(pack_p<FMT>(w[2], w[3]));
        }
        // ---- O^T
#pragma unroll
        for (int b = 0; b < C::BOXES; ++b)
#pragma unroll
          for (int z = 0; z < C::BOXB / 32; ++z) {
            if constexpr (Q8) {
              uint32_t h[4];                                     // bytes of keys 0 and 1: columns 0, 1 / 2, 3; of keys 2 and 3
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                h[2 * u] = flip_signs<FMT>(prmt(v[b][2 * u][z], v[b][2 * u + 1][z], 0x5140));
                h[2 * u + 1] = flip_signs<FMT>(prmt(v[b][2 * u][z], v[b][2 * u + 1][z], 0x7362));
              }
#pragma unroll
              for (int y = 0; y < 2; ++y) {
                const int j = b * (C::MT / C::BOXES) + 2 * z + y;
                const uint32_t a0 = codes_to_half2<FMT, 0>(h[y]), a1 = codes_to_half2<FMT, 1>(h[y]), a2 = codes_to_half2<FMT, 0>(h[2 + y]),
                               a3 = codes_to_half2<FMT, 1>(h[2 + y]);
#pragma unroll
                for (int t = 0; t < NT8; ++t) mma16816<FMT>(acc[j][t], a0, a1, a2, a3, pb[t][0], pb[t][1]);
              }
            } else {
              const int j = b * (C::MT / C::BOXES) + z;
              const uint32_t a0 = prmt(v[b][0][z], v[b][1][z], 0x5410), a1 = prmt(v[b][0][z], v[b][1][z], 0x7632),
                             a2 = prmt(v[b][2][z], v[b][3][z], 0x5410), a3 = prmt(v[b][2][z], v[b][3][z], 0x7632);
#pragma unroll
              for (int t = 0; t < NT8; ++t) mma16816<FMT>(acc[j][t], a0, a1, a2, a3, pb[t][0], pb[t][1]);
            }
          }
      }
      // (the products of the loop above have been issued, so what they need has been loaded: an arrival itself waits for no load)
      __syncwarp();
      if (lane == 0) mbar_arrive(&mi.empty[st]);
      if (++st == NS) { st = 0; ++lap; }
    }
    // ---- what this warp has: sums over its threads' keys, statistics; then, the ring being idle, O
#pragma unroll
    for (int t = 0; t < NT8; ++t)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) l[t][e] += __shfl_xor_sync(0xFFFFFFFFu, l[t][e], o);
        if (g == 0) mi.ml[warp][8 * t + 2 * a + e] = make_float2(m[t][e], l[t][e]);
      }
    named_barrier_sync(1, 32 * C::WARPS);                        // every warp has read its last stage
    float* const part = reinterpret_cast<float*>(smem) + (size_t)warp * N * D;
#pragma unroll
    for (int t = 0; t < NT8; ++t)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float f = Q8 ? 1.0f / cw[t][e] : 1.0f;
#pragma unroll
        for (int j = 0; j < C::MT; ++j) {
          constexpr int PER = C::MT / C::BOXES;
          const int d = (j / PER) * C::EPB + g * (C::EPB / 8) + 2 * (j % PER);
          *reinterpret_cast<float2*>(part + (8 * t + 2 * a + e) * D + d) = make_float2(acc[j][t][e] * f, acc[j][t][2 + e] * f);
        }
      }
  }
  __syncthreads();
  // ---- the warps' results added up, into the first warp's place or the slot
  for (int e = tid; e < n_rows * (D / 4); e += C::THREADS) {
    const int r = e / (D / 4), c = e % (D / 4);
    float top = -FLT_MAX, sum = 0.0f;
#pragma unroll
    for (int k = 0; k < C::WARPS; ++k) top = fmaxf(top, mi.ml[k][r].x);
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int k = 0; k < C::WARPS; ++k) {
      const float2 ml = mi.ml[k][r];
      const float f = fast_exp2(ml.x - top);
      const float4 y = reinterpret_cast<const float4*>(smem)[(k * N + r) * (D / 4) + c];
      sum = fmaf(f, ml.y, sum);
      o.x = fmaf(f, y.x, o.x); o.y = fmaf(f, y.y, o.y); o.z = fmaf(f, y.z, o.z); o.w = fmaf(f, y.w, o.w);
    }
    const size_t at = part0 + (size_t)r * prm.n_slots;
    bool none = sum == 0.0f || (C::CAUSAL && mi.odd);
    if constexpr (C::TREE) {
      none |= tm.sees[r] == 0;
      if (tm.odd & tm.sees[r]) {
        float x[4] = {o.x, o.y, o.z, o.w};
        add_odd<D, FMT, 4>(tr, prm, hkv, seq, entries, tm.odd & tm.sees[r], 4 * c, x);
        o = make_float4(x[0], x[1], x[2], x[3]);
      }
    }
    const float2 ml = none ? make_float2(-INFINITY, 0.0f) : make_float2(top, sum);
    if (finish) {
      reinterpret_cast<float4*>(smem)[r * (D / 4) + c] = o;
      if (c == 0) mi.all[r] = ml;
    } else {
      reinterpret_cast<float4*>(prm.part_o + at * D)[c] = o;
      if (c == 0) prm.part_ml[at] = ml;
    }
  }
  }
  if (!finish) return;

  // ---- the splits' results, the slots in memory and the new tokens' keys: a warp per row, the rows dealt out over the cluster
  if (prm.n_split > 1) cluster_sync_all(); else __syncthreads();
  const int G = prm.q.Hq / prm.q.Hkv;
  for (int r = split + prm.n_split * warp; r < n_rows; r += prm.n_split * (C::WARPS + 1)) {
    const int row = row0 + r, bi = row / G, i = bi % prm.q.w;
    RowSum<D> sum;
    float2 mine = make_float2(-INFINITY, 0.0f);
    if (lane < prm.n_split) {
      float y[2];
      ld_cluster<2>(map_to_cta(&mi.all[r], lane), y);
      mine = make_float2(y[0], y[1]);
    }
    sum.join(mine, prm.n_split, [&](int s, float (&y)[E]) { ld_cluster<E>(map_to_cta(reinterpret_cast<const float*>(smem) + r * D + lane * E, s), y); });
    const size_t slots = ((size_t)hkv * prm.total_rows + row) * fin.n_slots;
    sum.join_slots(fin.part_ml + slots, fin.part_o + slots * D, fin.n_slots, 0, 1, lane);
    if (fin.k_win != nullptr && (!C::CAUSAL || mi.odd)) {
      uint32_t y[E / 2];
      float q[E];
#pragma unroll
      for (int e = 0; e < E / 2; ++e) y[e] = reinterpret_cast<const uint32_t*>(smem + C::OFF_ROWS)[r * (D / 2) + lane * (E / 2) + e];
      RowSum<D>::unpack(y, q);
      sum.join_window(fin, q, hkv, bi / prm.q.w, i, 0, 1, lane);
    }
    if constexpr (C::TREE) { if (tm.sees[r] == 0) sum = RowSum<D>(); }
    sum.store(fin, hkv * G + row % G, bi, lane);
  }
  if (prm.n_split > 1) cluster_sync_all();                       // no CTA exits while another may read its shared memory
}

}  // namespace few
}  // namespace pc
