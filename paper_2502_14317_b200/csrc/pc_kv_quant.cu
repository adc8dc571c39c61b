// Rows of bf16 into the 8-bit caches and back (definition: pc_kv_cache in pc.h).
//
// Bound by memory: a row of keys or values is read once (2 d bytes) and written once (d + 4), or the reverse.  d / 8 lanes hold
// a row, 8 values each, so that its largest magnitude takes log2(d / 8) exchanges; the magnitudes are compared as the
// integers that their bits are, two at a time.  Keys and values of an entry go through one thread.
#include "pc_cache.h"
#include "pc_kernels.h"
#include "pc_kv8.cuh"
#include "pc_sm100.cuh"

namespace pc {

namespace {

constexpr int NT = 256;

template <int LANES>
__device__ __forceinline__ uint32_t row_max_bits(uint4 x) {
  uint32_t m = __vmaxu2(__vmaxu2(x.x & 0x7FFF7FFFu, x.y & 0x7FFF7FFFu), __vmaxu2(x.z & 0x7FFF7FFFu, x.w & 0x7FFF7FFFu));
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) m = __vmaxu2(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
  return max(m & 0xFFFFu, m >> 16);
}
__device__ __forceinline__ float lo16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi16(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

template <int FMT, int LANES>
__device__ __forceinline__ uint2 quantise(uint4 x, float& scale) {
  const uint32_t bits = row_max_bits<LANES>(x);
  const float a = __uint_as_float(bits << 16);
  const bool held = a >= KV_TINY && bits < 0x7F80u;
  const float r = held ? __fdiv_rn(top_code<FMT>(), a) : 0.0f;
  scale = bits >= 0x7F80u ? __uint_as_float(0x7FC00000u) : held ? __fdiv_rn(a, top_code<FMT>()) : 0.0f;
  if (!held) return make_uint2(0, 0);
  return make_uint2(values_to_codes<FMT>(__fmul_rn(lo16(x.x), r), __fmul_rn(hi16(x.x), r), __fmul_rn(lo16(x.y), r), __fmul_rn(hi16(x.y), r)),
                    values_to_codes<FMT>(__fmul_rn(lo16(x.z), r), __fmul_rn(hi16(x.z), r), __fmul_rn(lo16(x.w), r), __fmul_rn(hi16(x.w), r)));
}

// Work is dealt out in pieces of ROWS entries of one (sequence, kv-head); a group of lanes has U of them at a time, so that their loads
// (for a gather: their positions, then their rows) are in flight together.
constexpr int U = 4;
template <int LANES>
struct Piece {
  static constexpr int GROUPS = NT / LANES, ROWS = GROUPS * U;
  int per, bh, i;                                            // pieces of a head; this one's (sequence, kv-head) and the lanes' first entry
  __device__ __forceinline__ Piece(long long piece, int n) : per((n + ROWS - 1) / ROWS), bh((int)(piece / per)) {
    i = (int)(piece - (long long)bh * per) * ROWS + threadIdx.x / LANES;
  }
  static long long count(long long heads, int n) { return heads * ((n + ROWS - 1) / ROWS); }
};

}  // namespace

template <int D, int FMT, bool GATHER>
__global__ void __launch_bounds__(NT) kv_quantize_kernel(const KvWrite p, const long long pieces) {
  chain();
  constexpr int LANES = D / 8, GROUPS = Piece<LANES>::GROUPS;
  const int lane = threadIdx.x % LANES;
  // every lane of a warp goes through the same number of turns: the exchanges of row_max_bits are the whole warp's
  for (long long piece = blockIdx.x; piece < pieces; piece += gridDim.x) {
    const Piece<LANES> w(piece, p.n);
    const int b = w.bh / p.Hkv, h = w.bh - b * p.Hkv;
    long long to[U];                                         // entry of the cache, or -1
    const uint16_t *k_at[U], *v_at[U];                       // null: zeros
    if constexpr (GATHER) {
      int pos[U], chunk[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int e = w.i + u * GROUPS, r = e / p.per_chunk;
        to[u] = e < p.n ? (long long)h * p.capacity + e : -1;
        pos[u] = e < p.n ? __ldg(p.idx + ((long long)r * p.Hkv + h) * p.per_chunk + (e - r * p.per_chunk)) : -1;
        chunk[u] = e < p.n ? __ldg(p.kept + r) : 0;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool there = pos[u] >= 0;
        k_at[u] = there ? static_cast<const uint16_t*>(p.k_src) + chunk[u] * p.k_stride[0] + pos[u] * p.k_stride[1] + h * p.k_stride[2] : nullptr;
        v_at[u] = there ? static_cast<const uint16_t*>(p.v_src) + chunk[u] * p.v_stride[0] + pos[u] * p.v_stride[1] + h * p.v_stride[2] : nullptr;
        if (p.pos_out != nullptr && lane == 0 && to[u] >= 0) p.pos_out[(long long)h * p.n + w.i + u * GROUPS] = there ? pos[u] : -1;
      }
    } else {
      const long long at0 = (long long)p.at0 + (p.at ? p.at[b] : 0);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = w.i + u * GROUPS;
        const long long at = at0 + i;
        const bool there = i < p.n && at >= 0 && at < p.capacity;
        if (i < p.n && !there && lane == 0 && p.status) atomicCAS(p.status, 0, 401);
        to[u] = there ? (long long)w.bh * p.capacity + at : -1;
        k_at[u] = there ? static_cast<const uint16_t*>(p.k_src) + b * p.k_stride[0] + i * p.k_stride[1] + h * p.k_stride[2] : nullptr;
        v_at[u] = there ? static_cast<const uint16_t*>(p.v_src) + b * p.v_stride[0] + i * p.v_stride[1] + h * p.v_stride[2] : nullptr;
      }
    }
    uint4 xk[U], xv[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      xk[u] = xv[u] = make_uint4(0, 0, 0, 0);
      if (k_at[u] != nullptr) {
        xk[u] = __ldg(reinterpret_cast<const uint4*>(k_at[u]) + lane);
        xv[u] = __ldg(reinterpret_cast<const uint4*>(v_at[u]) + lane);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float sk, sv;
      const uint2 ck = quantise<FMT, LANES>(xk[u], sk), cv = quantise<FMT, LANES>(xv[u], sv);
      if (to[u] >= 0) {
        reinterpret_cast<uint2*>(p.k + to[u] * D)[lane] = ck;
        reinterpret_cast<uint2*>(p.v + to[u] * D)[lane] = cv;
        if (lane == 0) { p.k_scale[to[u]] = sk; p.v_scale[to[u]] = sv; }
      }
    }
  }
}

template <int D, int FMT>
__global__ void __launch_bounds__(NT) kv_dequantize_kernel(const KvRead p, const long long pieces) {
  chain();
  constexpr int LANES = D / 16, GROUPS = Piece<LANES>::GROUPS;                // 16 codes a lane
  const int lane = threadIdx.x % LANES;
  for (long long piece = blockIdx.x; piece < pieces; piece += gridDim.x) {
    const Piece<LANES> w(piece, p.n);
    const long long at0 = (long long)p.at0 + (p.at ? p.at[w.bh / p.Hkv] : 0);
    uint4 k[U], v[U];
    float sk[U], sv[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = w.i + u * GROUPS;
      const long long at = at0 + i;
      k[u] = v[u] = make_uint4(0, 0, 0, 0);
      sk[u] = sv[u] = 0.0f;
      if (i < p.n && at >= 0 && at < p.capacity) {
        const long long from = w.bh * p.capacity + at;
        k[u] = __ldg(reinterpret_cast<const uint4*>(p.k + from * D) + lane);
        v[u] = __ldg(reinterpret_cast<const uint4*>(p.v + from * D) + lane);
        sk[u] = __ldg(p.k_scale + from);
        sv[u] = __ldg(p.v_scale + from);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = w.i + u * GROUPS;
      if (i >= p.n) break;
      auto store = [&](void* to, const uint4& x, float s) {                  // 32 bytes, a whole sector, in one store
        const uint2 a = codes_to_bf16x4<FMT>(x.x, s), b = codes_to_bf16x4<FMT>(x.y, s), c = codes_to_bf16x4<FMT>(x.z, s), d = codes_to_bf16x4<FMT>(x.w, s);
        uint16_t* const o = static_cast<uint16_t*>(to) + ((long long)w.bh * p.n + i) * D + 16 * lane;
        if (p.sectors) {
          const float y[8] = {__uint_as_float(a.x), __uint_as_float(a.y), __uint_as_float(b.x), __uint_as_float(b.y),
                              __uint_as_float(c.x), __uint_as_float(c.y), __uint_as_float(d.x), __uint_as_float(d.y)};
          st_global_f32x8(o, y);
        } else {
          reinterpret_cast<uint4*>(o)[0] = make_uint4(a.x, a.y, b.x, b.y);
          reinterpret_cast<uint4*>(o)[1] = make_uint4(c.x, c.y, d.x, d.y);
        }
      };
      store(p.k_out, k[u], sk[u]);
      store(p.v_out, v[u], sv[u]);
    }
  }
}

namespace {

dim3 grid_for(long long pieces) { return dim3((unsigned)(pieces < 0x7FFFFFFF ? pieces : 0x7FFFFFFF)); }
template <int D, int FMT>
cudaError_t quantize_t(const KvWrite& w, bool gather, cudaStream_t st) {
  const long long pieces = Piece<D / 8>::count((long long)w.B * w.Hkv, w.n);
  return gather ? launch_chained(kv_quantize_kernel<D, FMT, true>, grid_for(pieces), dim3(NT), 0, st, 1, w, pieces)
                : launch_chained(kv_quantize_kernel<D, FMT, false>, grid_for(pieces), dim3(NT), 0, st, 1, w, pieces);
}
template <int D, int FMT>
cudaError_t dequantize_t(const KvRead& r, cudaStream_t st) {
  const long long pieces = Piece<D / 16>::count((long long)r.B * r.Hkv, r.n);
  return launch_chained(kv_dequantize_kernel<D, FMT>, grid_for(pieces), dim3(NT), 0, st, 1, r, pieces);
}

}  // namespace

cudaError_t launch_kv_quantize(const KvWrite& w, int format, int d, bool gather, cudaStream_t st) {
  if (d == 128) return format == FMT_INT8 ? quantize_t<128, FMT_INT8>(w, gather, st) : quantize_t<128, FMT_E4M3>(w, gather, st);
  return format == FMT_INT8 ? quantize_t<64, FMT_INT8>(w, gather, st) : quantize_t<64, FMT_E4M3>(w, gather, st);
}
cudaError_t launch_kv_dequantize(const KvRead& r, int format, int d, cudaStream_t st) {
  if (d == 128) return format == FMT_INT8 ? dequantize_t<128, FMT_INT8>(r, st) : dequantize_t<128, FMT_E4M3>(r, st);
  return format == FMT_INT8 ? dequantize_t<64, FMT_INT8>(r, st) : dequantize_t<64, FMT_E4M3>(r, st);
}

}  // namespace pc
