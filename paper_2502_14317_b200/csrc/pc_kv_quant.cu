// Rows of bf16 into the 8-bit caches and back (definition: pc_kv_cache in pc.h).
//
// Bound by memory: a row of keys or values is read once (2 d bytes) and written once (d + 4), or the reverse.  d / 8 lanes hold
// a row, 8 values each, and four entries at a time: the largest magnitudes of their eight rows (the bits as integers, two to a word) take 4 or 5 exchanges
// in all and end with one row a lane or two, which divides for it.  Keys and values of an entry go through one thread.
// Eight loads of a thread are on their way at once.  Measured, d = 128, 8 kv-heads: 64 x 512 tokens into e4m3 32.5 us = 6.27 TB/s (97 % of the copy bandwidth;
// with exchanges and divisions by every lane for every row 39.8), 16384 kept entries a kv-head gathered 21.5 = 4.7 TB/s (24.0), 1024 2.9 (4.0); 16 x 16384
// entries back to bf16 269 us = 6.05 TB/s; one token 3.4 to 4.4, a launch.
#include "pc_cache.h"
#include "pc_kernels.h"
#include "pc_kv8.cuh"
#include "pc_sm100.cuh"

namespace pc {

namespace {

constexpr int NT = 256;

__device__ __forceinline__ float lo16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi16(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// largest magnitudes of the halves of eight values' words, as the integers that their bits are
__device__ __forceinline__ uint32_t max_bits(uint4 x) {
  return __vmaxu2(__vmaxu2(x.x & 0x7FFF7FFFu, x.y & 0x7FFF7FFFu), __vmaxu2(x.z & 0x7FFF7FFFu, x.w & 0x7FFF7FFFu));
}
// Largest magnitude of row lane / (LANES / 8) of the eight that LANES lanes hold: two rows to a word, and with each of the first two exchanges a lane
// keeps half of the words.
template <int LANES>
__device__ __forceinline__ uint32_t max_of_rows(const uint32_t (&m)[8], int lane) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = __vmaxu2(prmt(m[2 * i], m[2 * i + 1], 0x5410), prmt(m[2 * i], m[2 * i + 1], 0x7632));
  const bool upper = lane & (LANES / 2), odd = lane & (LANES / 4);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t got = __shfl_xor_sync(0xFFFFFFFFu, upper ? w[i] : w[2 + i], LANES / 2);
    w[i] = __vmaxu2(upper ? w[2 + i] : w[i], got);
  }
  const uint32_t got = __shfl_xor_sync(0xFFFFFFFFu, odd ? w[0] : w[1], LANES / 4);
  uint32_t x = __vmaxu2(odd ? w[1] : w[0], got);
#pragma unroll
  for (int o = LANES / 8; o > 0; o >>= 1) x = __vmaxu2(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
  return lane & (LANES / 8) ? x >> 16 : x & 0xFFFFu;
}
// r and scale of a row (r 0: codes 0)
template <int FMT>
__device__ __forceinline__ float row_scale(uint32_t bits, float& scale) {
  const float a = __uint_as_float(bits << 16);
  const bool held = a >= KV_TINY && bits < 0x7F80u;
  scale = bits >= 0x7F80u ? __uint_as_float(0x7FC00000u) : held ? __fdiv_rn(a, top_code<FMT>()) : 0.0f;
  return held ? __fdiv_rn(top_code<FMT>(), a) : 0.0f;
}
template <int FMT>
__device__ __forceinline__ uint2 quantise(uint4 x, float r) {
  const uint2 c = make_uint2(values_to_codes<FMT>(__fmul_rn(lo16(x.x), r), __fmul_rn(hi16(x.x), r), __fmul_rn(lo16(x.y), r), __fmul_rn(hi16(x.y), r)),
                             values_to_codes<FMT>(__fmul_rn(lo16(x.z), r), __fmul_rn(hi16(x.z), r), __fmul_rn(lo16(x.w), r), __fmul_rn(hi16(x.w), r)));
  return r == 0.0f ? make_uint2(0, 0) : c;
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
  // every lane of a warp goes through the same number of turns: the exchanges of max_of_rows are the whole warp's
  for (long long piece = blockIdx.x; piece < pieces; piece += gridDim.x) {
    const Piece<LANES> w(piece, p.n);
    const int b = w.bh / p.Hkv, h = w.bh - b * p.Hkv;
    // entry i is the cache's entry first + i of row w.bh
    const long long first = GATHER ? 0 : (long long)p.at0 + (p.at ? p.at[b] : 0);
    auto written = [&](int i) { return i < p.n && (GATHER || (first + i >= 0 && first + i < p.capacity)); };
    const uint16_t* const k_head = static_cast<const uint16_t*>(p.k_src) + (GATHER ? 0 : b * p.k_stride[0]) + h * p.k_stride[2];
    const uint16_t* const v_head = static_cast<const uint16_t*>(p.v_src) + (GATHER ? 0 : b * p.v_stride[0]) + h * p.v_stride[2];
    uint4 x[2 * U];                                          // rows 2u: keys, 2u + 1: values
    if constexpr (GATHER) {
      int pos[U], chunk[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int e = w.i + u * GROUPS, r = (int)((unsigned long long)e * p.chunk_mul >> p.chunk_shift);       // e / per_chunk
        pos[u] = e < p.n ? __ldg(p.idx + ((long long)r * p.Hkv + h) * p.per_chunk + (e - r * p.per_chunk)) : -1;
        chunk[u] = e < p.n ? __ldg(p.kept + r) : 0;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int e = w.i + u * GROUPS;
        x[2 * u] = x[2 * u + 1] = make_uint4(0, 0, 0, 0);
        if (pos[u] >= 0) {                                   // (keys and values share strides)
          const long long off = chunk[u] * p.k_stride[0] + pos[u] * p.k_stride[1];
          x[2 * u] = __ldg(reinterpret_cast<const uint4*>(k_head + off) + lane);
          x[2 * u + 1] = __ldg(reinterpret_cast<const uint4*>(v_head + off) + lane);
        }
        if (p.pos_out != nullptr && lane == 0 && e < p.n) p.pos_out[(long long)h * p.n + e] = pos[u] >= 0 ? pos[u] : -1;
      }
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = w.i + u * GROUPS;
        x[2 * u] = x[2 * u + 1] = make_uint4(0, 0, 0, 0);
        if (written(i)) {
          x[2 * u] = __ldg(reinterpret_cast<const uint4*>(k_head + i * p.k_stride[1]) + lane);
          x[2 * u + 1] = __ldg(reinterpret_cast<const uint4*>(v_head + i * p.v_stride[1]) + lane);
        } else if (i < p.n && lane == 0 && p.status) {
          atomicCAS(p.status, 0, 401);
        }
      }
    }
    uint32_t m[2 * U];
#pragma unroll
    for (int i = 0; i < 2 * U; ++i) m[i] = max_bits(x[i]);
    float scale;
    const float r = row_scale<FMT>(max_of_rows<LANES>(m, lane), scale);
    const long long to = (long long)w.bh * p.capacity + first + w.i;
    {
      const int row = lane / (LANES / 8), i = row / 2 * GROUPS;                // of this lane
      if (lane % (LANES / 8) == 0 && written(w.i + i)) (row & 1 ? p.v_scale : p.k_scale)[to + i] = scale;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint2 ck = quantise<FMT>(x[2 * u], __shfl_sync(0xFFFFFFFFu, r, 2 * u * (LANES / 8), LANES)),
                  cv = quantise<FMT>(x[2 * u + 1], __shfl_sync(0xFFFFFFFFu, r, (2 * u + 1) * (LANES / 8), LANES));
      if (written(w.i + u * GROUPS)) {
        reinterpret_cast<uint2*>(p.k + (to + u * GROUPS) * D)[lane] = ck;
        reinterpret_cast<uint2*>(p.v + (to + u * GROUPS) * D)[lane] = cv;
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
