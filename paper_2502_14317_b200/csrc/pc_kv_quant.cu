// Rows of bf16 into the 8-bit caches and back (definition: pc_kv_cache in pc.h).
//
// Bound by memory: a row of keys or values is read once (2 d bytes) and written once (d + 4), or the reverse.  d / 8 lanes hold
// a row, 8 values each, so that its largest magnitude takes log2(d / 8) exchanges; the magnitudes are compared as the
// integers that their bits are, two at a time.  Keys and values of an entry go through one thread.
#include "pc_cache.h"
#include "pc_kernels.h"
#include "pc_kv8.cuh"

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

}  // namespace

template <int D, int FMT, bool GATHER>
__global__ void __launch_bounds__(NT) kv_quantize_kernel(const KvWrite p) {
  chain();
  constexpr int LANES = D / 8;
  const int lane = threadIdx.x % LANES;
  const long long n_rows = (long long)p.B * p.n * p.Hkv, step = (long long)gridDim.x * (NT / LANES);
  // every lane of a warp goes through the same number of turns: the exchanges of row_max_bits are the whole warp's
  for (long long row0 = (long long)blockIdx.x * (NT / LANES); row0 < n_rows; row0 += step) {
    const long long row = row0 + threadIdx.x / LANES;
    bool there = row < n_rows;
    uint4 xk = make_uint4(0, 0, 0, 0), xv = xk;
    long long to = 0;                                        // entry of the cache
    if (there) {
      if constexpr (GATHER) {                                // row = (kv-head, entry)
        const int h = (int)(row / p.n), e = (int)(row % p.n), r = e / p.per_chunk, t = e % p.per_chunk;
        const int pos = p.idx[((long long)r * p.Hkv + h) * p.per_chunk + t];
        if (pos >= 0) {
          const long long chunk = p.kept[r];
          xk = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.k_src) + chunk * p.k_stride[0] + pos * p.k_stride[1] + h * p.k_stride[2]) + lane);
          xv = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.v_src) + chunk * p.v_stride[0] + pos * p.v_stride[1] + h * p.v_stride[2]) + lane);
        }
        to = (long long)h * p.capacity + e;
        if (p.pos_out != nullptr && lane == 0) p.pos_out[row] = pos < 0 ? -1 : pos;
      } else {                                               // row = (sequence, token, kv-head)
        const int h = (int)(row % p.Hkv);
        const long long x = row / p.Hkv;
        const int i = (int)(x % p.n), b = (int)(x / p.n);
        const long long at = (long long)p.at0 + (p.at ? p.at[b] : 0) + i;
        if (at < 0 || at >= p.capacity) {
          if (lane == 0 && p.status) atomicCAS(p.status, 0, 401);
          there = false;
        } else {
          xk = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.k_src) + b * p.k_stride[0] + i * p.k_stride[1] + h * p.k_stride[2]) + lane);
          xv = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.v_src) + b * p.v_stride[0] + i * p.v_stride[1] + h * p.v_stride[2]) + lane);
        }
        to = ((long long)b * p.Hkv + h) * p.capacity + at;
      }
    }
    float sk, sv;
    const uint2 ck = quantise<FMT, LANES>(xk, sk), cv = quantise<FMT, LANES>(xv, sv);
    if (there) {
      reinterpret_cast<uint2*>(p.k + to * D)[lane] = ck;
      reinterpret_cast<uint2*>(p.v + to * D)[lane] = cv;
      if (lane == 0) { p.k_scale[to] = sk; p.v_scale[to] = sv; }
    }
  }
}

template <int D, int FMT>
__global__ void __launch_bounds__(NT) kv_dequantize_kernel(const KvRead p) {
  chain();
  constexpr int LANES = D / 16;                              // 16 codes a lane
  const int lane = threadIdx.x % LANES;
  const long long n_rows = (long long)p.B * p.Hkv * p.n;
  for (long long row = (long long)blockIdx.x * (NT / LANES) + threadIdx.x / LANES; row < n_rows; row += (long long)gridDim.x * (NT / LANES)) {
    const int i = (int)(row % p.n);
    const long long bh = row / p.n;
    const long long at = (long long)p.at0 + (p.at ? p.at[bh / p.Hkv] : 0) + i;
    uint4 k0 = make_uint4(0, 0, 0, 0), k1 = k0, v0 = k0, v1 = k0;
    if (at >= 0 && at < p.capacity) {
      const long long from = bh * p.capacity + at;
      const uint4 k = __ldg(reinterpret_cast<const uint4*>(p.k + from * D) + lane), v = __ldg(reinterpret_cast<const uint4*>(p.v + from * D) + lane);
      const float sk = __ldg(p.k_scale + from), sv = __ldg(p.v_scale + from);
      uint2 a = codes_to_bf16x4<FMT>(k.x, sk), b = codes_to_bf16x4<FMT>(k.y, sk);
      k0 = make_uint4(a.x, a.y, b.x, b.y);
      a = codes_to_bf16x4<FMT>(k.z, sk); b = codes_to_bf16x4<FMT>(k.w, sk);
      k1 = make_uint4(a.x, a.y, b.x, b.y);
      a = codes_to_bf16x4<FMT>(v.x, sv); b = codes_to_bf16x4<FMT>(v.y, sv);
      v0 = make_uint4(a.x, a.y, b.x, b.y);
      a = codes_to_bf16x4<FMT>(v.z, sv); b = codes_to_bf16x4<FMT>(v.w, sv);
      v1 = make_uint4(a.x, a.y, b.x, b.y);
    }
    uint4* const ko = reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.k_out) + row * D) + 2 * lane;
    uint4* const vo = reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.v_out) + row * D) + 2 * lane;
    ko[0] = k0; ko[1] = k1;
    vo[0] = v0; vo[1] = v1;
  }
}

namespace {

unsigned blocks_for(long long rows, int rows_per_block, int sm_count) {
  const long long need = (rows + rows_per_block - 1) / rows_per_block, most = (long long)sm_count * 8;
  return (unsigned)(need < most ? need : most);
}
template <int D, int FMT>
cudaError_t quantize_t(const KvWrite& w, bool gather, int sm_count, cudaStream_t st) {
  const dim3 grid(blocks_for((long long)w.B * w.n * w.Hkv, NT / (D / 8), sm_count));
  return gather ? launch_chained(kv_quantize_kernel<D, FMT, true>, grid, dim3(NT), 0, st, 1, w)
                : launch_chained(kv_quantize_kernel<D, FMT, false>, grid, dim3(NT), 0, st, 1, w);
}
template <int D, int FMT>
cudaError_t dequantize_t(const KvRead& r, int sm_count, cudaStream_t st) {
  return launch_chained(kv_dequantize_kernel<D, FMT>, dim3(blocks_for((long long)r.B * r.n * r.Hkv, NT / (D / 16), sm_count)), dim3(NT), 0, st, 1, r);
}

}  // namespace

cudaError_t launch_kv_quantize(const KvWrite& w, int format, int d, bool gather, int sm_count, cudaStream_t st) {
  if (d == 128) return format == FMT_INT8 ? quantize_t<128, FMT_INT8>(w, gather, sm_count, st) : quantize_t<128, FMT_E4M3>(w, gather, sm_count, st);
  return format == FMT_INT8 ? quantize_t<64, FMT_INT8>(w, gather, sm_count, st) : quantize_t<64, FMT_E4M3>(w, gather, sm_count, st);
}
cudaError_t launch_kv_dequantize(const KvRead& r, int format, int d, int sm_count, cudaStream_t st) {
  if (d == 128) return format == FMT_INT8 ? dequantize_t<128, FMT_INT8>(r, sm_count, st) : dequantize_t<128, FMT_E4M3>(r, sm_count, st);
  return format == FMT_INT8 ? dequantize_t<64, FMT_INT8>(r, sm_count, st) : dequantize_t<64, FMT_E4M3>(r, sm_count, st);
}

}  // namespace pc
