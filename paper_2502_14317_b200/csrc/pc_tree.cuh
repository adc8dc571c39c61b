// What the kernels on paged caches and drafted tokens share: positions' angles, places of entries, who sees whom.
#pragma once
#include "pc_sm100.cuh"
#include "pc_tree.h"

namespace pc {

// Part of a turn of pair t.  Every lane has another pair, and the constant cache serves one address at a time: sixteen uniform loads and choices.
__device__ __forceinline__ double part_of_turn(const Turns& u, int t) {
  double c = u.coarse[0], f = u.fine[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    if (t / 8 == i) c = u.coarse[i];
    if (t % 8 == i) f = u.fine[i];
  }
  return c * f;
}
// (cos, sin) of the angle of position p.  What p times the fp64 part of a turn leaves without whole turns goes to fp32 in two parts, the second, under 2^-25 of a
// turn, as a step along the circle.  The part of a turn and its product with p are roundings of fp64: the angle is off by up to 2^-51 p (found: 2^-52 p, 4.6e-7
// at 2^31), which up to positions of some 2^27 is less than the error of fp32's sine and cosine.  (Without the second part 2.8 % of random calls had a query's element on the other side of a border between two bf16 numbers than in 64 bits, with it 1.8 %.)
__device__ __forceinline__ float2 turned(double per, long long p) {
  const double x = per * (double)p, y = x - rint(x);
  const float f = (float)y, step = (float)(y - (double)f) * 6.2831853f;
  float s, c;
  sincospif(2.0f * f, &s, &c);
  return make_float2(fmaf(-s, step, c), fmaf(c, step, s));
}

__device__ __forceinline__ int page_of(const Pages& p, int e) { return (int)((unsigned long long)(unsigned)e * p.mul >> p.shift); }

// Who sees whom among the w <= 64 tokens of a sequence: lane l holds the tokens l and l + 32, bit j of a token's word: it sees token j (itself
// among them); 0: it is not there.  A parent in [0, token) or -1 (the context's end) is one; anything else, -2 by custom, says that the
// token is not there, and so are its descendants.  Every lane jumps to its ancestors in steps that double: log2(w) rounds.  The whole warp calls.
struct Seen {
  unsigned long long a, b;
  __device__ __forceinline__ unsigned long long of(int token) const {
    const unsigned long long x = __shfl_sync(0xFFFFFFFFu, a, token & 31), y = __shfl_sync(0xFFFFFFFFu, b, token & 31);
    return token < 32 ? x : y;
  }
};
__device__ __forceinline__ Seen tree_seen(const int* parents, int w, int lane) {
  Seen s;
  if (parents == nullptr) {
    s.a = lane < w ? (2ull << lane) - 1 : 0;
    s.b = lane + 32 < w ? (lane == 31 ? ~0ull : (2ull << (lane + 32)) - 1) : 0;
    return s;
  }
  auto first = [&](int i) {
    const int p = i < w ? __ldg(parents + i) : -2;
    return p < -1 || p >= i ? -2 : p;
  };
  int ja = first(lane), jb = first(lane + 32);
  s.a = 1ull << lane;
  s.b = 1ull << (lane + 32);
  for (int reach = 1; reach < w; reach *= 2) {
    auto jump = [&](int j, unsigned long long& bits) {
      const int from = j < 0 ? 0 : j;
      const unsigned long long got = s.of(from);
      const int x = __shfl_sync(0xFFFFFFFFu, ja, from & 31), y = __shfl_sync(0xFFFFFFFFu, jb, from & 31);
      if (j < 0) return j;
      bits |= got;
      return from < 32 ? x : y;
    };
    unsigned long long na = s.a, nb = s.b;
    const int ka = jump(ja, na), kb = w > 32 ? jump(jb, nb) : jb;
    s.a = na; s.b = nb; ja = ka; jb = kb;
  }
  if (ja != -1) s.a = 0;
  if (jb != -1) s.b = 0;
  return s;
}

}  // namespace pc
