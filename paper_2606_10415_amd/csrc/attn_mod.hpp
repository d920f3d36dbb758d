// Score modification shared by the forward and backward kernels of
// lt_attn_mod_* (internal to liblt).
//
//   s = scale q.k;  capped: s = cap tanh(s / cap);  biased: s -= slope |i - j|
//   query i sees the keys of one interval
//
// The kernels keep modified scores in base-2 units (z = s log2 e).
#pragma once

#include "packed.hpp"

#include "attn_tiles.hpp"

namespace lt {

constexpr float kModLog2e = 1.4426950408889634f;
constexpr float kModLn2 = 0.6931471805599453f;

// Visible keys lo .. hi - 1 of query i, clamped to 0 .. S; none: lo = hi = 0.
__device__ __forceinline__ void row_interval(const ScoreMod& m, int causal, int b, int S, int i, int& lo, int& hi) {
  lo = 0;
  hi = 0;
  if (i >= S) return;
  hi = causal ? i + 1 : S;
  if (m.lo) lo = max(m.lo[(int64_t)b * S + i], 0);
  if (m.hi) hi = min(m.hi[(int64_t)b * S + i], hi);
  if (lo >= hi) lo = hi = 0;
}

// The cap in base-2 units: z = C tanh(s / cap), C = cap log2 e, s the raw
// product.  With u = 1 / (1 + e^(2 s scale / cap)): tanh = 1 - 2 u and
// 1 - tanh^2 = 4 u (1 - u).  The absolute error is a few 2^-24 C, so that a
// probability is off by less than an FP16 half step up to caps of 1000.
struct Cap {
  float k2, c, c2;
  __device__ __forceinline__ Cap(float cap, float scale)
      : k2(cap > 0.f ? 2.f * scale / cap * kModLog2e : 0.f), c(cap * kModLog2e), c2(-2.f * cap * kModLog2e) {}
  __device__ __forceinline__ float u(float s) const {
    return __builtin_amdgcn_rcpf(1.f + fast_exp2(s * k2));
  }
  __device__ __forceinline__ float z(float u) const { return fmaf(c2, u, c); }
};

__device__ __forceinline__ int wave_min32(int v) {   // over lane % 32
#pragma unroll
  for (int m = 16; m >= 1; m >>= 1) v = min(v, __shfl_xor(v, m));
  return v;
}
__device__ __forceinline__ int wave_max32(int v) {
#pragma unroll
  for (int m = 16; m >= 1; m >>= 1) v = max(v, __shfl_xor(v, m));
  return v;
}

// Hull of the 32 queries whose intervals the lanes (lane % 32) hold; rows past
// S (valid = false) do not count.  Wave-uniform.
__device__ __forceinline__ QueryHull query_hull(int lo, int hi, bool valid) {
  const bool some = lo < hi;
  QueryHull h;
  h.lo = __builtin_amdgcn_readfirstlane(wave_min32(some ? lo : 0x7fffffff));
  h.hi = __builtin_amdgcn_readfirstlane(wave_max32(some ? hi : 0));
  h.all_lo = __builtin_amdgcn_readfirstlane(wave_max32(!valid ? 0 : some ? lo : 0x7fffffff));
  h.all_hi = __builtin_amdgcn_readfirstlane(wave_min32(!valid ? 0x7fffffff : some ? hi : 0));
  return h;
}

}  // namespace lt
