// Score modification shared by the forward and backward kernels of
// lt_attn_mod_* (internal to liblt).
//
//   s = scale q.k;  capped: s = cap tanh(s / cap);  biased: s -= slope |i - j|
//   query i sees the keys of one interval
//
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

// Stored scores.  The kernels keep a score as t with z = c t + const in base-2
// units, so that a probability is one FMA and one exp2 from it:
//   * without a cap t = q.k and c = scale log2 e;
//   * with one, tanh(x) = 1 - 2 u, u = 1 / (1 + e^(2 x)), x = scale q.k / cap: t = -u,
//     c = 2 cap log2 e, const = cap log2 e, and 1 - tanh^2 = 4 u (1 - u).  The
//     absolute error of z is a few 2^-24 c, so that a probability is off by less than
//     an FP16 half step up to caps of 1000.
// The bias in units of t is slope' |i - j|, slope' = slope log2 e / c.  Without a
// cap it enters as the initial value of the product's FP32 accumulator (its
// rounding there is relative to the bias: only keys whose probability the bias has
// made negligible see it).
template <bool CAP>
struct Score {
  float c, k2, off;        // t -> base-2 units, product -> exponent of u, const
  __device__ __forceinline__ Score(const ScoreMod& m, float scale)
      : c(CAP ? 2.f * m.cap * kModLog2e : scale * kModLog2e),
        k2(CAP ? 2.f * scale / m.cap * kModLog2e : 0.f),
        off(CAP ? m.cap * kModLog2e : 0.f) {}
  __device__ __forceinline__ float t(float s) const {
    if constexpr (CAP) return __builtin_amdgcn_rcpf(-1.f - fast_exp2(s * k2));
    return s;
  }
};

// With a distance bias most pairs of a steep head have no weight: their
// probability is a zero in FP16.  Where that holds for a whole tile of a wave, what
// follows the scores is left out:
//   * forward: probabilities below 2^-kNoneFwd of the row's offset; all such of a row
//     (at most 2^19 keys) are below half a step of its FP32 sum, which is at least 1;
//   * backward: below 2^-kNoneBwd, so that dS is an FP16 zero too, whatever dP - D is
//     (|dP| <= 128 * 65504^2 < 2^39).
// So the results are the same; only a non-finite V or dO behind such a weight is not
// seen.  Non-finite scores are never left out.
constexpr float kNoneFwd = 48.f;
constexpr float kNoneBwd = 66.f;
template <int N>
__device__ __forceinline__ bool all_finite(const f32x16 (&acc)[N]) {
  float m = 0.f;   // 0, or NaN
#pragma unroll
  for (int kb = 0; kb < N; ++kb)
#pragma unroll
    for (int r = 0; r < 16; ++r) m = fmaf(acc[kb][r], 0.f, m);
  return __builtin_amdgcn_ballot_w64(!(m == 0.f)) == 0;
}

// Values -slope' |d0 + n| of a 32-wide accumulator column, n = 8 (r / 4) + r % 4, r < 16,
// step by step of kb (32 more).  `side`: every d0 + n of the wave has that sign (+1, -1),
// or 0: mixed.  With a sign the value is linear in n: one add of a scalar each.
template <int N>
__device__ __forceinline__ void bias_init(f32x16 (&acc)[N], float slope, float d0, int side) {
  if (side != 0) {
    const float m = side > 0 ? -slope : slope;     // wave-uniform
    const float base = m * d0;
#pragma unroll
    for (int kb = 0; kb < N; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[kb][r] = fmaf(m, (float)(kb * 32 + 8 * (r >> 2) + (r & 3)), base);
  } else {
#pragma unroll
    for (int kb = 0; kb < N; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        acc[kb][r] = -slope * fabsf(d0 + (float)(kb * 32 + 8 * (r >> 2) + (r & 3)));
  }
}

// Non-finite values in places that a query does not see.  The products run over whole
// tiles, and 0 x NaN is NaN: a probability or dS of zero does not keep out a
// non-finite V, K, Q or dO.  The kernels pay nothing for that case on the way: where an
// accumulator of a wave ends up non-finite, they form it again one (query, key) pair at a time,
// over the pairs that see each other.
// this lane's half of a row product: features kk * 16 + 8 g + 0..7 of both
template <int KK>
__device__ __forceinline__ float half_dot(const half8 (&f)[KK], const lt_half* row) {
  float s = 0.f;
#pragma nounroll
  for (int kk = 0; kk < KK; ++kk) {
    half8 x = f[0];
#pragma unroll
    for (int i = 1; i < KK; ++i) x = kk == i ? f[i] : x;           // constant register indices
    const half8 y = as_half8(ld16(row + kk * 16));
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf((float)x[e], (float)y[e], s);
  }
  return s;
}
// acc[db][4 rq + e] += w * row[db * 32 + 8 rq + 4 g + e] where `on`
template <int DB>
__device__ __forceinline__ void add_row(f32x16 (&acc)[DB], bool on, float w, const lt_half* row, int g) {
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int rq = 0; rq < 4; ++rq) {
      const half4 x = *reinterpret_cast<const half4*>(row + db * 32 + 8 * rq + 4 * g);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[db][4 * rq + e] = on ? fmaf(w, (float)x[e], acc[db][4 * rq + e]) : acc[db][4 * rq + e];
    }
}

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
