// RMSNorm of every query and key head with the rotary embedding in the same
// pass, forward and backward, gfx950.
//
//   u = w x r,  r = (mean x^2 + eps)^(-1/2) per (token, head)
//   y_i = u_i cos a - u_{i+D/2} sin a,  y_{i+D/2} = u_{i+D/2} cos a + u_i sin a
//   back: g = inverse rotation of dy;  dx = r w g - r^3 x mean(g w x);
//         dw = sum over tokens and heads of g x r
//
// HBM-bound: 4 bytes an element forth, 6 back.  Separate norm and rotation
// passes would move 8 and 12.
//   * one wave per token, so that the token's cosines and sines are read once
//     for all its heads (few heads: several tokens, few tokens: several waves per token);
//     D / 16 lanes (rounded up to a power of two) take a head, each with eight
//     features and their rotation partners, so the rotation stays within a lane
//     and the norm's sum is a few lane exchanges;
//   * FP32 arithmetic, one rounding per output; r kept in FP32 for the backward;
//   * backward: every lane keeps its FP32 part of dw for the query heads, then for
//     the key heads (both at once take 200 registers and lose: 29 us for 27); a
//     workgroup writes one partial row, and qknorm_dw_sum adds the rows in order
//     (deterministic, no atomics).
// 4096 tokens of 40 + 8 heads of 128: forward 18 us (5.6 TB/s), backward 27 us
// (5.6 TB/s) and 4.5 us for the sums.

#include "packed.hpp"

#include "common.hpp"

namespace lt {
namespace {

constexpr int kWaves = kQkNormWaves;

// cosines and sines of the eight pairs 8 i .. 8 i + 7 at a token's position;
// NaN for a position outside the table
__device__ __forceinline__ void load_angles(const QkNormArgs& a, int64_t t, int i, float (&co)[8], float (&si)[8]) {
  const int p = a.POS ? a.POS[t] : (int)(t % a.S);
  const bool ok = p >= 0 && p < a.P;
  const float4* cs = reinterpret_cast<const float4*>(a.CS + ((int64_t)(ok ? p : 0) * (a.D / 2) + i * 8) * 2);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float4 v = cs[q];
    co[2 * q] = ok ? v.x : NAN;
    si[2 * q] = ok ? v.y : NAN;
    co[2 * q + 1] = ok ? v.z : NAN;
    si[2 * q + 1] = ok ? v.w : NAN;
  }
}

template <int LPR>
__device__ __forceinline__ float row_sum(float v) {   // over the LPR lanes of a head
#pragma unroll
  for (int m = LPR / 2; m >= 1; m >>= 1) v += __shfl_xor(v, m);
  return v;
}

// LPR lanes per head row
template <int LPR>
__global__ void __launch_bounds__(64 * kWaves)
qknorm_fwd_kernel(const QkNormArgs a, const HeadSplit hs, lt_half* Y, int64_t ldy, float* __restrict__ RSTD,
                  float eps) {
  constexpr int RPW = 64 / LPR;                    // head rows per wave
  const int lane = threadIdx.x & 63;
  const unsigned unit = blockIdx.x * kWaves + (threadIdx.x >> 6);
  const int row = lane / LPR, i = lane % LPR;
  const int64_t t = (int64_t)(unit / hs.parts) * (RPW >> hs.shift) + (row >> hs.shift);
  if (t >= a.T) return;                            // a head row's lanes leave together
  const int half = a.D / 2, heads = a.Hq + a.Hkv;
  const bool in = i * 8 < half;
  float co[8], si[8];
  load_angles(a, t, in ? i : 0, co, si);
  const float inv_d = 1.f / (float)a.D;
  const int first = ((unit % hs.parts) << hs.shift) + (row & ((1 << hs.shift) - 1));
  for (int h = first; h < heads; h += hs.parts << hs.shift) {
    const lt_half* x = a.X + t * a.ldx + (int64_t)h * a.D + i * 8;
    const lt_half* w = (h < a.Hq ? a.Wq : a.Wk) + i * 8;
    const u32x4 zero = {0, 0, 0, 0};
    const half8 x1 = as_half8(in ? ld16(x) : zero), x2 = as_half8(in ? ld16(x + half) : zero);
    const half8 w1 = as_half8(in ? ld16(w) : zero), w2 = as_half8(in ? ld16(w + half) : zero);
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss += (float)x1[e] * (float)x1[e] + (float)x2[e] * (float)x2[e];
    ss = row_sum<LPR>(ss);
    const float r = 1.f / sqrtf(ss * inv_d + eps);
    half8 y1, y2;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float u1 = (float)w1[e] * ((float)x1[e] * r), u2 = (float)w2[e] * ((float)x2[e] * r);
      y1[e] = (_Float16)(u1 * co[e] - u2 * si[e]);
      y2[e] = (_Float16)(u2 * co[e] + u1 * si[e]);
    }
    if (in) {
      lt_half* y = Y + t * ldy + (int64_t)h * a.D + i * 8;
      st16(y, as_u32x4(y1));
      st16(y + half, as_u32x4(y2));
    }
    if (i == 0) RSTD[t * heads + h] = r;
  }
}

template <int LPR>
__global__ void __launch_bounds__(64 * kWaves)
qknorm_bwd_kernel(const QkNormArgs a, const HeadSplit hq, const HeadSplit hk, const lt_half* dY, int64_t lddy, const float* __restrict__ RSTD, lt_half* dX,
                  int64_t lddx, float* __restrict__ part) {
  constexpr int RPW = 64 / LPR;
  __shared__ float red[kWaves][LPR * 16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = lane / LPR, i = lane % LPR;
  const int half = a.D / 2, heads = a.Hq + a.Hkv;
  const bool in = i * 8 < half;
  const float inv_d = 1.f / (float)a.D;
  const u32x4 zero = {0, 0, 0, 0};
  // query heads, then key heads; with gridDim.y = 2 one of them
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    if (gridDim.y == 2 && (int)blockIdx.y != which) continue;
    const HeadSplit hs = which ? hk : hq;
    const unsigned units = (unsigned)hs.groups * hs.parts;
    const lt_half* W = which ? a.Wk : a.Wq;
    const int h0 = which ? a.Hq : 0, h1 = which ? heads : a.Hq;
    const half8 w1 = as_half8(in ? ld16(W + i * 8) : zero), w2 = as_half8(in ? ld16(W + half + i * 8) : zero);
    float dw[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) dw[e] = 0.f;
    for (unsigned unit = blockIdx.x * kWaves + wave; unit < units; unit += gridDim.x * kWaves) {
      const int64_t t = (int64_t)(unit / hs.parts) * (RPW >> hs.shift) + (row >> hs.shift);
      if (t >= a.T) continue;                      // a head row's lanes together
      float co[8], si[8];
      load_angles(a, t, in ? i : 0, co, si);
      const int first = h0 + ((unit % hs.parts) << hs.shift) + (row & ((1 << hs.shift) - 1));
      for (int h = first; h < h1; h += hs.parts << hs.shift) {
        const lt_half* x = a.X + t * a.ldx + (int64_t)h * a.D + i * 8;
        const lt_half* dy = dY + t * lddy + (int64_t)h * a.D + i * 8;
        const half8 x1 = as_half8(in ? ld16(x) : zero), x2 = as_half8(in ? ld16(x + half) : zero);
        const half8 y1 = as_half8(in ? ld16(dy) : zero), y2 = as_half8(in ? ld16(dy + half) : zero);
        const float r = RSTD[t * heads + h];
        float g1[8], g2[8], dot = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          g1[e] = (float)y1[e] * co[e] + (float)y2[e] * si[e];
          g2[e] = (float)y2[e] * co[e] - (float)y1[e] * si[e];
          dw[e] += g1[e] * ((float)x1[e] * r);
          dw[8 + e] += g2[e] * ((float)x2[e] * r);
          g1[e] *= (float)w1[e];
          g2[e] *= (float)w2[e];
          dot += g1[e] * (float)x1[e] + g2[e] * (float)x2[e];
        }
        const float m = r * r * r * row_sum<LPR>(dot) * inv_d;
        half8 o1, o2;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          o1[e] = (_Float16)(r * g1[e] - m * (float)x1[e]);
          o2[e] = (_Float16)(r * g2[e] - m * (float)x2[e]);
        }
        if (in) {
          lt_half* dx = dX + t * lddx + (int64_t)h * a.D + i * 8;
          st16(dx, as_u32x4(o1));
          st16(dx + half, as_u32x4(o2));
        }
      }
    }
    // the wave's rows, then the workgroup's waves, in a fixed order
#pragma unroll
    for (int e = 0; e < 16; ++e)
#pragma unroll
      for (int m = LPR; m < 64; m <<= 1) dw[e] += __shfl_xor(dw[e], m);
    if (lane < LPR) {
#pragma unroll
      for (int e = 0; e < 16; ++e) red[wave][lane * 16 + e] = dw[e];
    }
    __syncthreads();
    for (int k = threadIdx.x; k < LPR * 16; k += 64 * kWaves) {
      const int c = k / 16, e = k % 16;            // lane of the row, its feature
      if (c * 8 < half) {
        float s = red[0][k];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) s += red[w][k];
        part[(int64_t)blockIdx.x * 2 * a.D + which * a.D + (e < 8 ? 0 : half) + c * 8 + (e & 7)] = s;
      }
    }
    __syncthreads();
  }
}

// dWq, dWk = sums of the partial rows.  Workgroup = 16 waves over 16 columns, so that a
// wave holds four rows of them: row group k of 64 sums partial rows k, k + 64, ... in
// order (eight loads in flight at a time), then the groups' sums are added in order.
constexpr int kSumWaves = 16;
constexpr int kSumCols = 16;

__global__ void __launch_bounds__(64 * kSumWaves)
qknorm_dw_sum_kernel(const float* __restrict__ part, int nparts, int D, lt_half* __restrict__ dWq,
                     lt_half* __restrict__ dWk) {
  constexpr int NG = 64 * kSumWaves / kSumCols;    // row groups
  __shared__ float red[NG][kSumCols];
  const int col = threadIdx.x % kSumCols, grp = threadIdx.x / kSumCols;
  const int j = blockIdx.x * kSumCols + col;       // 2 D is a multiple of 16
  float s = 0.f;
  for (int t = grp; t < nparts; t += 8 * NG) {
    float v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int tu = t + u * NG;
      v[u] = tu < nparts ? part[(int64_t)tu * 2 * D + j] : 0.f;
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) s += v[u];
  }
  red[grp][col] = s;
  __syncthreads();
  if (grp == 0) {
    float tot = 0.f;
#pragma unroll
    for (int v = 0; v < NG; ++v) tot += red[v][col];
    reinterpret_cast<_Float16*>(j < D ? dWq : dWk)[j < D ? j : j - D] = (_Float16)tot;
  }
}

// calls f with the lanes per head row as a constant
template <class F>
hipError_t with_lanes(int D, F f) {
  const int n = qknorm_lanes(D);
  if (n == 1) return f(std::integral_constant<int, 1>{});
  if (n == 2) return f(std::integral_constant<int, 2>{});
  if (n == 4) return f(std::integral_constant<int, 4>{});
  if (n == 8) return f(std::integral_constant<int, 8>{});
  return f(std::integral_constant<int, 16>{});
}

}  // namespace

hipError_t qknorm_fwd_launch(const QkNormArgs& a, lt_half* Y, int64_t ldy, float* RSTD, float eps, hipStream_t s) {
  const HeadSplit hs = qknorm_split(a.T, a.Hq + a.Hkv, a.D);
  return with_lanes(a.D, [&](auto L) {
    hipLaunchKernelGGL((qknorm_fwd_kernel<decltype(L)::value>), dim3((unsigned)qknorm_blocks(hs)), dim3(64 * kWaves),
                       0, s, a, hs, Y, ldy, RSTD, eps);
    return hipGetLastError();
  });
}

hipError_t qknorm_bwd_launch(const QkNormArgs& a, const lt_half* dY, int64_t lddy, const float* RSTD, lt_half* dX,
                             int64_t lddx, lt_half* dWq, lt_half* dWk, float* part, hipStream_t s) {
  const int nblk = qknorm_bwd_blocks(a.T, a.Hq, a.Hkv, a.D);
  const HeadSplit hq = qknorm_split(a.T, a.Hq, a.D), hk = qknorm_split(a.T, a.Hkv, a.D);
  const hipError_t e = with_lanes(a.D, [&](auto L) {
    hipLaunchKernelGGL((qknorm_bwd_kernel<decltype(L)::value>), dim3((unsigned)nblk, nblk <= 256 ? 2 : 1),
                       dim3(64 * kWaves), 0, s, a, hq, hk, dY, lddy, RSTD, dX, lddx, part);
    return hipGetLastError();
  });
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(qknorm_dw_sum_kernel, dim3((unsigned)(2 * a.D / kSumCols)), dim3(64 * kSumWaves), 0, s, part,
                     nblk, a.D, dWq, dWk);
  return hipGetLastError();
}

}  // namespace lt
