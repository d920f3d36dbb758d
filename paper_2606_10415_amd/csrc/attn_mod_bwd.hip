// Attention backward with modified scores, gfx950.
//
//   z = cap tanh(scale q.k / cap) - slope |i - j|,  P = exp(z - LSE) on visible pairs
//   dP = dO V^T,  dZ = P (dP - D),  D_i = rowsum(dO_i * O_i),  dS = dZ (1 - tanh^2)
//   dV = P^T dO,  dK = scale dS^T Q,  dQ = scale dS K
// with dK and dV summed over the query heads of a kv head.  A query that sees no
// key has dQ = 0, a key that no query sees dK = dV = 0.
//
// Kernels, none with an atomic:
//   1. attn_mod_rows: D_i and the base-2 LSE of every query and head; the
//      clamped interval of every query and the hull of every 32 queries'
//      intervals, which the other passes select their blocks by.  attn_mod_delta:
//      D_i again, in FP32, where the FP16 O is too coarse for it.
//   2. attn_mod_dkdv: key-major.  One workgroup per (batch, kv head, 256-key
//      tile); each of 8 waves owns 32 keys, with their K fragments and the dK, dV
//      accumulators in registers.  It lists the 64-query blocks that see some of
//      its keys, then streams (query head, listed block) pairs HBM -> LDS, double-
//      buffered.  S = Q K^T and dP = dO V^T put one key in a lane, so that P and
//      dS feed the dV / dK products from registers.  A wave skips the 32-query
//      groups that see none of its keys and compares key against interval only
//      where a group sees them in part.  It stores dS as FP16 blocks of 32 x 32 (the
//      rounding of any FP16 matrix operand).  Few workgroups: 128-key tiles whose
//      wave pairs share keys and split the queries, and shares of a tile's pairs
//      with FP32 partial sums in the workspace, added in order by attn_mod_sum.
//   3. attn_mod_dq: query-major dQ = scale dS K from the stored blocks.
// The (batch, kv head) pairs are taken in chunks, 2 and 3 for each, so that the
// workspace holds one chunk's dS.

#include <type_traits>

#include "attn_mod.hpp"

namespace lt {
namespace {

// Direct load of 16 bytes per lane into LDS, as lds_dma16_opaque, for data
// read once (non-temporal).  The wait states cover a descriptor word that a
// v_readfirstlane has just written as well as m0.
__device__ __forceinline__ void lds_dma16_stream(const void* base, uint32_t nrec, void* lds, uint32_t voff) {
  const uint64_t b = (uint64_t)base;
  u32x4 r;
  r[0] = __builtin_amdgcn_readfirstlane((uint32_t)b);
  r[1] = __builtin_amdgcn_readfirstlane((uint32_t)(b >> 32) & 0xffffu);
  r[2] = __builtin_amdgcn_readfirstlane(nrec);
  r[3] = 0x00020000u;
  const uint32_t m0v = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)lds);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds"
               :
               : "s"(m0v), "v"(voff), "s"(r)
               : "memory");
}

constexpr int NWA = 8;         // dK/dV: waves per workgroup
constexpr int BKV = NWA * 32;  // dK/dV: keys per workgroup (32 per wave)
constexpr int BQA = 64;        // dK/dV: queries per block (two 32-query halves)
constexpr int kMaxBlocks = kModMaxS / BQA;
// marks of dS blocks (with a distance bias): 0 no weight, found before the dK/dV pass,
// which then does not visit the block; kZeroBlock none either, found by that pass
constexpr uint8_t kLiveBlock = 1, kZeroBlock = 2;

// dS blocks of a head; block (query group qg, key group kg)
__device__ __forceinline__ int64_t ds_blocks(int n32, int causal) {
  return causal ? (int64_t)n32 * (n32 + 1) / 2 : (int64_t)n32 * n32;
}
__device__ __forceinline__ int64_t ds_block(int qg, int kg, int n32, int causal) {
  return causal ? (int64_t)qg * (qg + 1) / 2 + kg : (int64_t)qg * n32 + kg;
}

// ------------------------------------------------------------ 1: row terms, intervals, hulls
// D_i = rowsum(dO_i * O_i) = sum_j P_ij dP_ij.  Formed from the FP16 O, D is off by
// about 2^-12 |dO| |O|.  Where a softmax is spread over many keys |O| is small
// against |v| and that drowns in the rounding of dS; where it rests on a few keys
// dP - D cancels and it does not: with scores of standard deviation 9 it took
// the error of dQ and dK from 2.9e-4 to 5.5e-4 of their norm.  So queries whose O
// is not small are marked sharp, and attn_mod_delta forms their D again: those with
// |O|^2 > kFlat |v|^2 (v at the same position) in groups of 32 that are so on average, and
// elsewhere those with four times that.  At kFlat the D of the FP16 O adds 0.7e-4.
constexpr int kTile = kSharpTile;
constexpr float kFlat = 1.f / 16.f;

// Intervals and hulls of the 256 queries of block blk of the batch rows, a lane each.
__device__ __forceinline__ void rows_and_hulls(const AttnModBwdArgs& a, int blk) {
  const int B = a.sh.B, S = a.sh.S, n_sb = (S + 255) / 256;
  const int b = blk / n_sb, q = (blk % n_sb) * 256 + threadIdx.x;
  int lo, hi;
  row_interval(a.mod, a.sh.causal, b, S, q, lo, hi);
  if (q < S) {
    a.rows[(int64_t)b * S + q] = lo;
    a.rows[(int64_t)(B + b) * S + q] = hi;
  }
  // both halves of the wave are a group of 32
  const bool some = lo < hi;
  QueryHull h;
  h.lo = wave_min32(some ? lo : 0x7fffffff);
  h.hi = wave_max32(some ? hi : 0);
  h.all_lo = wave_max32(q >= S ? 0 : some ? lo : 0x7fffffff);
  h.all_hi = wave_min32(q >= S ? 0x7fffffff : some ? hi : 0);
  if ((threadIdx.x & 31) == 0 && q < S) a.hulls[(int64_t)b * ((S + 31) / 32) + q / 32] = h;
}

// Workgroups 0 .. n_tile - 1: 128 queries of one head, D / 8 lanes to a row (whole
// rows, coalesced).  The others: intervals and hulls.  HBM-bound: O and dO of 8192 tokens
// of 64 heads, 63 us (4.6 TB/s).
template <int D, bool CAP>
__global__ void __launch_bounds__(256)
attn_mod_rows_kernel(const AttnModBwdArgs a, unsigned n_tile) {
  __shared__ float2 norm_s[kTile];                 // |O|^2 - kFlat |v|^2, |v|^2
  const int B = a.sh.B, S = a.sh.S, Hq = a.sh.Hq;
  if (blockIdx.x >= n_tile) return rows_and_hulls(a, blockIdx.x - n_tile);
  constexpr int CPR = D / 8, RPI = 256 / CPR;      // lanes per row, rows per pass
  const int bh = blockIdx.x % (B * Hq);
  const int q0 = (int)(blockIdx.x / (B * Hq)) * kTile;
  const int b = bh / Hq, h = bh % Hq, kvh = h / (Hq / a.sh.Hkv);
  const int c8 = (threadIdx.x % CPR) * 8;
  const Score<CAP> sc(a.mod, a.sh.scale);
#pragma unroll
  for (int it = 0; it < kTile / RPI; ++it) {
    const int r = it * RPI + threadIdx.x / CPR, q = q0 + r;
    const u32x4 zero = {0, 0, 0, 0};
    const int64_t row = (int64_t)b * S + q, off = row * a.o_stride + (int64_t)h * D + c8;
    const half8 x = as_half8(q < S ? ld16(a.dO + off) : zero);
    const half8 o = as_half8(q < S ? ld16(a.O + off) : zero);
    const half8 v = as_half8(q < S ? ld16(a.V + row * a.kv_stride + (int64_t)kvh * D + c8) : zero);
    float d = 0.f, o2 = 0.f, v2 = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      d = fmaf((float)x[e], (float)o[e], d);
      o2 = fmaf((float)o[e], (float)o[e], o2);
      v2 = fmaf((float)v[e], (float)v[e], v2);
    }
#pragma unroll
    for (int m = CPR / 2; m >= 1; m >>= 1) {
      d += __shfl_xor(d, m);
      o2 += __shfl_xor(o2, m);
      v2 += __shfl_xor(v2, m);
    }
    if (c8 == 0) norm_s[r] = make_float2(o2 - kFlat * v2, v2);
    if (c8 == 0 && q < S) {
      const int64_t ri = (int64_t)bh * S + q;
      a.delta[ri] = d;
      a.lse2[ri] = a.LSE[ri] * kModLog2e - sc.off;
    }
  }
  __syncthreads();
  if (threadIdx.x < kTile) {                       // whole waves
    const float2 n = norm_s[threadIdx.x];
    float sum = n.x;
#pragma unroll
    for (int m = 16; m >= 1; m >>= 1) sum += __shfl_xor(sum, m);
    const uint64_t bal = __builtin_amdgcn_ballot_w64(sum <= 0.f ? !(n.x <= 3.f * kFlat * n.y) : !(n.x <= 0.f));
    if ((threadIdx.x & 31) == 0)
      a.sharp[((int64_t)bh * ((S + kTile - 1) / kTile) + q0 / kTile) * (kTile / 32) + threadIdx.x / 32] =
          (uint32_t)(threadIdx.x & 32 ? bal >> 32 : bal);
  }
}

// D of the sharp queries in FP32 from S and dP, as the forward forms O: two
// products.  One workgroup per (128 queries, or 64 with QSPLIT = 2 where the two waves of
// a query group take one 32-key block of a slice each) of one head; they walk the keys
// of their sharp queries.  `all` (short sequences, where another launch costs more than
// these products): every query is taken, the base-2 LSE is written too, and the
// workgroups from n_tile on do the intervals and hulls, in place of attn_mod_rows.
// With a distance bias the pass also says which dS blocks have any weight.
// Bound as the forward is, with two products to its two and one exp2.  8192 tokens of
// 64:8 heads of normal inputs, where few queries are sharp: 21 us; 2048 tokens of 40:8 heads, capped,
// window of 683: 54 us; 4096 tokens of 40 heads with ALiBi slopes: 104 us.
constexpr int NWD = 4;            // waves
constexpr int BKD = 64;           // keys per slice

template <int D, int QSPLIT, bool CAP, bool BIAS>
__global__ void __launch_bounds__(NWD * 64, 2)
attn_mod_delta_kernel(const AttnModBwdArgs a, int all, unsigned n_tile) {
  using RT = RowTile<D, NWD>;
  constexpr int KK = D / 16;
  constexpr int NQG = NWD / QSPLIT;                // query groups of 32
  constexpr int BQW = NQG * 32;                    // queries per workgroup
  constexpr int KBW = BKD / 32 / QSPLIT;           // 32-key blocks per slice and wave
  constexpr int TILE = BKD * RT::ROWB, STAGE = 2 * TILE;
  __shared__ __attribute__((aligned(1024))) char smem[2 * STAGE];
  __shared__ int hull_s[2][NWD];

  const int B = a.sh.B, S = a.sh.S, Hq = a.sh.Hq, Hkv = a.sh.Hkv, causal = a.sh.causal;
  if (blockIdx.x >= n_tile) return rows_and_hulls(a, blockIdx.x - n_tile);
  const int n_qt = (S + BQW - 1) / BQW;
  const int qt = n_qt - 1 - (int)(blockIdx.x / (B * Hq));   // later queries mostly see more keys: longest first
  int b, h;
  query_head(blockIdx.x % (B * Hq), B, Hq, Hkv, b, h);
  const uint32_t* marks = a.sharp + ((int64_t)b * Hq + h) * ((S + kTile - 1) / kTile) * (kTile / 32) + qt * NQG;
  if (!all && !BIAS) {
    uint32_t any = 0;
#pragma unroll
    for (int w = 0; w < NQG; ++w) any |= marks[w];
    if (!any) return;
  }

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lrow = lane & 31, g = lane >> 5;
  const int qg = wave % NQG, kpart = wave / NQG;
  const int kvh = h / (Hq / Hkv);
  const int qw0 = qt * BQW + qg * 32;
  const int myq = qw0 + lrow;                      // query owned by this lane
  const lt_half* Kp = a.K + (int64_t)b * S * a.kv_stride + (int64_t)kvh * D;
  const lt_half* Vp = a.V + (int64_t)b * S * a.kv_stride + (int64_t)kvh * D;
  const int64_t row = (int64_t)b * S + (myq < S ? myq : 0), ri = ((int64_t)b * Hq + h) * S + myq;

  const Score<CAP> sc(a.mod, a.sh.scale);
  const float lse2 = myq < S ? (all ? a.LSE[ri] * kModLog2e - sc.off : a.lse2[ri]) : 0.f;
  if (all && myq < S && g == 0 && kpart == 0) {
    a.lse2[ri] = lse2;
    a.delta[ri] = 0.f;                             // kept by queries that see nothing
  }
  int lo = 0, hi = 0;
  const uint32_t sharp = all ? ~0u : (uint32_t)__builtin_amdgcn_readfirstlane(qw0 < S ? marks[qg] : 0);
  if (BIAS || (sharp >> lrow & 1)) row_interval(a.mod, causal, b, S, myq, lo, hi);
  QueryHull wh = query_hull(lo, hi, myq < S);
  // with a distance bias: a group is taken whole or not at all, and finds which of its
  // dS blocks have any weight (kNoneBwd); a group that is not taken calls them live
  const int g32 = qt * NQG + qg;
  uint8_t* const live = a.live + ((int64_t)b * Hq + h) * ds_blocks((S + 31) / 32, causal) +
                        ds_block(qw0 < S ? g32 : 0, 0, (S + 31) / 32, causal);
  const int kg_lo = wh.lo < wh.hi ? wh.lo >> 5 : 0, kg_hi = wh.lo < wh.hi ? (wh.hi + 31) >> 5 : 0;
  if (BIAS && sharp == 0) {
    if (kpart == 0)
      for (int kg = kg_lo + lane; kg < kg_hi; kg += 64) live[kg] = kLiveBlock;
    wh.lo = 0x7fffffff;
    wh.hi = 0;
  }
  if (lane == 0) {
    hull_s[0][wave] = wh.lo;
    hull_s[1][wave] = wh.hi;
  }
  __syncthreads();
  int wg_lo = 0x7fffffff, wg_hi = 0;
#pragma unroll
  for (int w = 0; w < NWD; ++w) {
    wg_lo = min(wg_lo, hull_s[0][w]);
    wg_hi = max(wg_hi, hull_s[1][w]);
  }
  if (wg_lo >= wg_hi) return;                      // the same in every wave
  const int kt0 = __builtin_amdgcn_readfirstlane(wg_lo / BKD);
  const int kt1 = __builtin_amdgcn_readfirstlane((wg_hi + BKD - 1) / BKD);

  // Q and dO fragments (B operands of S^T = K Q^T and dP^T = V dO^T)
  half8 qf[KK], gf[KK];
  {
    const lt_half* qp = a.Q + row * a.q_stride + (int64_t)h * D + g * 8;
    const lt_half* gp = a.dO + row * a.o_stride + (int64_t)h * D + g * 8;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      qf[kk] = as_half8(myq < S ? ld16(qp + kk * 16) : u32x4{0, 0, 0, 0});
      gf[kk] = as_half8(myq < S ? ld16(gp + kk * 16) : u32x4{0, 0, 0, 0});
    }
  }
  const float slope = BIAS ? a.mod.slopes[h] * kModLog2e / sc.c : 0.f;   // in units of the stored scores
  uint32_t rlane[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) rlane[kk] = (uint32_t)RT::addr(lane & 31, kk * 2 + (lane >> 5));
  auto stage_load = [&](int kt, int buf) {
    char* st = smem + buf * STAGE;
    const int key0 = kt * BKD;
    RT::template dma<BKD>(st, Kp + (int64_t)key0 * a.kv_stride, a.kv_stride, S - key0, wave, lane);
    RT::template dma<BKD>(st + TILE, Vp + (int64_t)key0 * a.kv_stride, a.kv_stride, S - key0, wave, lane);
  };
  stage_load(kt0, 0);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) {
    loaded_here(qf[kk]);
    loaded_here(gf[kk]);
  }
  // this lane's shares of sum P dP and of sum P, which the LSE's rounding leaves 1e-7 or
  // so off 1: their quotient is a D that a row of one key cancels exactly
  float dex = 0.f, psum = 0.f;
  auto slice = [&](int kt, auto CUR_) {
    constexpr int cur = decltype(CUR_)::value;
    const char* st = smem + cur * STAGE;
    if (kt + 1 < kt1) stage_load(kt + 1, cur ^ 1);
    const int kb0 = QSPLIT > 1 ? kpart * 32 : 0;
    const int key0 = kt * BKD + kb0;
    if (key0 < wh.hi && key0 + KBW * 32 > wh.lo) {
      f32x16 sacc[KBW], pacc[KBW];
      const float d0 = (float)(key0 + 4 * g - myq);
      // keys all from, or all up to, the wave's queries
      const int side = key0 >= qw0 + 31 ? 1 : key0 + KBW * 32 - 1 <= qw0 ? -1 : 0;
#pragma unroll
      for (int kb = 0; kb < KBW; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          sacc[kb][r] = 0.f;
          pacc[kb][r] = 0.f;
        }
      if constexpr (BIAS && !CAP) bias_init(sacc, slope, d0, side);
      auto rd = [&](int off, int kb, int kk) {
        return as_half8(*reinterpret_cast<const u32x4*>(st + off + (kb0 + kb * 32) * RT::ROWB + rlane[kk]));
      };
      half8 kfr[2][KBW], vfr[2][KBW];
      const bool full = key0 >= wh.all_lo && key0 + KBW * 32 <= wh.all_hi;      // wave-uniform
      // scores (with a distance bias first, to see whether they have any weight), then dP
      auto products = [&](auto S_, auto P_) __attribute__((always_inline)) {
        constexpr bool WS = decltype(S_)::value, WP = decltype(P_)::value;
#pragma unroll
        for (int kb = 0; kb < KBW; ++kb) {
          if (WS) kfr[0][kb] = rd(0, kb, 0);
          if (WP) vfr[0][kb] = rd(TILE, kb, 0);
        }
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          if (kk + 1 < KK) {
#pragma unroll
            for (int kb = 0; kb < KBW; ++kb) {
              if (WS) kfr[(kk + 1) & 1][kb] = rd(0, kb, kk + 1);
              if (WP) vfr[(kk + 1) & 1][kb] = rd(TILE, kb, kk + 1);
            }
          }
#pragma unroll
          for (int kb = 0; kb < KBW; ++kb) {
            if (WS) sacc[kb] = mfma32(kfr[kk & 1][kb], qf[kk], sacc[kb]);
            if (WP) pacc[kb] = mfma32(vfr[kk & 1][kb], gf[kk], pacc[kb]);
          }
        }
      };
      bool none = false;
      if constexpr (BIAS) products(std::true_type{}, std::false_type{});
      else products(std::true_type{}, std::true_type{});
      if constexpr (CAP || BIAS) {
        float mx = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < KBW; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            sacc[kb][r] = sc.t(sacc[kb][r]);
            if constexpr (CAP && BIAS)
              sacc[kb][r] = fmaf(-slope, fabsf(d0 + (float)(kb * 32 + 8 * (r >> 2) + (r & 3))), sacc[kb][r]);
            if constexpr (BIAS) mx = fmaxf(mx, sacc[kb][r]);
          }
        if constexpr (BIAS) {
          none = full && __builtin_amdgcn_ballot_w64(!(fmaf(mx, sc.c, -lse2) < -kNoneBwd)) == 0 && all_finite(sacc);
          const int kg = (key0 >> 5) + lane;
          if (lane < KBW && kg >= kg_lo && kg < kg_hi) live[kg] = none ? 0 : kLiveBlock;
          if (!none) products(std::false_type{}, std::true_type{});
        }
      }
      if (!none) {
#pragma unroll
        for (int kb = 0; kb < KBW; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) sacc[kb][r] = fast_exp2(fmaf(sacc[kb][r], sc.c, -lse2));
        if (!full) {
#pragma unroll
          for (int kb = 0; kb < KBW; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int key = key0 + kb * 32 + 8 * (r >> 2) + 4 * g + (r & 3);
              const bool see = (key >= lo) & (key < hi);
              sacc[kb][r] = see ? sacc[kb][r] : 0.f;
              pacc[kb][r] = see ? pacc[kb][r] : 0.f;
            }
        }
#pragma unroll
        for (int kb = 0; kb < KBW; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            psum += sacc[kb][r];
            dex = fmaf(sacc[kb][r], pacc[kb][r], dex);
          }
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  };
  for (int kt = kt0; kt < kt1; kt += 2) {
    slice(kt, std::integral_constant<int, 0>{});
    if (kt + 1 < kt1) slice(kt + 1, std::integral_constant<int, 1>{});
  }
  dex += __shfl_xor(dex, 32);
  psum += __shfl_xor(psum, 32);
  if constexpr (QSPLIT > 1) {
    float2* red = reinterpret_cast<float2*>(smem); // free after the loop's last barrier
    if (kpart == 1) red[qg * 64 + lane] = make_float2(dex, psum);
    __syncthreads();
    if (kpart == 1) return;
    const float2 o = red[qg * 64 + lane];
    dex += o.x;
    psum += o.y;
  }
  if (myq < S && g == 0 && lo < hi && sharp != 0) a.delta[ri] = dex / psum;
}

// ------------------------------------------------------------ 2: dK/dV
template <int D>
struct DkdvSmem {
  using RT = RowTile<D, NWA>;
  static constexpr int TQ = BQA * RT::ROWB;             // one Q or dO block
  // Q and dO buffers first: every fragment read of them is a per-lane
  // register plus a constant below 64 KiB (the LDS instructions' offset field)
  static constexpr int Q_OFF = 0;                        // 2 buffers
  static constexpr int DO_OFF = Q_OFF + 2 * TQ;          // 2 buffers
  // per buffer five rows of 256 B, a 4-byte direct load of 64 lanes each:
  // base-2 LSE, D, interval starts and ends, the two hulls
  static constexpr int NROW = 5;
  static constexpr int ROW_OFF = DO_OFF + 2 * TQ;
  static constexpr int V_OFF = ROW_OFF + 2 * NROW * 256; // V tile [BKV][D]
  static constexpr int BYTES = V_OFF + BKV * RT::ROWB;
  static_assert(BQA == 64 && DO_OFF + 2 * TQ <= 65536, "one load per row, offsets fit the offset field");
};

// Bound by the matrix and vector units in turn, and by registers (no room for
// a second set of scores).  8 D flop a visible pair: 8192 tokens of 64:8 heads in six
// documents 1066 us (820 TFLOP/s); 4096 tokens of 40 heads with ALiBi slopes 315 us, 403
// if the pass finds out itself which blocks have no weight.
// KSPLIT = 1: 8 key groups of 32 (256 keys), every wave walks both 32-query
// halves of each block.  KSPLIT = 2: 4 key groups (128 keys); waves w and w + 4
// own the same keys, take one half each, and their FP32 accumulators are added
// through LDS at the end.
template <int D, int KSPLIT, bool CAP, bool BIAS>
__global__ void __launch_bounds__(NWA * 64, 1)
attn_mod_dkdv_kernel(const AttnModBwdArgs a, int bkv0, int nb) {
  using SM = DkdvSmem<D>;
  using RT = RowTile<D, NWA>;
  constexpr int KK = D / 16;       // MFMA steps over the head dim
  constexpr int DB = D / 32;       // 32-feature blocks
  constexpr int NKG = NWA / KSPLIT;                // key groups of 32
  constexpr int BK = NKG * 32;                     // keys per workgroup
  static_assert(KSPLIT == 1 || NKG * 2 * DB * 4 * 64 * 16 <= SM::BYTES, "reduction fits in LDS");
  __shared__ __attribute__((aligned(1024))) char smem[SM::BYTES];
  __shared__ uint16_t blocks[kMaxBlocks];          // 64-query blocks that see some key of the tile
  __shared__ int counts[NWA];

  const int B = a.sh.B, S = a.sh.S, Hq = a.sh.Hq, Hkv = a.sh.Hkv, causal = a.sh.causal;
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);   // uniform: scalar addressing
  const int lrow = lane & 31;
  const int g = lane >> 5;
  const int kg = wave % NKG;                       // key group
  const int kpart = wave / NKG;                    // query half taken (KSPLIT = 2)

  const int lbkv = blockIdx.x % nb;                // pair within the chunk
  const int slot = blockIdx.x / nb;
  const int nsh = a.plan.nsplit;
  const int jt = slot / nsh;                       // key tile
  const int sp = slot % nsh;                       // share of its pairs
  const int b = (bkv0 + lbkv) / Hkv;
  const int kvh = (bkv0 + lbkv) % Hkv;
  const int G = Hq / Hkv;
  const int n32 = (S + 31) / 32;
  const int64_t nblk = ds_blocks(n32, causal);
  const int kbase = jt * BK;
  const int kw0 = kbase + kg * 32;                 // this wave's first key
  const int mykey = kw0 + lrow;                    // key owned by this lane (S, dP columns)

  const lt_half* Kp = a.K + (int64_t)b * S * a.kv_stride + (int64_t)kvh * D;
  const lt_half* Vp = a.V + (int64_t)b * S * a.kv_stride + (int64_t)kvh * D;
  const QueryHull* hulls = a.hulls + (int64_t)b * n32;

  // ---- V tile -> LDS (B operand of dP = dO V^T); rows past S read as zero ----
  RT::template dma<BK>(smem + SM::V_OFF, Vp + (int64_t)kbase * a.kv_stride, a.kv_stride, S - kbase, wave, lane);
  // ---- K fragments (B operand of S = Q K^T) ----
  half8 kf[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk)
    kf[kk] = mykey < S ? as_half8(ld16(Kp + (int64_t)mykey * a.kv_stride + kk * 16 + g * 8))
                       : as_half8(u32x4{0, 0, 0, 0});

  // ---- list the tile's query blocks, ascending; with a distance bias and room for
  // them the (query head, block) pairs, of those that have a live dS block ----
  const int n_qb = (S + BQA - 1) / BQA;
  const bool pairs = BIAS && (int64_t)G * n_qb <= kMaxBlocks;
  const int n_cand = pairs ? G * n_qb : n_qb;
  int n_list = 0;
  for (int i0 = 0; i0 < n_cand; i0 += NWA * 64) {
    const int code = i0 + tid, i = pairs ? code % n_qb : code;
    bool sees = false;
    if (code < n_cand) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int qg = 2 * i + u;
        if (qg < n32) {
          const QueryHull h = hulls[qg];
          bool on = h.lo < kbase + BK && h.hi > kbase;
          if (BIAS && pairs && on) {
            const uint8_t* live = a.live + ((int64_t)b * Hq + kvh * G + code / n_qb) * nblk;
            on = false;
            for (int k = max(kbase >> 5, h.lo >> 5); k < min((kbase + BK) >> 5, (h.hi + 31) >> 5); ++k)
              on |= live[ds_block(qg, k, n32, causal)] != 0;
          }
          sees |= on;
        }
      }
    }
    const uint64_t bal = __builtin_amdgcn_ballot_w64(sees);
    if (lane == 0) counts[wave] = __popcll(bal);
    __syncthreads();
    int at = n_list;
#pragma unroll
    for (int w = 0; w < NWA; ++w) {
      if (w < wave) at += counts[w];
      n_list += counts[w];
    }
    if (sees) blocks[at + __popcll(bal & ((1ull << lane) - 1))] = (uint16_t)code;
    __syncthreads();
  }
  n_list = __builtin_amdgcn_readfirstlane(n_list);

  // lane part of the row-fragment address of step kk (rows rb + lane % 32,
  // rb a multiple of 16, so the swizzle depends on the lane only)
  uint32_t rlane[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) rlane[kk] = (uint32_t)RT::addr(lane & 31, kk * 2 + (lane >> 5));
  const uint32_t vrow0 = __builtin_amdgcn_readfirstlane(SM::V_OFF + kg * 32 * RT::ROWB);

  f32x16 dkacc[DB], dvacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      dkacc[db][r] = 0.f;
      dvacc[db][r] = 0.f;
    }

  const float scale = a.sh.scale;
  const Score<CAP> sc(a.mod, scale);
  // The (query head, listed block) pairs, head-major, in nsh contiguous shares.
  // Within a head the blocks run last to first: the key tiles of one kv head
  // (on one XCD by the workgroup order) then move in step under a causal mask,
  // and share each Q / dO block through that XCD's L2.
  const int total = pairs ? n_list : G * n_list;
  const int it0 = (int)((int64_t)sp * total / nsh);
  const int n_iter = (int)((int64_t)(sp + 1) * total / nsh) - it0;
  auto pair_of = [&](int i, int& j, int& qbase) {   // j: query head within the group
    const int it = it0 + i;
    if (BIAS && pairs) {                           // heads last to first too
      const int code = __builtin_amdgcn_readfirstlane((int)blocks[n_list - 1 - it]);
      j = code / n_qb;
      qbase = code % n_qb * BQA;
      return;
    }
    j = it / n_list;
    qbase = __builtin_amdgcn_readfirstlane((int)blocks[n_list - 1 - it % n_list]) * BQA;
  };
  // Q, dO, LSE, D and the intervals of queries past S read as zero: they see nothing
  auto stage = [&](int j, int qbase, int buf) {
    const int h = kvh * G + j;
    RT::template dma<BQA>(smem + SM::Q_OFF + buf * SM::TQ,
                          a.Q + ((int64_t)b * S + qbase) * a.q_stride + (int64_t)h * D, a.q_stride, S - qbase,
                          wave, lane);
    RT::template dma<BQA>(smem + SM::DO_OFF + buf * SM::TQ,
                          a.dO + ((int64_t)b * S + qbase) * a.o_stride + (int64_t)h * D, a.o_stride, S - qbase,
                          wave, lane);
    if (wave < SM::NROW) {
      const int nv = S - qbase < BQA ? S - qbase : BQA;
      const void* src = wave == 0   ? (const void*)(a.lse2 + ((int64_t)b * Hq + h) * S + qbase)
                        : wave == 1 ? (const void*)(a.delta + ((int64_t)b * Hq + h) * S + qbase)
                        : wave == 2 ? (const void*)(a.rows + (int64_t)b * S + qbase)
                        : wave == 3 ? (const void*)(a.rows + (int64_t)(B + b) * S + qbase)
                                    : (const void*)(hulls + qbase / 32);
      const int n = wave < 4 ? nv : (nv > 32 ? 2 : 1) * (int)(sizeof(QueryHull) / 4);
      lds_dma4_opaque(src, (uint32_t)(n * 4), smem + SM::ROW_OFF + (buf * SM::NROW + wave) * 256,
                      (uint32_t)(lane * 4));
    }
  };

  int j = 0, qbase = 0;                            // of the current pair
  if (n_iter > 0) {
    pair_of(0, j, qbase);
    stage(j, qbase, 0);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) loaded_here(kf[kk]);

  // two pairs per trip, so that the buffer index is a constant
  auto iteration = [&](int it, auto CUR_) {
    const int cur = CUR_;   // a constant in the unrolled main path
    int jn = j, qn = qbase;
    // that buffer was last read before the previous barrier
    if (it + 1 < n_iter) {
      pair_of(it + 1, jn, qn);
      stage(jn, qn, cur ^ 1);
    }
    const int h = kvh * G + j;
    const char* qs = smem + SM::Q_OFF + cur * SM::TQ;
    const char* dos = smem + SM::DO_OFF + cur * SM::TQ;
    const char* rowp = smem + SM::ROW_OFF + cur * SM::NROW * 256;
    const float* lse_s = reinterpret_cast<const float*>(rowp);
    const float* del_s = reinterpret_cast<const float*>(rowp + 256);
    const int* lo_s = reinterpret_cast<const int*>(rowp + 512);
    const int* hi_s = reinterpret_cast<const int*>(rowp + 768);
    const float slope = BIAS ? a.mod.slopes[h] * kModLog2e / sc.c : 0.f;   // in units of the stored scores

    auto half = [&](int ih) {
      const int hq = KSPLIT > 1 ? kpart : ih;
      const int qh = qbase + hq * 32;              // 32-query half hq of the block
      const int4 hv = *reinterpret_cast<const int4*>(rowp + 1024 + hq * 16);
      const int hlo = __builtin_amdgcn_readfirstlane(hv.x);
      const int hhi = __builtin_amdgcn_readfirstlane(hv.y);
      const int all_lo = __builtin_amdgcn_readfirstlane(hv.z);
      const int all_hi = __builtin_amdgcn_readfirstlane(hv.w);
      if (qh < S && hlo < kw0 + 32 && hhi > kw0) { // wave-uniform
        f32x16 sacc1[1], pacc;
        f32x16& sacc = sacc1[0];
        const float d0 = (float)(qh + 4 * g - mykey);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          sacc[r] = 0.f;
          pacc[r] = 0.f;
        }
        // queries all from, or all up to, the wave's keys
        if constexpr (BIAS && !CAP) bias_init(sacc1, slope, d0, qh >= kw0 + 31 ? 1 : qh + 31 <= kw0 ? -1 : 0);
        // fragments of step kk+1 are read before the MFMAs of step kk; the Q
        // and dO reads are a lane register plus a constant, the V read's address
        // is added right before it (kept there: holding eight V addresses
        // through the loop does not fit the register budget)
        auto rdq = [&](int kk) {
          return as_half8(*reinterpret_cast<const u32x4*>(smem + SM::Q_OFF + cur * SM::TQ + hq * 32 * RT::ROWB +
                                                          rlane[kk]));
        };
        auto rdo = [&](int kk) {
          return as_half8(*reinterpret_cast<const u32x4*>(smem + SM::DO_OFF + cur * SM::TQ + hq * 32 * RT::ROWB +
                                                          rlane[kk]));
        };
        auto rdv = [&](int kk) {
          uint32_t ad;
          asm volatile("v_add_u32 %0, %1, %2" : "=v"(ad) : "v"(rlane[kk]), "s"(vrow0));
          return as_half8(*reinterpret_cast<const u32x4*>(smem + ad));
        };
        char* const dsb = reinterpret_cast<char*>(a.ds) +
                          (((int64_t)lbkv * G + j) * nblk + ds_block(qh >> 5, kw0 >> 5, n32, causal)) * kDsBlockBytes;
        uint8_t* const live = a.live + ((int64_t)b * Hq + h) * nblk + ds_block(qh >> 5, kw0 >> 5, n32, causal);
        const bool full = kw0 >= all_lo && kw0 + 32 <= all_hi;     // wave-uniform
        half8 fd, fv;
        if constexpr (BIAS) {
          // the scores first, to see whether the block has any weight (kNoneBwd)
          half8 fq = rdq(0);
          __builtin_amdgcn_s_setprio(1);
#pragma unroll
          for (int kk = 0; kk < KK; ++kk) {
            half8 nq = fq;
            if (kk + 1 < KK) nq = rdq(kk + 1);
            sacc = mfma32(fq, kf[kk], sacc);
            fq = nq;
          }
          __builtin_amdgcn_s_setprio(0);
          float mx = -INFINITY;
#pragma unroll
          for (int rq = 0; rq < 4; ++rq) {
            const float4 l4 = *reinterpret_cast<const float4*>(lse_s + hq * 32 + 8 * rq + 4 * g);
            const float lv[4] = {l4.x, l4.y, l4.z, l4.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float t = sc.t(sacc[4 * rq + e]);
              if constexpr (CAP) t = fmaf(-slope, fabsf(d0 + (float)(8 * rq + e)), t);
              mx = fmaxf(mx, fmaf(t, sc.c, -lv[e]));
            }
          }
          const bool none = full && __builtin_amdgcn_ballot_w64(!(mx < -kNoneBwd)) == 0 && all_finite(sacc1);
          if (none) {
            if (lane == 0) *live = kZeroBlock;     // not 0: other shares of the tile list the pair by it
            return;
          }
          fd = rdo(0);
          fv = rdv(0);
          __builtin_amdgcn_s_setprio(1);
#pragma unroll
          for (int kk = 0; kk < KK; ++kk) {
            half8 nd = fd, nv = fv;
            if (kk + 1 < KK) {
              nd = rdo(kk + 1);
              nv = rdv(kk + 1);
            }
            pacc = mfma32(fd, fv, pacc);
            fd = nd;
            fv = nv;
          }
        } else {
          half8 fq = rdq(0);
          fd = rdo(0);
          fv = rdv(0);
          __builtin_amdgcn_s_setprio(1);
#pragma unroll
          for (int kk = 0; kk < KK; ++kk) {
            half8 nq = fq, nd = fd, nv = fv;
            if (kk + 1 < KK) {
              nq = rdq(kk + 1);
              nd = rdo(kk + 1);
              nv = rdv(kk + 1);
            }
            sacc = mfma32(fq, kf[kk], sacc);
            pacc = mfma32(fd, fv, pacc);
            if (kk + 1 < KK) {
              __builtin_amdgcn_sched_group_barrier(0x100, 3, 0);   // the three reads
              __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);   // then the two MFMAs
            }
            fq = nq;
            fd = nd;
            fv = nv;
          }
        }
        __builtin_amdgcn_s_setprio(0);
        // P = exp2(c t - LSE2), dS = P (dP - D) (1 - tanh^2)
        float p[16], ds[16];
#pragma unroll
        for (int rq = 0; rq < 4; ++rq) {
          const int ql0 = hq * 32 + 8 * rq + 4 * g;
          const float4 l4 = *reinterpret_cast<const float4*>(lse_s + ql0);
          const float4 d4 = *reinterpret_cast<const float4*>(del_s + ql0);
          const float lv[4] = {l4.x, l4.y, l4.z, l4.w};
          const float dv[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = 4 * rq + e;
            float t = sc.t(sacc[r]);
            ds[r] = pacc[r] - dv[e];
            if constexpr (CAP) {
              const float u4 = -4.f * t;               // 1 - tanh^2 = 4 u (1 - u), u = -t
              ds[r] *= fmaf(u4, t, u4);
              if constexpr (BIAS) t = fmaf(-slope, fabsf(d0 + (float)(8 * rq + e)), t);
            }
            p[r] = fast_exp2(fmaf(t, sc.c, -lv[e]));
          }
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) ds[r] *= p[r];
        if (!full) {                               // some query sees them in part
#pragma unroll
          for (int rq = 0; rq < 4; ++rq) {
            const int ql0 = hq * 32 + 8 * rq + 4 * g;
            const int4 l4 = *reinterpret_cast<const int4*>(lo_s + ql0);
            const int4 h4 = *reinterpret_cast<const int4*>(hi_s + ql0);
            const int lv[4] = {l4.x, l4.y, l4.z, l4.w};
            const int hw[4] = {h4.x, h4.y, h4.z, h4.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const bool see = (mykey >= lv[e]) & (mykey < hw[e]);
              p[4 * rq + e] = see ? p[4 * rq + e] : 0.f;
              ds[4 * rq + e] = see ? ds[4 * rq + e] : 0.f;
            }
          }
        }
        half8 pp[2], pds[2];
#pragma unroll
        for (int kc = 0; kc < 2; ++kc) {
          pp[kc] = pack8(p[8 * kc], p[8 * kc + 1], p[8 * kc + 2], p[8 * kc + 3], p[8 * kc + 4],
                         p[8 * kc + 5], p[8 * kc + 6], p[8 * kc + 7]);
          pds[kc] = pack8(ds[8 * kc], ds[8 * kc + 1], ds[8 * kc + 2], ds[8 * kc + 3],
                          ds[8 * kc + 4], ds[8 * kc + 5], ds[8 * kc + 6], ds[8 * kc + 7]);
        }
        // dS block for the dQ pass, as held here (lane-major, 32 bytes per
        // lane); written once, read once: non-temporal
        {
          char* dst = dsb + lane * 32;
          __builtin_nontemporal_store(as_u32x4(pds[0]), reinterpret_cast<u32x4*>(dst));
          __builtin_nontemporal_store(as_u32x4(pds[1]), reinterpret_cast<u32x4*>(dst + 16));
        }
        __builtin_amdgcn_s_setprio(1);
        //   dV^T += dO^T P,  dK^T += Q^T dS
        // steps (kc, db): the transposed dO and Q fragments of step s + 1 are
        // read before step s's two MFMAs, into the other of two register sets
        constexpr int NST = 2 * DB;
        half8 tdo[2], tq[2];
        auto rd_tr = [&](int st_, half8& x, half8& y) {
          const int kc = st_ / DB, db = st_ % DB;
          x = RT::template tr_frag<true>(dos, hq * 32 + kc * 16, db * 32, lane);
          y = RT::template tr_frag<true>(qs, hq * 32 + kc * 16, db * 32, lane);
        };
        rd_tr(0, tdo[0], tq[0]);
#pragma unroll
        for (int st_ = 0; st_ < NST; ++st_) {
          const int kc = st_ / DB, db = st_ % DB;
          if (st_ + 1 < NST) rd_tr(st_ + 1, tdo[(st_ + 1) & 1], tq[(st_ + 1) & 1]);
          dvacc[db] = mfma32(tdo[st_ & 1], pp[kc], dvacc[db]);
          dkacc[db] = mfma32(tq[st_ & 1], pds[kc], dkacc[db]);
          // the groups count from the top of the block: the first read group
          // holds steps 0 and 1 (two transposed reads per fragment)
          if (st_ + 1 < NST) {
            if (st_ == 0)
              __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
            else
              __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
          }
        }
        __builtin_amdgcn_s_setprio(0);
      }
    };
    if constexpr (KSPLIT == 1) {
#pragma unroll
      for (int ih = 0; ih < BQA / 32; ++ih) half(ih);
    } else {
      half(0);
    }
    j = jn;
    qbase = qn;
    // next block resident for every wave; nobody reads this buffer any more
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  };
  if constexpr (KSPLIT == 1) {
    for (int it = 0; it < n_iter; it += 2) {
      iteration(it, std::integral_constant<int, 0>{});
      if (it + 1 < n_iter) iteration(it + 1, std::integral_constant<int, 1>{});
    }
  } else {
    for (int it = 0; it < n_iter; ++it) iteration(it, it & 1);
  }

  if constexpr (KSPLIT > 1) {
    // all of LDS is free after the loop's last barrier: the second wave of
    // each pair passes its dK, dV accumulators through it (lane-major float4,
    // conflict-free) to the first, which adds them
    float4* red = reinterpret_cast<float4*>(smem);
    auto at = [&](int which, int db, int rq) { return (((kg * 2 + which) * DB + db) * 4 + rq) * 64 + lane; };
    if (kpart == 1) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int rq = 0; rq < 4; ++rq) {
          red[at(0, db, rq)] = make_float4(dkacc[db][4 * rq], dkacc[db][4 * rq + 1], dkacc[db][4 * rq + 2],
                                           dkacc[db][4 * rq + 3]);
          red[at(1, db, rq)] = make_float4(dvacc[db][4 * rq], dvacc[db][4 * rq + 1], dvacc[db][4 * rq + 2],
                                           dvacc[db][4 * rq + 3]);
        }
    }
    __syncthreads();
    if (kpart != 0) return;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int rq = 0; rq < 4; ++rq) {
        const float4 k = red[at(0, db, rq)];
        const float4 v = red[at(1, db, rq)];
        const float kv[4] = {k.x, k.y, k.z, k.w}, vv[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          dkacc[db][4 * rq + e] += kv[e];
          dvacc[db][4 * rq + e] += vv[e];
        }
      }
  }

  if (!(all_finite(dkacc) & all_finite(dvacc))) {  // a non-finite Q or dO somewhere in the tiles
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        dkacc[db][r] = 0.f;
        dvacc[db][r] = 0.f;
      }
    const int64_t krow = mykey < S ? mykey : S - 1;
    half8 vf[KK];
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) vf[kk] = as_half8(ld16(Vp + krow * a.kv_stride + kk * 16 + g * 8));
#pragma nounroll
    for (int it = 0; it < n_iter; ++it) {
      int jh, qb;
      pair_of(it, jh, qb);
      const int h = kvh * G + jh;
      const float slope = BIAS ? a.mod.slopes[h] * kModLog2e / sc.c : 0.f;
#pragma nounroll
      for (int q = qb; q < min(qb + BQA, S); ++q) {
        const int64_t row = (int64_t)b * S + q, ri = ((int64_t)b * Hq + h) * S + q;
        const lt_half* qp = a.Q + row * a.q_stride + (int64_t)h * D;
        const lt_half* gp = a.dO + row * a.o_stride + (int64_t)h * D;
        float s = half_dot(kf, qp + 8 * g), dp = half_dot(vf, gp + 8 * g);
        s += __shfl_xor(s, 32);
        dp += __shfl_xor(dp, 32);
        float t = sc.t(s), w = dp - a.delta[ri];
        if constexpr (CAP) w *= -4.f * t * (1.f + t);
        if constexpr (BIAS) t = fmaf(-slope, fabsf((float)(q - mykey)), t);
        const float p = fast_exp2(fmaf(t, sc.c, -a.lse2[ri]));
        const bool see = (mykey >= a.rows[(int64_t)b * S + q]) & (mykey < a.rows[(int64_t)(B + b) * S + q]);
        add_row(dvacc, see, p, gp, g);
        add_row(dkacc, see, p * w, qp, g);
      }
    }
  }

  // ---- write dK = scale * acc, dV (or this share's FP32 partial sums) ----
  if (mykey >= S) return;
  if (nsh > 1) {
    float* pk = a.part + (((int64_t)lbkv * nsh + sp) * S + mykey) * D;
    float* pv = pk + (int64_t)nb * nsh * S * D;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int rq = 0; rq < 4; ++rq) {
        const int d = db * 32 + 8 * rq + 4 * g;
        *reinterpret_cast<float4*>(pk + d) = make_float4(dkacc[db][4 * rq], dkacc[db][4 * rq + 1],
                                                         dkacc[db][4 * rq + 2], dkacc[db][4 * rq + 3]);
        *reinterpret_cast<float4*>(pv + d) = make_float4(dvacc[db][4 * rq], dvacc[db][4 * rq + 1],
                                                         dvacc[db][4 * rq + 2], dvacc[db][4 * rq + 3]);
      }
  } else {
    lt_half* dkp = a.dK + ((int64_t)b * S + mykey) * a.dkv_stride + (int64_t)kvh * D;
    lt_half* dvp = a.dV + ((int64_t)b * S + mykey) * a.dkv_stride + (int64_t)kvh * D;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int rq = 0; rq < 4; ++rq) {
        half4 k4, v4;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          k4[e] = (_Float16)(dkacc[db][4 * rq + e] * scale);
          v4[e] = (_Float16)dvacc[db][4 * rq + e];
        }
        *reinterpret_cast<half4*>(dkp + db * 32 + 8 * rq + 4 * g) = k4;
        *reinterpret_cast<half4*>(dvp + db * 32 + 8 * rq + 4 * g) = v4;
      }
  }
}

// dK = scale * sum of the shares' partials, dV = sum, in share order.  HBM-bound: two
// shares of 8192 x 8 keys 26 us (4.5 TB/s).
template <int D>
__global__ void __launch_bounds__(256)
attn_mod_sum_kernel(const AttnModBwdArgs a, int bkv0, int nb) {
  constexpr int CPR = D / 8;                       // 8-element chunks per row
  const int S = a.sh.S, Hkv = a.sh.Hkv, nsh = a.plan.nsplit;
  const int64_t gid = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (gid >= (int64_t)nb * S * CPR) return;
  const int d0 = (int)(gid % CPR) * 8;
  const int key = (int)((gid / CPR) % S);
  const int lbkv = (int)(gid / ((int64_t)CPR * S));
  const int b = (bkv0 + lbkv) / Hkv, kvh = (bkv0 + lbkv) % Hkv;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const float* src = a.part + (((int64_t)(which * nb + lbkv) * nsh) * S + key) * D + d0;
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int t = 0; t < nsh; ++t) {
      const float4 x = *reinterpret_cast<const float4*>(src + (int64_t)t * S * D);
      const float4 y = *reinterpret_cast<const float4*>(src + (int64_t)t * S * D + 4);
      acc[0] += x.x; acc[1] += x.y; acc[2] += x.z; acc[3] += x.w;
      acc[4] += y.x; acc[5] += y.y; acc[6] += y.z; acc[7] += y.w;
    }
    const float f = which == 0 ? a.sh.scale : 1.f;
    const half8 o = pack8(acc[0] * f, acc[1] * f, acc[2] * f, acc[3] * f, acc[4] * f, acc[5] * f, acc[6] * f,
                          acc[7] * f);
    st16((which == 0 ? a.dK : a.dV) + ((int64_t)b * S + key) * a.dkv_stride + (int64_t)kvh * D + d0, as_u32x4(o));
  }
}

// ------------------------------------------------------------ 3: dQ from dS
constexpr int BKQ = 64;         // keys per slice (two 32-key groups)

// NWQ waves per workgroup, one 32-query group each; two slices in flight while
// one is used (three for the smaller workgroups).  HBM-bound, by the dS blocks: 8192
// tokens of 64:8 heads in six documents read 1.7 GB in 402 us (4.3 TB/s), 2 D flop a pair.
template <int D, int NWQ>
struct DqSmem {
  using RT = RowTile<D, NWQ>;
  static constexpr int NS = NWQ == 8 ? 3 : 4;
  static constexpr int KT = BKQ * RT::ROWB;          // K slice [64][D]
  static constexpr int DSW = 2 * kDsBlockBytes;      // one wave's two dS blocks of a slice
  static constexpr int STAGE = KT + NWQ * DSW;
  static constexpr int BYTES = NS * STAGE;
  // direct loads per wave and stage: K rows, then always four 1 KiB dS loads
  // (of blocks that the mask drops a zero-length buffer), so that the count
  // behind each vmcnt wait is fixed
  static constexpr int LOADS = KT / 1024 / NWQ + 4;
};

// B operand dS^T of dQ^T = K^T dS^T from one dS block in LDS (lane-major,
// 32 bytes per lane of the dK/dV pass): lane L gets stored query position
// L % 32 at keys kb + 8 (j / 4) + 4 (L / 32) + j % 4, j = 0..7 (the key order of
// RowTile::tr_frag<true>).
__device__ __forceinline__ half8 ds_tr_frag(const char* blk, int kb, int lane) {
  v4s part[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int k = kb + 8 * h + 4 * (lane >> 5) + ((lane & 15) >> 2);
    part[h] = lds_read_tr16(blk + (k + 32 * ((lane >> 4) & 1)) * 32 + 8 * (lane & 3));
  }
  return as_half8(pack_v4s_pair(part[0], part[1]));
}

template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt field");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// MARKS (with a distance bias): only the blocks that their marks call live are read, and
// only slices that some wave of the workgroup has one in.
template <int D, int NWQ, bool MARKS>
__global__ void __launch_bounds__(NWQ * 64, 1)
attn_mod_dq_kernel(const AttnModBwdArgs a, int bkv0, int nb) {
  using SM = DqSmem<D, NWQ>;
  using RT = RowTile<D, NWQ>;
  constexpr int BQQ = NWQ * 32;                    // queries per workgroup
  constexpr int NSQ = SM::NS;
  constexpr int DB = D / 32;
  static_assert(SM::BYTES <= 160 * 1024, "stages fit in LDS");
  __shared__ __attribute__((aligned(1024))) char smem[SM::BYTES];

  const int S = a.sh.S, Hq = a.sh.Hq, Hkv = a.sh.Hkv, causal = a.sh.causal;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n32 = (S + 31) / 32;
  const int n_qt = (S + BQQ - 1) / BQQ;
  const int G = Hq / Hkv;
  const int slot = blockIdx.x / (nb * G);
  const int qt = n_qt - 1 - slot;                  // later queries mostly see more keys: longest first
  // the query heads of one kv head on one XCD where the chunk is a multiple of 8
  const int lbkv = (blockIdx.x % (nb * G)) % nb;
  const int j = (blockIdx.x % (nb * G)) / nb;
  const int b = (bkv0 + lbkv) / Hkv;
  const int kvh = (bkv0 + lbkv) % Hkv;
  const int h = kvh * G + j;
  const int qg = qt * NWQ + wave;                  // this wave's 32-query group
  const QueryHull* hulls = a.hulls + (int64_t)b * n32;
  // key groups that some query of the group, of the workgroup, sees
  int kg0 = 0, kg_end = 0, wg_lo = 0x7fffffff, wg_hi = 0;
#pragma unroll
  for (int w = 0; w < NWQ; ++w) {
    const int q = qt * NWQ + w;
    if (q < n32) {
      const int lo = hulls[q].lo, hi = hulls[q].hi;
      wg_lo = min(wg_lo, lo);
      wg_hi = max(wg_hi, hi);
      if (w == wave && lo < hi) {
        kg0 = lo >> 5;
        kg_end = (hi + 31) >> 5;
      }
    }
  }
  kg0 = __builtin_amdgcn_readfirstlane(kg0);
  kg_end = __builtin_amdgcn_readfirstlane(kg_end);
  const int ks0 = __builtin_amdgcn_readfirstlane(wg_lo < wg_hi ? wg_lo / BKQ : 0);
  const int ks1 = __builtin_amdgcn_readfirstlane(wg_lo < wg_hi ? (wg_hi + BKQ - 1) / BKQ : 0);

  const lt_half* Kp = a.K + (int64_t)b * S * a.kv_stride + (int64_t)kvh * D;
  const int64_t nblk = ds_blocks(n32, causal);
  // block (qg, 0); block (qg, kg) follows at kg * 2 KiB
  const char* dsq = reinterpret_cast<const char*>(a.ds) +
                    (((int64_t)lbkv * G + j) * nblk + ds_block(qg < n32 ? qg : 0, 0, n32, causal)) * kDsBlockBytes;

  f32x16 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[db][r] = 0.f;

  // live blocks of 64 key groups (32 slices) from 64 win: this wave's, any wave's
  int win = -1;
  uint64_t mine_w = 0, any_w = 0;
  auto load_window = [&](int w) {
    win = w;
    const int kg = w * 64 + lane;
    bool mine = false, any = false;
#pragma unroll
    for (int u = 0; u < NWQ; ++u) {
      const int q = qt * NWQ + u;
      if (q >= n32) continue;
      const QueryHull hu = hulls[q];
      const bool on = hu.lo < hu.hi && kg >= hu.lo >> 5 && kg < (hu.hi + 31) >> 5 &&
                      a.live[((int64_t)b * Hq + h) * nblk + ds_block(q, kg, n32, causal)] == kLiveBlock;
      any |= on;
      if (u == wave) mine = on;
    }
    mine_w = __builtin_amdgcn_ballot_w64(mine);
    any_w = __builtin_amdgcn_ballot_w64(any);
  };
  // the next slice from ks on to go through (ks1: none), and this wave's two blocks of it
  auto next_slice = [&](int ks, uint32_t& own) {
    if constexpr (!MARKS) {
      own = (2 * ks >= kg0 && 2 * ks < kg_end ? 1 : 0) | (2 * ks + 1 >= kg0 && 2 * ks + 1 < kg_end ? 2 : 0);
      return ks;
    }
    for (; ks < ks1; ks = (win + 1) * 32) {
      if (ks >> 5 != win) load_window(ks >> 5);
      const uint64_t left = any_w >> (2 * (ks & 31));
      if (left) {
        ks += __builtin_ctzll(left) >> 1;
        own = (uint32_t)(mine_w >> (2 * (ks & 31))) & 3;
        return ks;
      }
    }
    return ks1;
  };

  // the staged-th slice (keys from ks * 64) -> stage staged % NSQ; K rows past S read
  // as zero.  owns: two bits a stage, which of the wave's blocks are there
  int staged = 0;
  uint32_t owns = 0, own = 0;
  int ks = ks1;
  auto advance = [&](int from) {
    ks = __builtin_amdgcn_readfirstlane(from < ks1 ? next_slice(from, own) : ks1);
    own = __builtin_amdgcn_readfirstlane(own);
  };
  advance(ks0);
  auto stage_next = [&] {
    if (ks >= ks1) return;
    const int slot = staged % NSQ;
    char* st = smem + slot * SM::STAGE;
    RT::template dma<BKQ>(st, Kp + (int64_t)ks * BKQ * a.kv_stride, a.kv_stride, S - ks * BKQ, wave, lane);
    char* mine = st + SM::KT + wave * SM::DSW;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const bool in = own >> c & 1;
      const char* src = dsq + (int64_t)(in ? 2 * ks + c : 0) * kDsBlockBytes;
      const uint32_t nrec = in ? kDsBlockBytes : 0u;
      lds_dma16_stream(src, nrec, mine + c * kDsBlockBytes, (uint32_t)(lane * 16));
      lds_dma16_stream(src, nrec, mine + c * kDsBlockBytes + 1024, (uint32_t)(1024 + lane * 16));
    }
    owns = __builtin_amdgcn_readfirstlane((owns & ~(3u << (2 * slot))) | own << (2 * slot));
    ++staged;
    advance(ks + 1);
  };

  // slices after the next one may stay in flight, up to NSQ - 2 of them
  auto wait_next = [&](int behind) {
    if (behind >= NSQ - 2) wait_vmcnt<(NSQ - 2) * SM::LOADS>();
    else if (NSQ > 3 && behind == 1) wait_vmcnt<SM::LOADS>();
    else wait_vmcnt<0>();
  };
#pragma unroll
  for (int i = 0; i < NSQ - 1; ++i) stage_next();
  wait_next(staged - 1);                           // slice 0 resident
  __syncthreads();
  for (int i = 0; i < staged; ++i) {
    // the stage of slice i + NSQ - 1 was last read before the previous barrier
    stage_next();
    const char* st = smem + (i % NSQ) * SM::STAGE;
    const char* mine = st + SM::KT + wave * SM::DSW;
    const uint32_t now = owns >> (2 * (i % NSQ));
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      if (now >> c & 1) {
#pragma unroll
        for (int kc = 0; kc < 2; ++kc) {
          //   dQ^T += K^T dS^T  (K^T read transposed, keys in accumulator order)
          const half8 bds = ds_tr_frag(mine + c * kDsBlockBytes, kc * 16, lane);
#pragma unroll
          for (int db = 0; db < DB; ++db)
            acc[db] = mfma32(RT::template tr_frag<true>(st, c * 32 + kc * 16, db * 32, lane), bds, acc[db]);
        }
      }
    }
    // the next slice resident for every wave (later slices' loads may still be
    // in flight); nobody reads this stage any more
    wait_next(staged - (i + 2));
    __syncthreads();
  }

  // ---- dQ = scale * acc -> FP16; lane L holds stored query position L % 32 ----
  if (qg < n32) {
    const int pos = lane & 31;
    const int q = qg * 32 + 8 * ((pos & 15) >> 2) + 4 * (pos >> 4) + (pos & 3);
    const int g = lane >> 5;
    if (!all_finite(acc)) {                        // a non-finite K somewhere in the tiles
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[db][r] = 0.f;
      int lo, hi;
      row_interval(a.mod, causal, b, S, q, lo, hi);
#pragma nounroll
      for (int k = kg0 * 32; k < min(kg_end * 32, S); ++k) {
        if (MARKS && a.live[((int64_t)b * Hq + h) * nblk + ds_block(qg, k >> 5, n32, causal)] != kLiveBlock) continue;
        const char* el = dsq + (int64_t)(k >> 5) * kDsBlockBytes + ((k & 31) + 32 * (pos >> 4)) * 32 + (pos & 15) * 2;
        add_row(acc, (k >= lo) & (k < hi), (float)*reinterpret_cast<const _Float16*>(el),
                Kp + (int64_t)k * a.kv_stride, g);
      }
    }
    if (q < S) {
      lt_half* qp = a.dQ + ((int64_t)b * S + q) * a.dq_stride + (int64_t)h * D;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int rq = 0; rq < 4; ++rq) {
          half4 o;
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] = (_Float16)(acc[db][4 * rq + e] * a.sh.scale);
          *reinterpret_cast<half4*>(qp + db * 32 + 8 * rq + 4 * g) = o;
        }
    }
  }
}

constexpr int64_t kDeltaSlots = 512;  // workgroup slots: two per CU
constexpr int kOnePassS = 512;        // longest sequence whose D is all formed from S and dP
constexpr int64_t kDqHalfWgs = 128;   // 256-query workgroups up to which they hold 128

template <int D, bool CAP, bool BIAS>
hipError_t launch_bwd(const AttnModBwdArgs& a, hipStream_t s) {
  const AttnShape& sh = a.sh;
  const unsigned n_rows = (unsigned)((int64_t)sh.B * ((sh.S + 255) / 256));
  const int64_t n_tile = (int64_t)((sh.S + kTile - 1) / kTile) * sh.B * sh.Hq;
  const int64_t n_tile64 = (int64_t)((sh.S + 63) / 64) * sh.B * sh.Hq;
  if (sh.S <= kOnePassS && n_tile <= kDeltaSlots) {
    hipLaunchKernelGGL((attn_mod_delta_kernel<D, 2, CAP, BIAS>), dim3((unsigned)n_tile64 + n_rows), dim3(NWD * 64), 0, s,
                       a, 1, (unsigned)n_tile64);
  } else {
    hipLaunchKernelGGL((attn_mod_rows_kernel<D, CAP>), dim3((unsigned)n_tile + n_rows), dim3(256), 0, s, a,
                       (unsigned)n_tile);
    hipError_t er = hipGetLastError();
    if (er != hipSuccess) return er;
    // 64-query tiles where 128-query ones would not fill the CUs twice
    if (n_tile > kDeltaSlots)
      hipLaunchKernelGGL((attn_mod_delta_kernel<D, 1, CAP, BIAS>), dim3((unsigned)n_tile), dim3(NWD * 64), 0, s, a, 0,
                         (unsigned)n_tile);
    else
      hipLaunchKernelGGL((attn_mod_delta_kernel<D, 2, CAP, BIAS>), dim3((unsigned)n_tile64), dim3(NWD * 64), 0, s, a,
                         0, (unsigned)n_tile64);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int pairs = sh.B * sh.Hkv, grp = sh.Hq / sh.Hkv;
  const int n_kt = (sh.S + a.plan.ktile - 1) / a.plan.ktile;
  for (int bkv0 = 0; bkv0 < pairs; bkv0 += a.plan.chunk) {
    const int nb = pairs - bkv0 < a.plan.chunk ? pairs - bkv0 : a.plan.chunk;
    const dim3 kgrid((unsigned)((int64_t)n_kt * a.plan.nsplit * nb));
    if (a.plan.ktile == BKV)
      hipLaunchKernelGGL((attn_mod_dkdv_kernel<D, 1, CAP, BIAS>), kgrid, dim3(NWA * 64), 0, s, a, bkv0, nb);
    else
      hipLaunchKernelGGL((attn_mod_dkdv_kernel<D, 2, CAP, BIAS>), kgrid, dim3(NWA * 64), 0, s, a, bkv0, nb);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (a.plan.nsplit > 1) {
      const int64_t chunks = (int64_t)nb * sh.S * (D / 8);
      hipLaunchKernelGGL((attn_mod_sum_kernel<D>), dim3((unsigned)((chunks + 255) / 256)), dim3(256), 0, s, a, bkv0,
                         nb);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    // longest query tiles first under a causal mask
    auto launch_dq = [&](auto W_) {
      constexpr int NWQ = decltype(W_)::value;
      const int n_qt = (sh.S + NWQ * 32 - 1) / (NWQ * 32);
      hipLaunchKernelGGL((attn_mod_dq_kernel<D, NWQ, BIAS>), dim3((unsigned)((int64_t)n_qt * nb * grp)), dim3(NWQ * 64), 0,
                         s, a, bkv0, nb);
    };
    if ((int64_t)((sh.S + 255) / 256) * nb * grp > kDqHalfWgs) launch_dq(std::integral_constant<int, 8>{});
    else launch_dq(std::integral_constant<int, 4>{});
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  return e;
}

template <int D>
hipError_t launch_bwd_d(const AttnModBwdArgs& a, hipStream_t s) {
  if (a.mod.cap > 0.f) return a.mod.slopes ? launch_bwd<D, true, true>(a, s) : launch_bwd<D, true, false>(a, s);
  return a.mod.slopes ? launch_bwd<D, false, true>(a, s) : launch_bwd<D, false, false>(a, s);
}

}  // namespace

hipError_t attn_mod_bwd_launch(const AttnModBwdArgs& a, hipStream_t s) {
  return a.sh.D == 128 ? launch_bwd_d<128>(a, s) : launch_bwd_d<64>(a, s);
}

}  // namespace lt
