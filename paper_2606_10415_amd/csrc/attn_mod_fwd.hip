// Attention forward with modified scores, gfx950: O and the row log-sum-exp of
//
//     z_ij = cap tanh(scale q_i.k_j / cap) - slope_h |i - j|   (each part optional)
//
// over the keys lo_i <= j < hi_i that query i sees (j <= i too when causal).  A
// query that sees no key gets O = 0 and LSE = -inf.
//
//   * one workgroup = 4 waves = one (batch, query head, 128-query tile), or 64
//     queries when 128-query tiles would fill at most one round of the CUs' two
//     workgroup slots, and in a last round that is at most half full: then the two waves
//     of a query group take one 32-key block of each slice each and merge their
//     states through LDS;
//   * S^T = K Q^T with 32x32x16 MFMA, so that a lane owns one query and its
//     interval sits in two registers.  The workgroup walks the 64-key slices of
//     the hull of its queries' intervals, last slice first (under a causal mask the
//     nearest keys, which a distance bias makes the heaviest), a wave skips the slices
//     that none of its 32 queries sees, compares key against interval only in
//     slices that some of them see in part, and with a distance bias leaves a slice
//     after its scores where none has weight;
//   * K and V slices go HBM -> LDS by direct loads, double-buffered; O^T += V^T P^T
//     takes V^T by the LDS transpose read in the accumulator's key order, so that
//     P goes from the score registers, rounded to FP16 (the rounding of every
//     FP16 matrix operand), straight into the product;
//   * one pass: running maximum and sum in FP32, the maximum raised only when a
//     row exceeds it by more than 2^8 in probability.
//
// Bound by the matrix and vector units in turn: two waves a SIMD, whose products and
// softmax overlap poorly.  4 D flop a visible pair: 8192 tokens of 64:8 heads in six
// documents 528 us (827 TFLOP/s; a large matrix product reaches 1300 here), 4096 tokens of 32
// heads causal 156 us (880), with a cap 199 (690: an exp2 and a reciprocal more a score),
// 40 heads with ALiBi slopes 157 (steep heads leave most slices after their scores).
// One wave a SIMD with the next slice's scores placed under this one's softmax needs more
// registers than there are: 396 spilled, 567 TFLOP/s.

#include <type_traits>

#include "attn_mod.hpp"

namespace lt {
namespace {

constexpr int NW = 4;        // waves per workgroup, 32 queries each
constexpr int BKV = 64;      // keys per LDS slice
constexpr int BQ = NW * 32;  // queries per workgroup
constexpr float kLazy = 8.f; // log2 of the largest probability before a rescale
constexpr int64_t kFwdSlots = 512;      // workgroup slots: two per CU

template <int D>
struct FwdSmem {
  using RT = RowTile<D, NW>;
  static constexpr int TILE = BKV * RT::ROWB;     // one K or V slice
  static constexpr int STAGE = 2 * TILE;          // K then V
};

// Query tile qt (of 128 queries, or 64 with QSPLIT = 2) of (batch, head) bh.
template <int D, int QSPLIT, bool CAP, bool BIAS>
__device__ __forceinline__ void
fwd_tile(const lt_half* __restrict__ Q, const lt_half* __restrict__ K, const lt_half* __restrict__ V,
         int64_t q_stride, int64_t kv_stride, lt_half* __restrict__ O, int64_t o_stride, float* __restrict__ LSE,
         const ScoreMod& mod, int B, int S, int Hq, int Hkv, float scale, int causal, int qt, unsigned bh,
         char* smem, int (*hull_s)[NW]) {
  using SM = FwdSmem<D>;
  using RT = RowTile<D, NW>;
  constexpr int KB = BKV / 32;     // 32-key blocks per slice
  constexpr int DB = D / 32;       // 32-feature blocks
  constexpr int KK = D / 16;       // MFMA steps over the head dim
  constexpr int NQG = NW / QSPLIT;                 // query groups of 32
  constexpr int BQW = NQG * 32;                    // queries per workgroup
  constexpr int KBW = KB / QSPLIT;                 // 32-key blocks per slice and wave
  static_assert(QSPLIT == 1 || NQG * DB * 4 * 64 * 16 + NQG * 64 * 8 <= 2 * SM::STAGE, "merge fits in LDS");

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);   // uniform: scalar addressing
  const int lrow = lane & 31;
  const int g = lane >> 5;
  const int qg = wave % NQG;                       // query group
  const int kpart = wave / NQG;                    // which block of each slice (QSPLIT = 2)

  int b, h;
  query_head(bh, B, Hq, Hkv, b, h);
  const int kvh = h / (Hq / Hkv);
  const int q0 = qt * BQW;
  const int qw0 = q0 + qg * 32;
  const int myq = qw0 + lrow;                      // query owned by this lane

  const lt_half* Kp = K + (int64_t)b * S * kv_stride + (int64_t)kvh * D;
  const lt_half* Vp = V + (int64_t)b * S * kv_stride + (int64_t)kvh * D;
  const Score<CAP> sc(mod, scale);
  const float c = sc.c;
  const float slope = BIAS ? mod.slopes[h] * kModLog2e / c : 0.f;   // in units of the stored scores
  const float lazy_raw = kLazy / c;

  // Q fragments (B operand of S^T = K Q^T): column = this lane's query,
  // reduction indices kk*16 + 8g + 0..7.
  half8 qf[KK];
  {
    const lt_half* qp = Q + ((int64_t)b * S + myq) * q_stride + (int64_t)h * D + g * 8;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
      qf[kk] = myq < S ? as_half8(ld16(qp + kk * 16)) : as_half8(u32x4{0, 0, 0, 0});
  }

  int lo, hi;                                      // this query's keys
  row_interval(mod, causal, b, S, myq, lo, hi);
  const QueryHull wh = query_hull(lo, hi, myq < S);
  if (lane == 0) {
    hull_s[0][wave] = wh.lo;
    hull_s[1][wave] = wh.hi;
  }
  __syncthreads();
  int wg_lo = 0x7fffffff, wg_hi = 0;
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    wg_lo = min(wg_lo, hull_s[0][w]);
    wg_hi = max(wg_hi, hull_s[1][w]);
  }
  const int kt0 = __builtin_amdgcn_readfirstlane(wg_lo < wg_hi ? wg_lo / BKV : 0);
  const int kt1 = __builtin_amdgcn_readfirstlane(wg_lo < wg_hi ? (wg_hi + BKV - 1) / BKV : 0);

  // lane part of the K row-fragment address of step kk (rows rb + lane % 32,
  // rb a multiple of 16, so the swizzle depends on the lane only)
  uint32_t rlane[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) rlane[kk] = (uint32_t)RT::addr(lane & 31, kk * 2 + (lane >> 5));

  f32x16 oacc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[db][r] = 0.f;
  float m_run = -INFINITY;   // running max (stored scores) used as the exponent offset
  float lsum = 0.f;          // this lane's share of the row sum

  // K, V rows past S read as zero (no query's interval reaches them)
  auto stage_load = [&](int kt, int buf) {
    char* st = smem + buf * SM::STAGE;
    const int key0 = kt * BKV;
    RT::template dma<BKV>(st, Kp + (int64_t)key0 * kv_stride, kv_stride, S - key0, wave, lane);
    RT::template dma<BKV>(st + SM::TILE, Vp + (int64_t)key0 * kv_stride, kv_stride, S - key0, wave, lane);
  };
  if (kt0 < kt1) stage_load(kt1 - 1, 0);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();

  // two slices per trip, so that the stage index is a constant and every LDS
  // fragment address is a per-lane register plus the instruction's offset
  auto slice = [&](int kt, auto CUR_) {
    constexpr int cur = decltype(CUR_)::value;
    const char* st = smem + cur * SM::STAGE;
    // that stage was last read before the previous barrier
    if (kt > kt0) stage_load(kt - 1, cur ^ 1);

    const int kb0 = QSPLIT > 1 ? kpart * 32 : 0;
    const int key0 = kt * BKV + kb0;               // this wave's keys: KBW * 32 from here
    if (key0 < wh.hi && key0 + KBW * 32 > wh.lo) {
      // ---- S^T = K Q^T ----
      f32x16 sacc[KBW];
      const float d0 = (float)(key0 + 4 * g - myq);
      // keys all up to, or all from, the wave's queries
      const int side = key0 >= qw0 + 31 ? 1 : key0 + KBW * 32 - 1 <= qw0 ? -1 : 0;
      if constexpr (BIAS && !CAP) {
        bias_init(sacc, slope, d0, side);
      } else {
#pragma unroll
        for (int kb = 0; kb < KBW; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) sacc[kb][r] = 0.f;
      }
      // K fragments of step kk+1 are read before the MFMAs of step kk, into
      // the other of two register sets
      auto rdk = [&](int kb, int kk) {
        return as_half8(*reinterpret_cast<const u32x4*>(st + (kb0 + kb * 32) * RT::ROWB + rlane[kk]));
      };
      half8 kfr[2][KBW];
#pragma unroll
      for (int kb = 0; kb < KBW; ++kb) kfr[0][kb] = rdk(kb, 0);
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        if (kk + 1 < KK) {
#pragma unroll
          for (int kb = 0; kb < KBW; ++kb) kfr[(kk + 1) & 1][kb] = rdk(kb, kk + 1);
        }
#pragma unroll
        for (int kb = 0; kb < KBW; ++kb) sacc[kb] = mfma32(kfr[kk & 1][kb], qf[kk], sacc[kb]);
        // the scheduling groups count from the top of the block: the first
        // read group holds step 0's reads and step 1's
        if (kk + 1 < KK) {
          if (kk == 0)
            __builtin_amdgcn_sched_group_barrier(0x100, 2 * KBW, 0);
          else
            __builtin_amdgcn_sched_group_barrier(0x100, KBW, 0);
          __builtin_amdgcn_sched_group_barrier(0x008, KBW, 0);
        }
      }

      // ---- cap (and bias behind it) ----
      if constexpr (CAP) {
#pragma unroll
        for (int kb = 0; kb < KBW; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            sacc[kb][r] = sc.t(sacc[kb][r]);
            if constexpr (BIAS)
              sacc[kb][r] = fmaf(-slope, fabsf(d0 + (float)(kb * 32 + 8 * (r >> 2) + (r & 3))), sacc[kb][r]);
          }
      }

      // ---- mask, row max ----
      const bool partly = key0 < wh.all_lo || key0 + KBW * 32 > wh.all_hi;   // wave-uniform
      if (partly) {
#pragma unroll
        for (int kb = 0; kb < KBW; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int key = key0 + kb * 32 + 8 * (r >> 2) + 4 * g + (r & 3);
            sacc[kb][r] = ((key >= lo) & (key < hi)) ? sacc[kb][r] : -INFINITY;
          }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < KBW; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sacc[kb][r]);
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      // a slice of no weight ends here (kNoneFwd); the slices run from the last, so that a
      // causal row has its nearest keys, and its maximum, first
      const bool none = BIAS && !partly && __builtin_amdgcn_ballot_w64(!(mx < m_run - kNoneFwd / c)) == 0 &&
                        all_finite(sacc);

      // ---- raise the running max only past the lazy margin ----
      const bool raise = mx > m_run + lazy_raw;    // m_run = -inf until the query's first key
      if (__builtin_amdgcn_ballot_w64(raise)) {    // wave-uniform branch
        const float m_new = raise ? mx : m_run;
        const float alpha = raise ? fast_exp2((m_run - m_new) * c) : 1.f;   // 0 on the first raise
        m_run = m_new;
        lsum *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r) oacc[db][r] *= alpha;
      }

      // ---- P = exp2(z - m), row sum, FP16 P^T fragments ----
      // (a query without a key so far: every score is -inf, P = exp2(-inf) = 0)
      if (!none) {
        const float mc = m_run == -INFINITY ? 0.f : m_run * c;
        half8 pf[KBW][2];
#pragma unroll
        for (int kb = 0; kb < KBW; ++kb) {
          float p[16];
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            p[r] = fast_exp2(fmaf(sacc[kb][r], c, -mc));
            lsum += p[r];
          }
#pragma unroll
          for (int kc = 0; kc < 2; ++kc)
            pf[kb][kc] = pack8(p[8 * kc + 0], p[8 * kc + 1], p[8 * kc + 2], p[8 * kc + 3],
                               p[8 * kc + 4], p[8 * kc + 5], p[8 * kc + 6], p[8 * kc + 7]);
        }

        // ---- O^T += V^T P^T (V^T read transposed, keys in accumulator order) ----
        const char* vs = st + SM::TILE;
#pragma unroll
        for (int kb = 0; kb < KBW; ++kb)
#pragma unroll
          for (int kc = 0; kc < 2; ++kc)
#pragma unroll
            for (int db = 0; db < DB; ++db)
              oacc[db] = mfma32(RT::template tr_frag<true>(vs, kb0 + kb * 32 + kc * 16, db * 32, lane), pf[kb][kc],
                                oacc[db]);
      }
    }

    // next slice resident for every wave; nobody reads this stage any more
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  };
  for (int kt = kt1 - 1; kt >= kt0; kt -= 2) {
    slice(kt, std::integral_constant<int, 0>{});
    if (kt > kt0) slice(kt - 1, std::integral_constant<int, 1>{});
  }

  if constexpr (QSPLIT > 1) {
    // every stage is free after the loop's last barrier: the second wave of
    // each pair passes O (lane-major float4), its running max and row-sum
    // share to the first, which rescales both to the larger max and adds
    float4* red = reinterpret_cast<float4*>(smem);
    float2* ml = reinterpret_cast<float2*>(smem + NQG * DB * 4 * 64 * 16);
    if (kpart == 1) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int rq = 0; rq < 4; ++rq)
          red[((qg * DB + db) * 4 + rq) * 64 + lane] = make_float4(
              oacc[db][4 * rq], oacc[db][4 * rq + 1], oacc[db][4 * rq + 2], oacc[db][4 * rq + 3]);
      ml[qg * 64 + lane] = make_float2(m_run, lsum);
    }
    __syncthreads();
    if (kpart != 0) return;
    const float2 o2 = ml[qg * 64 + lane];
    const float m = fmaxf(m_run, o2.x);
    // a wave that saw no key of this query has m_run = -inf, a zero row sum and O
    const float a1 = m_run == -INFINITY ? 0.f : fast_exp2((m_run - m) * c);
    const float a2 = o2.x == -INFINITY ? 0.f : fast_exp2((o2.x - m) * c);
    m_run = m;
    lsum = lsum * a1 + o2.y * a2;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int rq = 0; rq < 4; ++rq) {
        const float4 v = red[((qg * DB + db) * 4 + rq) * 64 + lane];
        oacc[db][4 * rq] = oacc[db][4 * rq] * a1 + v.x * a2;
        oacc[db][4 * rq + 1] = oacc[db][4 * rq + 1] * a1 + v.y * a2;
        oacc[db][4 * rq + 2] = oacc[db][4 * rq + 2] * a1 + v.z * a2;
        oacc[db][4 * rq + 3] = oacc[db][4 * rq + 3] * a1 + v.w * a2;
      }
  }

  // ---- normalise and store O, LSE ----
  const float lt = lsum + __shfl_xor(lsum, 32);
  if (!all_finite(oacc)) {                         // a non-finite V somewhere in the tiles
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) oacc[db][r] = 0.f;
    const float mc = m_run == -INFINITY ? 0.f : m_run * c;
#pragma nounroll
    for (int j = wh.lo; j < wh.hi; ++j) {
      float s = half_dot(qf, Kp + (int64_t)j * kv_stride + 8 * g);
      s += __shfl_xor(s, 32);
      float t = sc.t(s);
      if constexpr (BIAS) t = fmaf(-slope, fabsf((float)(j - myq)), t);
      add_row(oacc, (j >= lo) & (j < hi), fast_exp2(fmaf(t, c, -mc)), Vp + (int64_t)j * kv_stride, g);
    }
  }
  if (myq < S) {
    const float inv = lo < hi ? 1.f / lt : 0.f;
    lt_half* op = O + ((int64_t)b * S + myq) * o_stride + (int64_t)h * D;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int rq = 0; rq < 4; ++rq) {
        half4 o;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = lo < hi ? (_Float16)(oacc[db][4 * rq + e] * inv) : (_Float16)0.f;
        *reinterpret_cast<half4*>(op + db * 32 + 8 * rq + 4 * g) = o;
      }
    if (g == 0)
      LSE[((int64_t)b * Hq + h) * S + myq] =
          lo < hi ? (m_run * c + sc.off) * kModLn2 + __logf(lt) : -INFINITY;
  }
}

// Workgroups 0 .. n_head - 1: 128 queries each, the last ones of every head first (later
// queries mostly see more keys: longest first); the others 64 each.
template <int D, bool HEAD, bool CAP, bool BIAS>
__global__ void __launch_bounds__(NW * 64, 2)
attn_mod_fwd_kernel(const lt_half* __restrict__ Q, const lt_half* __restrict__ K, const lt_half* __restrict__ V,
                    int64_t q_stride, int64_t kv_stride, lt_half* __restrict__ O, int64_t o_stride,
                    float* __restrict__ LSE, const ScoreMod mod, int B, int S, int Hq, int Hkv, float scale,
                    int causal, unsigned n_head) {
  __shared__ __attribute__((aligned(1024))) char smem[2 * FwdSmem<D>::STAGE];
  __shared__ int hull_s[2][NW];
  const unsigned heads = B * Hq, bh = blockIdx.x % heads;
  const int row = blockIdx.x / heads;
  if (HEAD && blockIdx.x < n_head)
    return fwd_tile<D, 1, CAP, BIAS>(Q, K, V, q_stride, kv_stride, O, o_stride, LSE, mod, B, S, Hq, Hkv, scale,
                                     causal, (S + BQ - 1) / BQ - 1 - row, bh, smem, hull_s);
  fwd_tile<D, 2, CAP, BIAS>(Q, K, V, q_stride, kv_stride, O, o_stride, LSE, mod, B, S, Hq, Hkv, scale, causal,
                            (int)(gridDim.x / heads) - 1 - row, bh, smem, hull_s);
}

template <int D, bool CAP, bool BIAS>
hipError_t launch_fwd(const AttnModFwdArgs& a, hipStream_t s) {
  const AttnShape& sh = a.sh;
  // 64-query workgroups where 128-query ones would fill at most one round of the
  // slots (short sequences), and for the rows of tiles of a last round that is at most half
  // full: 2048 tokens of 40 heads, 640 workgroups, window of 683 and cap: 53.5 us against 60.1, with
  // 64 queries throughout 65; 8 x 1024 tokens of 10 heads, full: 53.9 against 56.3; level or a
  // little better in 16 other shapes of 576 to 4096 workgroups
  const int64_t heads = (int64_t)sh.B * sh.Hq, rows = (sh.S + BQ - 1) / BQ, wgs = rows * heads;
  const int64_t last = (wgs % kFwdSlots + heads - 1) / heads;
  const int64_t head = wgs <= kFwdSlots ? 0 : last * heads <= kFwdSlots / 2 ? rows - last : rows;
  const int64_t tail = head == 0 ? (sh.S + BQ / 2 - 1) / (BQ / 2) : 2 * (rows - head);
  const dim3 grid((unsigned)((head + tail) * heads));
  if (head > 0)
    hipLaunchKernelGGL((attn_mod_fwd_kernel<D, true, CAP, BIAS>), grid, dim3(NW * 64), 0, s, a.Q, a.K, a.V, a.q_stride,
                       a.kv_stride, a.O, a.o_stride, a.LSE, a.mod, sh.B, sh.S, sh.Hq, sh.Hkv, sh.scale, sh.causal,
                       (unsigned)(head * heads));
  else
    hipLaunchKernelGGL((attn_mod_fwd_kernel<D, false, CAP, BIAS>), grid, dim3(NW * 64), 0, s, a.Q, a.K, a.V,
                       a.q_stride, a.kv_stride, a.O, a.o_stride, a.LSE, a.mod, sh.B, sh.S, sh.Hq, sh.Hkv, sh.scale,
                       sh.causal, 0u);
  return hipGetLastError();
}

template <int D>
hipError_t launch_fwd_d(const AttnModFwdArgs& a, hipStream_t s) {
  if (a.mod.cap > 0.f) return a.mod.slopes ? launch_fwd<D, true, true>(a, s) : launch_fwd<D, true, false>(a, s);
  return a.mod.slopes ? launch_fwd<D, false, true>(a, s) : launch_fwd<D, false, false>(a, s);
}

}  // namespace

hipError_t attn_mod_fwd_launch(const AttnModFwdArgs& a, hipStream_t s) {
  return a.sh.D == 128 ? launch_fwd_d<128>(a, s) : launch_fwd_d<64>(a, s);
}

}  // namespace lt
