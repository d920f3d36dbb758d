// Internal launcher interface of the packed-sequence operators (attention with
// modified scores, QK norm with rotation, embedding): packed_api.cpp checks
// the arguments, then calls these.
#pragma once

#include "kernels.hpp"

namespace lt {

// ---------------------------------------------------------------- attention with modified scores
// Which scores there are and what becomes of them.  Query i of batch row b
// sees the keys lo <= j < hi (row_interval in attn_mod.hpp).
struct ScoreMod {
  const int32_t* lo;      // [B, S] first visible key, or null: 0
  const int32_t* hi;      // [B, S] end of the visible keys, or null: S
  const float* slopes;    // [Hq] distance bias, or null: none
  float cap;              // tanh cap, 0: none
};

struct AttnModFwdArgs {
  AttnShape sh;
  ScoreMod mod;
  const lt_half* Q;
  const lt_half* K;
  const lt_half* V;
  int64_t q_stride, kv_stride;
  lt_half* O;
  int64_t o_stride;
  float* LSE;
};

// The hull of a group of 32 queries: some query of the group sees keys
// lo .. hi - 1 (none: lo >= hi), every query of it sees keys all_lo .. all_hi - 1.
struct QueryHull {
  int lo, hi, all_lo, all_hi;
};

// How the backward is launched.  The (batch, kv head) pairs are taken `chunk`
// at a time, each chunk's dK/dV pass followed by its dQ pass, so that the dS
// blocks in the workspace are one chunk's: a chunk is as large as keeps them
// within kModDsBudget, but has at least the workgroups to fill the CUs twice.
// (Chunks small enough for the 256 MB last-level cache lose: 4096 tokens of 40 heads
// in 4 chunks 1240 us, in one 990.)
//   ktile: keys per dK/dV workgroup, 256 or 128; nsplit: equal shares of a key tile's
// (query head, visible 64-query block) pairs, with partial sums when above 1.  Both
// by the estimated time of the pass: a 64-query block of a 256-key tile takes 4.3 us
// at D = 128 (0.55 of it for 128 keys, 1.8 at least), a workgroup's start and end 6, the
// sum pass 4 and what its partials take at 5 TB/s.  The interval of each query is on
// the device only, so that a causal mask is taken for the mean of equal key tiles
// (documents, windows) and of shrinking ones.  Measured against shares by the rule of
// lt_attn_bwd over 13 shapes x 4 masks: 0.96 of the time in the mean, 4 padded sequences of
// 333 tokens of 16 heads 34 us against 49, 2048 tokens of 40:8 heads 210 against 234.
constexpr int64_t kModDsBudget = (int64_t)8 << 30;
constexpr int kModMaxS = 1 << 19;         // the dK/dV pass lists a tile's 64-query blocks in LDS
constexpr int kModMaxShares = 16;
struct AttnModPlan {
  int chunk, ktile, nsplit;
};
inline AttnModPlan attn_mod_plan(int B, int S, int Hq, int Hkv, int D, int causal) {
  constexpr int64_t kCUs = 256;
  const int64_t pairs = (int64_t)B * Hkv, grp = Hq / Hkv, n_qb = ((int64_t)S + 63) / 64;
  const int64_t per_pair = grp * attn_bwd_ds_blocks(S, causal) * kDsBlockBytes;
  const int64_t fill = 2 * kCUs / ((((int64_t)S + 255) / 256) * grp);
  const int64_t fit = kModDsBudget / per_pair;
  int64_t c = fit > fill ? fit : fill;
  c = c < 1 ? 1 : c > pairs ? pairs : c;
  const int64_t chunks = (pairs + c - 1) / c;
  c = (pairs + chunks - 1) / chunks;
  AttnModPlan best = {(int)c, 256, 1};
  double best_us = 0;
  for (int ktile = 256; ktile >= 128; ktile /= 2) {
    const int64_t n_kt = ((int64_t)S + ktile - 1) / ktile;
    double block = 4.3 * D / 128 * (ktile == 256 ? 1.0 : 0.55);
    if (block < 1.8) block = 1.8;
    for (int n = 1; n <= kModMaxShares && (n == 1 || n <= grp * (n_qb < 4 ? n_qb : 4)); ++n) {
      const int64_t longest = (grp * n_qb + n - 1) / n, wgs = n_kt * c * n;
      double blocks = (double)((wgs + kCUs - 1) / kCUs * longest);
      if (causal) {
        const double even = 0.54 * (double)(grp * n_qb * n_kt * c) / kCUs;
        blocks = 0.5 * blocks + 0.5 * (even > (double)longest ? even : (double)longest);
      }
      double us = blocks * block + 6.0 * (wgs > kCUs ? (double)wgs / kCUs : 1.0);
      if (n > 1) us += 4.0 + n + (double)(n * c) * S * D * 16 / 5.0e6;
      if (best_us == 0 || us < best_us) {
        best_us = us;
        best = {(int)c, ktile, n};
      }
    }
  }
  return best;
}
// Workspace parts of the backward, in order, each 256-byte aligned: D and the
// base-2 LSE [B, Hq, S] FP32, the rows' intervals [2][B, S] and the hulls
// [B][ceil(S / 32)], a bit for every query of a head (tiles of kSharpTile), one chunk's
// dS blocks, a byte for every dS block of every head (used with a distance bias), one
// chunk's partial dK and dV.
constexpr int kSharpTile = 128;
struct AttnModWs {
  size_t lse2, rows, hulls, sharp, ds, live, part, total;
};
inline AttnModWs attn_mod_ws(int B, int S, int Hq, int Hkv, int D, int causal) {
  const AttnModPlan p = attn_mod_plan(B, S, Hq, Hkv, D, causal);
  const size_t n32 = ((size_t)S + 31) / 32;
  AttnModWs w;
  w.lse2 = align256((size_t)B * Hq * S * sizeof(float));
  w.rows = 2 * w.lse2;
  w.hulls = w.rows + align256((size_t)2 * B * S * sizeof(int32_t));
  w.sharp = w.hulls + align256((size_t)B * n32 * sizeof(QueryHull));
  w.ds = w.sharp + align256((size_t)B * Hq * (((size_t)S + kSharpTile - 1) / kSharpTile) * (kSharpTile / 8));
  const size_t blocks = (size_t)attn_bwd_ds_blocks(S, causal);
  w.live = w.ds + align256((size_t)p.chunk * (Hq / Hkv) * blocks * kDsBlockBytes);
  w.part = w.live + align256((size_t)B * Hq * blocks);
  w.total = w.part + (p.nsplit > 1 ? align256((size_t)2 * p.chunk * p.nsplit * S * D * sizeof(float)) : 0);
  return w;
}

struct AttnModBwdArgs {
  AttnShape sh;
  ScoreMod mod;
  const lt_half* Q;
  const lt_half* K;
  const lt_half* V;
  int64_t q_stride, kv_stride;
  const lt_half* O;
  const lt_half* dO;
  int64_t o_stride;
  const float* LSE;
  lt_half* dQ;
  lt_half* dK;
  lt_half* dV;
  int64_t dq_stride, dkv_stride;
  AttnModPlan plan;
  float* delta;           // workspace, see AttnModWs
  float* lse2;
  int32_t* rows;
  QueryHull* hulls;
  uint32_t* sharp;
  lt_half* ds;
  uint8_t* live;          // [B, Hq] blocks: kLiveBlock, or the block is not written
  float* part;
};

hipError_t attn_mod_fwd_launch(const AttnModFwdArgs& a, hipStream_t s);
hipError_t attn_mod_bwd_launch(const AttnModBwdArgs& a, hipStream_t s);

// ---------------------------------------------------------------- QK norm with rotation
struct QkNormArgs {
  const lt_half* X;       // [T, >= (Hq + Hkv) D] heads before the norm
  int64_t ldx;
  const lt_half* Wq;      // [D] norm weights
  const lt_half* Wk;
  const float* CS;        // [P][D / 2] (cos, sin)
  int P;
  const int32_t* POS;     // [T] or null: t % S
  int64_t T;
  int S, Hq, Hkv, D;
};
// lanes per head row: D / 16 rounded up to a power of two
inline int qknorm_lanes(int D) {
  int l = 1;
  while (l < D / 16) l *= 2;
  return l;
}
// How a wave's head rows are divided: 2^shift heads of a token (all of them, up to what a
// wave holds) by as many tokens as that leaves room for, a token group; and where there
// are few groups, each one's heads over several waves, up to 2048 waves (eight per CU), since
// a wave's time is then its passes' latency.  80 tokens of 64 + 8 heads: forward 3.1
// us instead of 8.7.
struct HeadSplit {
  int shift, groups, parts;
};
inline HeadSplit qknorm_split(int64_t T, int heads, int D) {
  const int rows = 64 / qknorm_lanes(D);
  HeadSplit h = {0, 0, 1};
  while ((1 << h.shift) < heads && (1 << h.shift) < rows) ++h.shift;
  const int64_t tokens = rows >> h.shift;
  h.groups = (int)((T + tokens - 1) / tokens);
  const int passes = (heads + (1 << h.shift) - 1) >> h.shift, most = 2048 / h.groups;
  if (most > 1) h.parts = most < passes ? most : passes;
  return h;
}
// Backward: query and key heads one after the other in every workgroup or, up to 256
// workgroups, in workgroups of their own.  dW partial sums: one FP32 row of 2 D
// per workgroup, at most 512 of them (two tokens a wave at T = 4096: 27 us; 1024 31 us,
// 256 36 us).
constexpr int kQkNormWaves = 4;
inline int qknorm_blocks(const HeadSplit& h) {
  const int64_t units = (int64_t)h.groups * h.parts;
  return (int)((units + kQkNormWaves - 1) / kQkNormWaves);
}
inline int qknorm_bwd_blocks(int64_t T, int Hq, int Hkv, int D) {
  const int q = qknorm_blocks(qknorm_split(T, Hq, D)), k = qknorm_blocks(qknorm_split(T, Hkv, D));
  const int b = q > k ? q : k;
  return b < 512 ? b : 512;
}
inline size_t qknorm_bwd_ws_bytes(int64_t T, int Hq, int Hkv, int D) {
  return align256((size_t)qknorm_bwd_blocks(T, Hq, Hkv, D) * 2 * D * sizeof(float));
}
hipError_t qknorm_fwd_launch(const QkNormArgs& a, lt_half* Y, int64_t ldy, float* RSTD, float eps, hipStream_t s);
hipError_t qknorm_bwd_launch(const QkNormArgs& a, const lt_half* dY, int64_t lddy, const float* RSTD, lt_half* dX,
                             int64_t lddx, lt_half* dWq, lt_half* dWk, float* part, hipStream_t s);

// ---------------------------------------------------------------- embedding
// Gradient: the tokens are sorted by row (stable); a row of more than kEmbedPart
// tokens is summed in pieces of so many.
constexpr int kEmbedPart = 16;
// rows of the table per sorting workgroup: a power of two that gives 128 to 256
// workgroups where the table has the rows for it
inline int embed_sort_rows(int64_t V) {
  int r = 32;
  while (r < 1024 && V / (2 * r) >= 128) r *= 2;
  return r;
}
inline int64_t embed_parts(int64_t T) { return (T + kEmbedPart - 1) / kEmbedPart; }
// Workspace: start [V + 1] (first sorted position of a row), tokens [T] in
// sorted order, two FP32 partial rows per kEmbedPart positions, each 256-byte
// aligned.
struct EmbedWs {
  size_t tokens, part, total;
};
inline EmbedWs embed_bwd_ws(int64_t T, int64_t H, int64_t V) {
  EmbedWs w;
  w.tokens = align256((size_t)(V + 1) * sizeof(int32_t));
  w.part = w.tokens + align256((size_t)T * sizeof(int32_t));
  w.total = w.part + align256((size_t)2 * embed_parts(T) * H * sizeof(float));
  return w;
}
// workgroups of the largest launch (256 threads each, below 2^32 threads)
inline bool embed_fits(int64_t T, int64_t H, int64_t V) {
  return T < (int64_t)1 << 24 && V < (int64_t)1 << 25 &&
         embed_parts(T) * ((H + 511) / 512) + V / 4 + 1 < (int64_t)1 << 24;
}
struct EmbedBwdArgs {
  const int64_t* ids;
  const lt_half* dY;
  int64_t lddy;
  float scale;
  int accumulate;
  lt_half* dW;
  int64_t lddw;
  int64_t T, H, V;
  int32_t* start;         // workspace, see EmbedWs
  int32_t* tokens;
  float* part;
};
hipError_t embed_fwd_launch(const int64_t* ids, const lt_half* W, int64_t ldw, float scale, lt_half* Y, int64_t ldy,
                            int64_t T, int64_t H, int64_t V, hipStream_t s);
hipError_t embed_bwd_launch(const EmbedBwdArgs& a, hipStream_t s);

}  // namespace lt
