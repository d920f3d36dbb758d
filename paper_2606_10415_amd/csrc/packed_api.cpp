// C ABI of the packed-sequence operators: argument checks, workspace layout and
// dispatch.  Declarations and the full contract are in include/lt.h.
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "packed.hpp"

namespace {

lt_status fail(lt_status s, const char* fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  return lt::set_error(s, buf);
}

lt_status ok() { return lt::set_error(LT_OK, ""); }

lt_status from_hip(hipError_t e, const char* what) {
  if (e == hipSuccess) return ok();
  return fail(LT_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

bool aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// element counts are formed from these products
constexpr int64_t kMaxRows = ((int64_t)1 << 31) - 1;
// a launch has fewer than 2^32 threads: 64-query tiles of at most 512, tokens of 64
constexpr int64_t kMaxTiles = (int64_t)1 << 22;
constexpr int64_t kMaxTokens = (int64_t)1 << 25;

// rows of up to 256 are loaded with 32-bit byte offsets
constexpr int64_t kMaxAttnStride = (int64_t)1 << 22;

constexpr float kMaxCap = 1000.f;

// rows * heads up to kMaxRows, checked without overflow
bool too_many(int64_t rows, int64_t heads) { return rows > kMaxRows / heads; }

lt_status check_workspace(const void* ws, size_t given, size_t need) {
  if (!ws || given < need)
    return fail(LT_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, ws ? given : (size_t)0);
  if (!aligned(ws, 256)) return fail(LT_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  return LT_OK;
}

bool attn_mod_shape_ok(int B, int S, int Hq, int Hkv, int D) {
  return B >= 1 && S >= 1 && Hq >= 1 && Hkv >= 1 && Hq % Hkv == 0 && (D == 64 || D == 128) && S <= lt::kModMaxS &&
         !too_many((int64_t)B * S, Hq) && ((int64_t)S + 63) / 64 * B * Hq <= kMaxTiles;
}

lt_status check_attn_mod(const void* Q, const void* K, const void* V, int64_t q_stride, int64_t kv_stride,
                         const void* O, int64_t o_stride, const float* LSE, const lt::ScoreMod& m, int B, int S,
                         int Hq, int Hkv, int D, float scale, int causal) {
  if (!Q || !K || !V || !O || !LSE) return fail(LT_ERR_INVALID_ARG, "NULL Q/K/V/O/LSE pointer");
  if (B < 1 || S < 1 || Hq < 1 || Hkv < 1 || D < 1)
    return fail(LT_ERR_INVALID_ARG, "B, S, Hq, Hkv, D must be >= 1 (got %d %d %d %d %d)", B, S, Hq, Hkv, D);
  if (Hq % Hkv != 0) return fail(LT_ERR_INVALID_ARG, "Hq (%d) must be a multiple of Hkv (%d)", Hq, Hkv);
  if (causal != 0 && causal != 1) return fail(LT_ERR_INVALID_ARG, "causal must be 0 or 1");
  if (!(scale > 0.f) || !std::isfinite(scale)) return fail(LT_ERR_INVALID_ARG, "scale must be finite and > 0");
  if (!(m.cap >= 0.f) || !std::isfinite(m.cap)) return fail(LT_ERR_INVALID_ARG, "cap must be finite and >= 0");
  if (q_stride < (int64_t)Hq * D || o_stride < (int64_t)Hq * D || kv_stride < (int64_t)Hkv * D)
    return fail(LT_ERR_INVALID_ARG, "q/kv/o row stride smaller than the row length");
  if (D != 64 && D != 128) return fail(LT_ERR_UNSUPPORTED, "head dim %d not in {64, 128}", D);
  if (S > lt::kModMaxS) return fail(LT_ERR_UNSUPPORTED, "S above 2^19");
  if (m.cap > kMaxCap || (m.cap > 0.f && !std::isfinite(4.f * scale / m.cap)))
    return fail(LT_ERR_UNSUPPORTED, "cap above 1000, or scale / cap too large");
  if ((q_stride | kv_stride | o_stride) & 7)
    return fail(LT_ERR_UNSUPPORTED, "row strides must be multiples of 8 elements");
  if (q_stride >= kMaxAttnStride || kv_stride >= kMaxAttnStride || o_stride >= kMaxAttnStride)
    return fail(LT_ERR_UNSUPPORTED, "row strides must be < 2^22 elements (32-bit buffer offsets)");
  if (!aligned(Q, 16) || !aligned(K, 16) || !aligned(V, 16) || !aligned(O, 16))
    return fail(LT_ERR_UNSUPPORTED, "Q/K/V/O must be 16-byte aligned");
  if (!aligned(LSE, 4) || !aligned(m.lo, 4) || !aligned(m.hi, 4) || !aligned(m.slopes, 4))
    return fail(LT_ERR_UNSUPPORTED, "LSE, LO, HI and slopes must be 4-byte aligned");
  if (!attn_mod_shape_ok(B, S, Hq, Hkv, D)) return fail(LT_ERR_UNSUPPORTED, "B*S*Hq too large");
  return LT_OK;
}

lt_status check_qknorm(const void* X, int64_t ldx, const void* Wq, const void* Wk, const float* CS, int P,
                       const int32_t* POS, const void* Y, int64_t ldy, const float* RSTD, int B, int S, int Hq,
                       int Hkv, int D) {
  if (!X || !Wq || !Wk || !CS || !Y || !RSTD) return fail(LT_ERR_INVALID_ARG, "NULL pointer");
  if (B < 1 || S < 1 || Hq < 1 || Hkv < 1 || D < 2 || P < 1) return fail(LT_ERR_INVALID_ARG, "non-positive size");
  if (!POS && S > P) return fail(LT_ERR_INVALID_ARG, "the table has %d positions, S is %d", P, S);
  if (ldx < ((int64_t)Hq + Hkv) * D || ldy < ((int64_t)Hq + Hkv) * D)
    return fail(LT_ERR_INVALID_ARG, "row stride smaller than (Hq + Hkv) * D");
  if ((D & 15) || D > 256) return fail(LT_ERR_UNSUPPORTED, "D must be a multiple of 16 and <= 256");
  if ((ldx | ldy) & 7) return fail(LT_ERR_UNSUPPORTED, "row strides must be multiples of 8 elements");
  if (!aligned(X, 16) || !aligned(Wq, 16) || !aligned(Wk, 16) || !aligned(CS, 16) || !aligned(Y, 16))
    return fail(LT_ERR_UNSUPPORTED, "X, weights, CS and outputs must be 16-byte aligned");
  if (!aligned(RSTD, 4) || !aligned(POS, 4)) return fail(LT_ERR_UNSUPPORTED, "RSTD and POS must be 4-byte aligned");
  if (too_many((int64_t)B * S, (int64_t)Hq + Hkv) || (int64_t)B * S > kMaxTokens)
    return fail(LT_ERR_UNSUPPORTED, "B*S or B*S*(Hq+Hkv) too large");
  if (X == Y && ldx != ldy) return fail(LT_ERR_INVALID_ARG, "in place: one row stride");
  return LT_OK;
}

lt_status check_embed(const int64_t* ids, const void* A, int64_t lda, const void* C, int64_t ldc, float scale,
                      int64_t T, int64_t H, int64_t V) {
  if (T < 0 || H < 1 || V < 1) return fail(LT_ERR_INVALID_ARG, "T < 0, H < 1 or V < 1");
  if (!A || !C || (!ids && T > 0)) return fail(LT_ERR_INVALID_ARG, "NULL pointer");
  if (lda < H || ldc < H) return fail(LT_ERR_INVALID_ARG, "row stride smaller than H");
  if (!std::isfinite(scale)) return fail(LT_ERR_INVALID_ARG, "scale must be finite");
  if ((H & 7) || H > 65536) return fail(LT_ERR_UNSUPPORTED, "H must be a multiple of 8 and <= 65536");
  if ((lda | ldc) & 7) return fail(LT_ERR_UNSUPPORTED, "row strides must be multiples of 8 elements");
  if (!lt::embed_fits(T, H, V)) return fail(LT_ERR_UNSUPPORTED, "too many tokens, columns or rows for one launch");
  if (!aligned(A, 16) || !aligned(C, 16)) return fail(LT_ERR_UNSUPPORTED, "rows must be 16-byte aligned");
  if (!aligned(ids, 8)) return fail(LT_ERR_UNSUPPORTED, "ids must be 8-byte aligned");
  return LT_OK;
}

}  // namespace

extern "C" {

lt_status lt_attn_mod_fwd(const lt_half* Q, const lt_half* K, const lt_half* V, int64_t q_row_stride,
                          int64_t kv_row_stride, lt_half* O, int64_t o_row_stride, float* LSE, const int32_t* LO,
                          const int32_t* HI, const float* slopes, float cap, int B, int S, int Hq, int Hkv, int D,
                          float scale, int causal, lt_stream stream) {
  const lt::ScoreMod m{LO, HI, slopes, cap};
  lt_status st = check_attn_mod(Q, K, V, q_row_stride, kv_row_stride, O, o_row_stride, LSE, m, B, S, Hq, Hkv, D, scale,
                                causal);
  if (st != LT_OK) return st;
  lt::AttnModFwdArgs a{{B, S, Hq, Hkv, D, scale, causal}, m, Q, K, V, q_row_stride, kv_row_stride, O, o_row_stride,
                       LSE};
  return from_hip(lt::attn_mod_fwd_launch(a, reinterpret_cast<hipStream_t>(stream)), "attn_mod_fwd launch");
}

size_t lt_attn_mod_bwd_workspace_size(int B, int S, int Hq, int Hkv, int D, int causal) {
  if (!attn_mod_shape_ok(B, S, Hq, Hkv, D) || (causal != 0 && causal != 1)) return 0;
  return lt::attn_mod_ws(B, S, Hq, Hkv, D, causal).total;
}

lt_status lt_attn_mod_bwd(const lt_half* Q, const lt_half* K, const lt_half* V, int64_t q_row_stride,
                          int64_t kv_row_stride, const lt_half* O, const lt_half* dO, int64_t o_row_stride,
                          const float* LSE, const int32_t* LO, const int32_t* HI, const float* slopes, float cap,
                          lt_half* dQ, lt_half* dK, lt_half* dV, int64_t dq_row_stride, int64_t dkv_row_stride,
                          void* workspace, size_t ws_bytes, int B, int S, int Hq, int Hkv, int D, float scale,
                          int causal, lt_stream stream) {
  const lt::ScoreMod m{LO, HI, slopes, cap};
  lt_status st = check_attn_mod(Q, K, V, q_row_stride, kv_row_stride, O, o_row_stride, LSE, m, B, S, Hq, Hkv, D, scale,
                                causal);
  if (st != LT_OK) return st;
  if (!dO || !dQ || !dK || !dV) return fail(LT_ERR_INVALID_ARG, "NULL dO/dQ/dK/dV pointer");
  if (dq_row_stride < (int64_t)Hq * D || dkv_row_stride < (int64_t)Hkv * D)
    return fail(LT_ERR_INVALID_ARG, "dq/dkv row stride smaller than the row length");
  if ((dq_row_stride | dkv_row_stride) & 7)
    return fail(LT_ERR_UNSUPPORTED, "row strides must be multiples of 8 elements");
  if (dq_row_stride >= kMaxAttnStride || dkv_row_stride >= kMaxAttnStride)
    return fail(LT_ERR_UNSUPPORTED, "dq/dkv row strides must be < 2^22 elements");
  if (!aligned(dO, 16) || !aligned(dQ, 16) || !aligned(dK, 16) || !aligned(dV, 16))
    return fail(LT_ERR_UNSUPPORTED, "dO/dQ/dK/dV must be 16-byte aligned");
  const lt::AttnModWs w = lt::attn_mod_ws(B, S, Hq, Hkv, D, causal);
  if ((st = check_workspace(workspace, ws_bytes, w.total)) != LT_OK) return st;
  char* ws = static_cast<char*>(workspace);
  lt::AttnModBwdArgs a{{B, S, Hq, Hkv, D, scale, causal},
                       m,
                       Q,
                       K,
                       V,
                       q_row_stride,
                       kv_row_stride,
                       O,
                       dO,
                       o_row_stride,
                       LSE,
                       dQ,
                       dK,
                       dV,
                       dq_row_stride,
                       dkv_row_stride,
                       lt::attn_mod_plan(B, S, Hq, Hkv, D, causal),
                       reinterpret_cast<float*>(ws),
                       reinterpret_cast<float*>(ws + w.lse2),
                       reinterpret_cast<int32_t*>(ws + w.rows),
                       reinterpret_cast<lt::QueryHull*>(ws + w.hulls),
                       reinterpret_cast<uint32_t*>(ws + w.sharp),
                       reinterpret_cast<lt_half*>(ws + w.ds),
                       reinterpret_cast<uint8_t*>(ws + w.live),
                       reinterpret_cast<float*>(ws + w.part)};
  return from_hip(lt::attn_mod_bwd_launch(a, reinterpret_cast<hipStream_t>(stream)), "attn_mod_bwd launch");
}

lt_status lt_qknorm_rope_fwd(const lt_half* X, int64_t ldx, const lt_half* Wq, const lt_half* Wk, const float* CS,
                             int P, const int32_t* POS, lt_half* Y, int64_t ldy, float* RSTD, int B, int S, int Hq,
                             int Hkv, int D, float eps, lt_stream stream) {
  lt_status st = check_qknorm(X, ldx, Wq, Wk, CS, P, POS, Y, ldy, RSTD, B, S, Hq, Hkv, D);
  if (st != LT_OK) return st;
  if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(LT_ERR_INVALID_ARG, "eps must be finite and >= 0");
  lt::QkNormArgs a{X, ldx, Wq, Wk, CS, P, POS, (int64_t)B * S, S, Hq, Hkv, D};
  return from_hip(lt::qknorm_fwd_launch(a, Y, ldy, RSTD, eps, reinterpret_cast<hipStream_t>(stream)),
                  "qknorm_rope_fwd launch");
}

size_t lt_qknorm_rope_bwd_workspace_size(int B, int S, int Hq, int Hkv, int D) {
  if (B < 1 || S < 1 || Hq < 1 || Hkv < 1 || D < 2 || (D & 15) || D > 256 ||
      too_many((int64_t)B * S, (int64_t)Hq + Hkv) || (int64_t)B * S > kMaxTokens)
    return 0;
  return lt::qknorm_bwd_ws_bytes((int64_t)B * S, Hq, Hkv, D);
}

lt_status lt_qknorm_rope_bwd(const lt_half* dY, int64_t lddy, const lt_half* X, int64_t ldx, const lt_half* Wq,
                             const lt_half* Wk, const float* RSTD, const float* CS, int P, const int32_t* POS,
                             lt_half* dX, int64_t lddx, lt_half* dWq, lt_half* dWk, void* workspace, size_t ws_bytes,
                             int B, int S, int Hq, int Hkv, int D, lt_stream stream) {
  lt_status st = check_qknorm(X, ldx, Wq, Wk, CS, P, POS, dX, lddx, RSTD, B, S, Hq, Hkv, D);
  if (st != LT_OK) return st;
  if (!dY || !dWq || !dWk) return fail(LT_ERR_INVALID_ARG, "NULL dY/dWq/dWk pointer");
  if (lddy < ((int64_t)Hq + Hkv) * D) return fail(LT_ERR_INVALID_ARG, "row stride smaller than (Hq + Hkv) * D");
  if (lddy & 7) return fail(LT_ERR_UNSUPPORTED, "row strides must be multiples of 8 elements");
  if (!aligned(dY, 16) || !aligned(dWq, 2) || !aligned(dWk, 2))
    return fail(LT_ERR_UNSUPPORTED, "dY must be 16-byte, dWq and dWk 2-byte aligned");
  if (dY == dX && lddy != lddx) return fail(LT_ERR_INVALID_ARG, "in place: one row stride");
  if ((st = check_workspace(workspace, ws_bytes, lt::qknorm_bwd_ws_bytes((int64_t)B * S, Hq, Hkv, D))) != LT_OK) return st;
  lt::QkNormArgs a{X, ldx, Wq, Wk, CS, P, POS, (int64_t)B * S, S, Hq, Hkv, D};
  return from_hip(lt::qknorm_bwd_launch(a, dY, lddy, RSTD, dX, lddx, dWq, dWk, static_cast<float*>(workspace),
                                        reinterpret_cast<hipStream_t>(stream)),
                  "qknorm_rope_bwd launch");
}

lt_status lt_embed_fwd(const int64_t* ids, const lt_half* W, int64_t ldw, float scale, lt_half* Y, int64_t ldy,
                       int64_t T, int64_t H, int64_t V, lt_stream stream) {
  lt_status st = check_embed(ids, W, ldw, Y, ldy, scale, T, H, V);
  if (st != LT_OK) return st;
  if (T == 0) return ok();
  return from_hip(lt::embed_fwd_launch(ids, W, ldw, scale, Y, ldy, T, H, V, reinterpret_cast<hipStream_t>(stream)),
                  "embed_fwd launch");
}

size_t lt_embed_bwd_workspace_size(int64_t T, int64_t H, int64_t V) {
  if (T < 0 || H < 1 || V < 1 || (H & 7) || H > 65536 || !lt::embed_fits(T, H, V)) return 0;
  return lt::embed_bwd_ws(T, H, V).total;
}

lt_status lt_embed_bwd(const int64_t* ids, const lt_half* dY, int64_t lddy, float scale, int accumulate, lt_half* dW,
                       int64_t lddw, void* workspace, size_t ws_bytes, int64_t T, int64_t H, int64_t V,
                       lt_stream stream) {
  // dY may be NULL when there is no token
  lt_status st = check_embed(ids, T > 0 ? dY : dW, T > 0 ? lddy : H, dW, lddw, scale, T, H, V);
  if (st != LT_OK) return st;
  if (accumulate != 0 && accumulate != 1) return fail(LT_ERR_INVALID_ARG, "accumulate must be 0 or 1");
  const lt::EmbedWs w = lt::embed_bwd_ws(T, H, V);
  if ((st = check_workspace(workspace, ws_bytes, w.total)) != LT_OK) return st;
  if (T == 0 && accumulate) return ok();
  char* ws = static_cast<char*>(workspace);
  lt::EmbedBwdArgs a{ids,
                     dY,
                     lddy,
                     scale,
                     accumulate,
                     dW,
                     lddw,
                     T,
                     H,
                     V,
                     reinterpret_cast<int32_t*>(ws),
                     reinterpret_cast<int32_t*>(ws + w.tokens),
                     reinterpret_cast<float*>(ws + w.part)};
  return from_hip(lt::embed_bwd_launch(a, reinterpret_cast<hipStream_t>(stream)), "embed_bwd launch");
}

}  // extern "C"
