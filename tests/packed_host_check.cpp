// Host-only check of the packed-sequence operators' C ABI layer
// (csrc/packed_api.cpp) under AddressSanitizer and UndefinedBehaviorSanitizer.
//
// The launchers below stand in for the kernel translation units: each checks
// that what it was handed lies inside what the caller passed and that its plan
// covers the work, and returns hipErrorNoDevice (reported as LT_ERR_HIP).  No
// device code is compiled and no GPU call is made.
#include <hip/hip_runtime.h>

#include <climits>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <string>

#include "lt.h"
#include "../paper_2606_10415_amd/csrc/packed.hpp"

static int g_failures = 0, g_launches = 0;
static uintptr_t g_lo = 0, g_hi = 0;   // workspace of the current call

#define CHECK(cond, ...)                                          \
  do {                                                            \
    if (!(cond)) {                                                \
      ++g_failures;                                               \
      std::fprintf(stderr, "FAILED %s:%d: ", __FILE__, __LINE__); \
      std::fprintf(stderr, __VA_ARGS__);                          \
      std::fprintf(stderr, "\n");                                 \
    }                                                             \
  } while (0)

static uintptr_t inside(const void* p, size_t bytes, uintptr_t after, const char* what) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p);
  CHECK(a >= g_lo && a + bytes <= g_hi, "%s outside the workspace", what);
  CHECK(a >= after, "%s overlaps the part before it", what);
  CHECK((a & 255) == 0, "%s not 256-byte aligned", what);
  return a + bytes;
}

namespace lt {
static std::string g_error;
lt_status set_error(lt_status s, const char* msg) {
  g_error = msg;
  return s;
}
hipError_t attn_mod_fwd_launch(const AttnModFwdArgs&, hipStream_t) {
  ++g_launches;
  return hipErrorNoDevice;
}
hipError_t attn_mod_bwd_launch(const AttnModBwdArgs& a, hipStream_t) {
  ++g_launches;
  const AttnShape& s = a.sh;
  const size_t rows = (size_t)s.B * s.Hq * s.S * 4, n32 = ((size_t)s.S + 31) / 32, grp = s.Hq / s.Hkv;
  const int pairs = s.B * s.Hkv;
  CHECK(a.plan.chunk >= 1 && a.plan.chunk <= pairs, "chunk %d of %d", a.plan.chunk, pairs);
  CHECK(a.plan.ktile == 256 || a.plan.ktile == 128, "key tile %d", a.plan.ktile);
  CHECK(a.plan.nsplit >= 1, "shares %d", a.plan.nsplit);
  uintptr_t at = inside(a.delta, rows, 0, "D");
  at = inside(a.lse2, rows, at, "LSE2");
  at = inside(a.rows, (size_t)2 * s.B * s.S * 4, at, "intervals");
  at = inside(a.hulls, (size_t)s.B * n32 * 16, at, "hulls");
  at = inside(a.sharp, (size_t)s.B * s.Hq * (((size_t)s.S + 127) / 128) * 16, at, "marks");
  const size_t blocks = s.causal ? n32 * (n32 + 1) / 2 : n32 * n32;
  at = inside(a.ds, (size_t)a.plan.chunk * grp * blocks * 2048, at, "dS blocks");
  at = inside(a.live, (size_t)s.B * s.Hq * blocks, at, "dS marks");
  if (a.plan.nsplit > 1) inside(a.part, (size_t)2 * a.plan.chunk * a.plan.nsplit * s.S * s.D * 4, at, "partials");
  return hipErrorNoDevice;
}
hipError_t qknorm_fwd_launch(const QkNormArgs& a, lt_half*, int64_t, float*, float, hipStream_t) {
  ++g_launches;
  CHECK(a.POS || a.S <= a.P, "positions outside the table");
  return hipErrorNoDevice;
}
hipError_t qknorm_bwd_launch(const QkNormArgs& a, const lt_half*, int64_t, const float*, lt_half*, int64_t, lt_half*,
                             lt_half*, float* part, hipStream_t) {
  ++g_launches;
  CHECK(a.POS || a.S <= a.P, "positions outside the table");
  inside(part, (size_t)qknorm_bwd_blocks(a.T, a.Hq, a.Hkv, a.D) * 2 * a.D * 4, 0, "dw partials");
  return hipErrorNoDevice;
}
hipError_t embed_fwd_launch(const int64_t*, const lt_half*, int64_t, float, lt_half*, int64_t, int64_t, int64_t,
                            int64_t, hipStream_t) {
  ++g_launches;
  return hipErrorNoDevice;
}
hipError_t embed_bwd_launch(const EmbedBwdArgs& a, hipStream_t) {
  ++g_launches;
  uintptr_t at = inside(a.start, (size_t)(a.V + 1) * 4, 0, "row starts");
  at = inside(a.tokens, (size_t)a.T * 4, at, "sorted tokens");
  inside(a.part, (size_t)2 * ((a.T + kEmbedPart - 1) / kEmbedPart) * a.H * 4, at, "partial rows");
  const int r = embed_sort_rows(a.V);
  CHECK(r >= 32 && r <= 1024 && (r & (r - 1)) == 0, "rows per sorting workgroup %d", r);
  return hipErrorNoDevice;
}
}  // namespace lt

int main(int argc, char** argv) {
  const int n = argc > 1 ? std::atoi(argv[1]) : 1000;
  std::mt19937_64 rng(1);
  auto pick = [&](std::initializer_list<int64_t> v) { return *(v.begin() + rng() % v.size()); };
  auto ptr = [&]() -> void* {
    const int r = rng() % 40;
    return r == 0 ? nullptr : reinterpret_cast<void*>((uintptr_t)0x10000000 + (r == 1 ? 2 : r == 2 ? 8 : 0));
  };
  int valid = 0;
  for (int it = 0; it < n; ++it) {
    const bool wild = rng() % 4 == 0;
    const int B = (int)(wild ? pick({-1, 0, 1, 3, 1 << 20, INT_MAX}) : pick({1, 2, 8, 33}));
    const int S = (int)(wild ? pick({-5, 0, 1, 77, 1 << 19, (1 << 19) + 1, INT_MAX})
                             : pick({1, 2, 31, 333, 1024, 4096, 8191, 32768, 131072}));
    const int Hkv = (int)(wild ? pick({-1, 0, 1, 3, INT_MAX}) : pick({1, 2, 8, 32}));
    const int Hq = wild ? (int)pick({-1, 0, 4, INT_MAX}) : (int)(Hkv * pick({1, 2, 5, 8}));
    const int D = (int)(wild ? pick({0, 16, 100, 256, 512, INT_MAX}) : pick({64, 128}));
    const int causal = (int)(wild ? pick({-1, 0, 1, 2}) : pick({0, 1}));
    const float scale = wild ? (float)pick({0, -1, 1}) : 0.1f;
    const float cap = wild ? (float)pick({-1, 0, 30, 2000}) : (float)pick({0, 30});
    const int64_t qs = wild ? pick({0, 128, 1 << 21, INT64_MAX, INT64_MIN}) : (int64_t)(Hq + 2 * Hkv) * D + 8;
    const int64_t os = wild ? pick({0, 128, 1 << 21, INT64_MAX, 4097}) : (int64_t)Hq * D;
    lt_half* h[12];
    for (auto& p : h) p = (lt_half*)ptr();
    auto* lo = (int32_t*)(rng() % 2 ? ptr() : nullptr);
    auto* hi = (int32_t*)(rng() % 2 ? ptr() : nullptr);
    auto* sl = (float*)(rng() % 2 ? ptr() : nullptr);
    int before = g_launches;
    lt_status st = lt_attn_mod_fwd(h[0], h[1], h[2], qs, qs, h[3], os, (float*)h[4], lo, hi, sl, cap, B, S, Hq, Hkv, D,
                                   scale, causal, nullptr);
    CHECK((st == LT_ERR_HIP) == (g_launches == before + 1), "forward status %d", st);
    valid += st == LT_ERR_HIP;

    size_t need = lt_attn_mod_bwd_workspace_size(B, S, Hq, Hkv, D, causal);
    const size_t given = rng() % 8 ? need : need / 2;
    g_lo = (uintptr_t)1 << 40;
    g_hi = g_lo + given;
    before = g_launches;
    st = lt_attn_mod_bwd(h[0], h[1], h[2], qs, qs, h[3], h[5], os, (float*)h[4], lo, hi, sl, cap, h[6], h[7], h[8], qs,
                         qs, (void*)g_lo, given, B, S, Hq, Hkv, D, scale, causal, nullptr);
    CHECK((st == LT_ERR_HIP) == (g_launches == before + 1), "backward status %d", st);
    CHECK(st != LT_ERR_HIP || (given == need && need > 0), "launched with %zu of %zu", given, need);
    valid += st == LT_ERR_HIP;

    const int P = (int)pick({0, 1, 100, 131072});
    const int Dn = (int)(wild ? pick({0, 8, 24, 272}) : pick({16, 96, 128, 256}));
    const int64_t ld = wild ? pick({0, 128, INT64_MAX}) : (int64_t)(Hq + Hkv) * Dn;
    before = g_launches;
    st = lt_qknorm_rope_fwd(h[0], ld, h[1], h[2], (float*)h[3], P, lo, h[4], ld, (float*)h[5], B, S, Hq, Hkv, Dn,
                            wild ? -1.f : 1e-6f, nullptr);
    CHECK((st == LT_ERR_HIP) == (g_launches == before + 1), "norm status %d", st);
    valid += st == LT_ERR_HIP;
    need = lt_qknorm_rope_bwd_workspace_size(B, S, Hq, Hkv, Dn);
    g_hi = g_lo + need;
    before = g_launches;
    st = lt_qknorm_rope_bwd(h[0], ld, h[1], ld, h[2], h[3], (float*)h[4], (float*)h[5], P, lo, h[6], ld, h[7], h[8],
                            (void*)g_lo, need, B, S, Hq, Hkv, Dn, nullptr);
    CHECK((st == LT_ERR_HIP) == (g_launches == before + 1), "norm backward status %d", st);
    valid += st == LT_ERR_HIP;

    const int64_t T = wild ? pick({-1, 0, 1, INT64_MAX}) : pick({0, 1, 777, 65536, 1 << 29});
    const int64_t V = wild ? pick({-1, 0, 1, INT64_MAX}) : pick({1, 1000, 152064, (1 << 30) - 1});
    const int64_t H = wild ? pick({0, 4, 8, INT64_MAX}) : pick({8, 4096, 65536});
    auto* ids = (const int64_t*)ptr();
    before = g_launches;
    st = lt_embed_fwd(ids, h[0], H, 1.f, h[1], H, T, H, V, nullptr);
    CHECK((st == LT_ERR_HIP) == (g_launches == before + 1), "embedding status %d", st);
    valid += st == LT_ERR_HIP;
    need = lt_embed_bwd_workspace_size(T, H, V);
    g_hi = g_lo + need;
    before = g_launches;
    st = lt_embed_bwd(ids, h[0], H, 1.f, (int)(rng() % 2), h[1], H, (void*)g_lo, need, T, H, V, nullptr);
    CHECK((st == LT_ERR_HIP) == (g_launches == before + 1), "embedding gradient status %d", st);
    valid += st == LT_ERR_HIP;
  }
  std::printf("%d calls reached a launcher, %d failures\n", valid, g_failures);
  return g_failures == 0 && valid > n / 4 ? 0 : 1;
}
