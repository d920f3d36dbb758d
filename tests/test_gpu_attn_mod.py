"""GPU parity of lt_attn_mod_fwd / lt_attn_mod_bwd against the float64 oracle,
element by element.

Bounds (first-order error analysis, evaluated in float64 for every element; h =
2^-11 is half an FP16 step relative to the value, s = 2^-25 half its subnormal step):

  scores   |ds| <= 2^-23 (D + 8) scale |q|.|k|  (FP32 sums of exact products)
                  + 2^-20 cap  (exp2, reciprocal and their FP32 roundings, 2 C du)
                  + 2^-22 (|s| + |slope (i - j)| + |LSE|) + 2^-22  (products, exp2)
  row sum  dl <= sum_j P ds + 2^-24 S;   LSE: dl + 2^-21 + 2^-22 |LSE|
  O        sum_j P (h + ds + dl + 2^-23 S)|v| + s sum_seen |v|  (P as FP16; row sums are
           at least 1 in the kernel's units) + h |O| + s
  P back   dp = ds + dLSE
  dS       |dS| (h + dp) + s + P w (2^-23 (D + 8) |dO|.|v| + sum_f |dO| dO-row error
           of O + 2^-23 (D + 8) |dO|.|O|) + 2^-20 P |dP - D|  (the cap's derivative)
  dV, dK, dQ  the products with these errors, FP32 sums 2^-23 n, and h, s at the end
"""

import math

import numpy as np
import pytest

import oracle

pytestmark = pytest.mark.gpu

H, SUB = 2.0 ** -11, 2.0 ** -25


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a ROCm device"
    from paper_2606_10415_amd import lt
    return torch, lt


def f16(rng, *shape, std=1.0):
    return (rng.standard_normal(shape, dtype=np.float32) * std).astype(np.float16)


def make_mask(kind, B, S, rng):
    """(LO, HI, causal)"""
    i = np.arange(S, dtype=np.int32)
    lo, hi = np.zeros((B, S), np.int32), np.full((B, S), S, np.int32)
    if kind == "causal":
        return None, None, 1
    if kind == "full":
        return None, None, 0
    for b in range(B):
        cuts = sorted(set(rng.integers(0, S, size=min(S, 5)).tolist()) | {0})
        start = np.zeros(S, np.int32)
        end = np.full(S, S, np.int32)
        for a, e in zip(cuts, cuts[1:] + [S]):
            start[a:e], end[a:e] = a, e
        if kind == "docs":
            lo[b] = start
        elif kind == "docs_full":
            lo[b], hi[b] = start, end
        elif kind == "prefix":
            lo[b], hi[b] = start, np.maximum(i + 1, start + (end - start) // 3)
        elif kind == "pad":
            n = max(1, S - 3 - (S // 3) * (b % 2)) if S > 4 else 1
            hi[b] = np.where(i < n, n, 0)
        elif kind == "window":
            lo[b] = i - max(1, S // 5) + 1
        elif kind == "wild":                        # any interval at all, empty ones, far out of range
            x, y = rng.integers(-3, S + 4, size=S), rng.integers(-3, S + 4, size=S)
            lo[b], hi[b] = np.minimum(x, y), np.maximum(x, y)
            swap = rng.random(S) < 0.2
            lo[b, swap], hi[b, swap] = hi[b, swap], lo[b, swap]
            lo[b, rng.random(S) < 0.02] = -2 ** 31
            hi[b, rng.random(S) < 0.02] = 2 ** 31 - 1
    if kind == "docs":
        return lo, None, 1
    if kind == "window":
        return lo, None, 1
    if kind == "wild":
        return lo, hi, int(rng.integers(0, 2))
    return lo, hi, 0


def run_gpu(env, x, Hkv, D, scale, mask, cap, slopes, bwd=True, pad=0, stream=None):
    """x: Q [B,S,Hq,D], K, V [B,S,Hkv,D], dO.  Rows of the fused buffers have ``pad`` more columns and
    there are two rows behind the last; both must keep what they hold."""
    torch, lt = env
    B, S, Hq, _ = x["Q"].shape
    T, W = B * S, (Hq + 2 * Hkv) * D
    qkv = np.full((T + 2, W + pad), 7.0, np.float16)
    qkv[:T, :W] = np.concatenate([x[n].reshape(T, -1) for n in "QKV"], 1)
    QKV = torch.from_numpy(qkv).cuda()
    heads = lambda t: (t.data_ptr(), t.data_ptr() + 2 * Hq * D, t.data_ptr() + 2 * (Hq + Hkv) * D)
    lo, hi, causal = mask
    up = lambda a: None if a is None else torch.from_numpy(a).cuda()
    LO, HI, SL = up(lo), up(hi), up(slopes)
    O = torch.full((T + 2, Hq * D + pad), 3.0, dtype=torch.float16, device="cuda")
    O[:T, :Hq * D] = float("nan")
    LSE = torch.full((B, Hq, S), float("nan"), device="cuda")
    q, k, v = heads(QKV)
    lt.lt_attn_mod_fwd(q, k, v, W + pad, W + pad, O, Hq * D + pad, LSE, LO, HI, SL, cap, B, S, Hq, Hkv, D, scale,
                       causal, stream)
    res = {}
    if bwd:
        dO = torch.zeros((T + 2, Hq * D + pad), dtype=torch.float16, device="cuda")
        dO[:T, :Hq * D] = torch.from_numpy(x["dO"].reshape(T, -1)).cuda()
        dQKV = torch.full((T + 2, W + pad), 5.0, dtype=torch.float16, device="cuda")
        dQKV[:T, :W] = float("nan")
        n = lt.lt_attn_mod_bwd_workspace_size(B, S, Hq, Hkv, D, causal)
        ws = torch.full((n + 256,), 0xff, dtype=torch.uint8, device="cuda")      # NaN patterns
        dq, dk, dv = heads(dQKV)
        lt.lt_attn_mod_bwd(q, k, v, W + pad, W + pad, O, dO, Hq * D + pad, LSE, LO, HI, SL, cap, dq, dk, dv, W + pad,
                           W + pad, ws, n, B, S, Hq, Hkv, D, scale, causal, stream)
        torch.cuda.synchronize()
        assert bool((ws[n:] == 0xff).all())
        d = dQKV.cpu().numpy()
        assert np.all(d[T:] == 5.0) and np.all(d[:, W:] == 5.0)
        res["dQ"] = d[:T, :Hq * D].reshape(B, S, Hq, D)
        res["dK"] = d[:T, Hq * D:(Hq + Hkv) * D].reshape(B, S, Hkv, D)
        res["dV"] = d[:T, (Hq + Hkv) * D:W].reshape(B, S, Hkv, D)
    torch.cuda.synchronize()
    o = O.cpu().numpy()
    assert np.all(o[T:] == 3.0) and np.all(o[:, Hq * D:] == 3.0)
    res["O"], res["LSE"] = o[:T, :Hq * D].reshape(B, S, Hq, D), LSE.cpu().numpy()
    return res


def check(got, x, Hkv, scale, mask, cap, slopes, heads=None):
    B, S, Hq, D = x["Q"].shape
    lo, hi, causal = mask
    G = Hq // Hkv
    worst = {}

    def within(name, a, ref, tol):
        err = np.abs(a.astype(np.float64) - ref)
        bad = ~(err <= tol)
        worst[name] = max(worst.get(name, 0.0), float(np.max(err / tol)))
        assert not bad.any(), (name, int(bad.sum()), np.argwhere(bad)[:4].tolist(), worst)

    for b in range(B):
        l, h_ = oracle.intervals(S, None if lo is None else lo[b], None if hi is None else hi[b], bool(causal))
        for kv in range(Hkv):
            if heads is not None and (b, kv) not in heads:
                continue
            acc = {n: 0.0 for n in ("dK", "dV", "tK", "tV")}
            for h in range(kv * G, kv * G + G):
                q, k, v = x["Q"][b, :, h], x["K"][b, :, kv], x["V"][b, :, kv]
                slope = 0.0 if slopes is None else float(slopes[h])
                r = oracle.attn_mod_head(q, k, v, scale, l, h_, cap, slope, x["dO"][b, :, h])
                q, k, v, do = (np.where(m[:, None], a.astype(np.float64), 0.0) for a, m in
                               ((q, r["see"].any(1)), (k, r["see"].any(0)), (v, r["see"].any(0)),
                                (x["dO"][b, :, h], r["see"].any(1))))
                p, see, some = r["p"], r["see"], r["see"].any(1)
                aq, ak, av, ado = abs(q), abs(k), abs(v), abs(do)
                i = np.arange(S)
                lse = np.where(some, r["lse"], 0.0)
                s = abs(np.where(see, scale * (q @ k.T), 0.0))
                dist = abs(slope) * abs(i[:, None] - i[None, :])
                des = (2.0 ** -23 * (D + 8) * scale * (aq @ ak.T) + 2.0 ** -20 * cap +
                       2.0 ** -22 * (np.minimum(s, cap if cap > 0 else s) + dist + abs(lse)[:, None] + 1.0))
                dl = (p * des).sum(1) + 2.0 ** -24 * S
                got_lse = got["LSE"][b, h]
                assert np.all(got_lse[~some] == -np.inf)
                dlse = dl + 2.0 ** -21 + 2.0 ** -22 * abs(lse)
                within("LSE", np.where(some, got_lse, 0.0), lse, dlse)
                tO = ((p * (H + des + dl[:, None] + 2.0 ** -23 * S)) @ av + SUB * (see.astype(float) @ av) +
                      H * abs(r["o"]) + SUB)
                within("O", got["O"][b, :, h], r["o"], tO)
                assert np.all(got["O"][b, ~some, h] == 0)
                if "dQ" not in got:
                    continue
                dp = des + dlse[:, None]
                dD = (ado * tO).sum(1) + 2.0 ** -23 * (D + 8) * (ado * abs(r["o"])).sum(1)
                ddp = 2.0 ** -23 * (D + 8) * (ado @ av.T)
                tds = np.where(see, abs(r["ds"]) * (H + dp) + SUB + p * r["w"] * (ddp + dD[:, None]) +
                               2.0 ** -20 * p * abs(r["dp"] - r["delta"][:, None]), 0.0)
                n = 2.0 ** -23 * (S + 8)
                tQ = scale * (tds @ ak + n * (abs(r["ds"]) @ ak)) + H * abs(r["dq"]) + SUB
                within("dQ", got["dQ"][b, :, h], r["dq"], tQ)
                assert np.all(got["dQ"][b, ~some, h] == 0)
                n *= G
                acc["dK"] = acc["dK"] + r["dk"]
                acc["dV"] = acc["dV"] + r["dv"]
                acc["tK"] = acc["tK"] + scale * (tds.T @ aq + n * (abs(r["ds"]).T @ aq))
                tp = np.where(see, p * (H + dp) + SUB, 0.0)
                acc["tV"] = acc["tV"] + tp.T @ ado + n * (p.T @ ado)
            if "dQ" not in got:
                continue
            within("dK", got["dK"][b, :, kv], acc["dK"], acc["tK"] + H * abs(acc["dK"]) + SUB)
            within("dV", got["dV"][b, :, kv], acc["dV"], acc["tV"] + H * abs(acc["dV"]) + SUB)
    return worst


def inputs(seed, B, S, Hq, Hkv, D, std=1.0):
    rng = np.random.Generator(np.random.PCG64(seed))
    return rng, dict(Q=f16(rng, B, S, Hq, D, std=std), K=f16(rng, B, S, Hkv, D, std=std), V=f16(rng, B, S, Hkv, D),
                     dO=f16(rng, B, S, Hq, D))


def slopes_of(n):
    return np.array([2.0 ** (-8.0 * (k + 1) / n) for k in range(n)], np.float32)


CASES = [
    # B, S, Hq, Hkv, D, mask, cap, slopes, std of q and k, padding columns
    (1, 1, 1, 1, 64, "causal", 0.0, False, 1.0, 0),
    (2, 1, 4, 2, 128, "pad", 30.0, True, 1.0, 8),
    (1, 2, 2, 1, 64, "docs", 0.0, False, 1.0, 0),
    (3, 33, 3, 3, 128, "docs", 0.0, False, 1.0, 0),
    (1, 64, 2, 2, 64, "full", 20.0, False, 3.0, 8),
    (2, 65, 4, 1, 128, "prefix", 0.0, True, 1.0, 0),
    (4, 130, 4, 4, 64, "pad", 0.0, False, 1.0, 16),
    (1, 127, 5, 1, 128, "window", 50.0, False, 4.0, 0),
    (2, 257, 4, 2, 128, "docs_full", 0.0, False, 1.0, 0),
    (2, 300, 6, 2, 64, "wild", 0.0, False, 1.0, 8),
    (2, 301, 4, 4, 128, "wild", 25.0, True, 3.0, 0),
    (1, 515, 8, 2, 128, "docs", 30.0, True, 2.0, 0),
    (1, 700, 2, 2, 64, "causal", 0.0, True, 1.0, 0),
    (8, 259, 16, 16, 64, "docs", 0.0, False, 1.0, 0),
    (1, 1111, 8, 8, 128, "prefix", 0.0, False, 1.0, 0),
    (1, 1030, 40, 8, 128, "window", 0.0, False, 1.0, 0),
    (1, 900, 2, 1, 64, "full", 1000.0, False, 1.0, 0),
    (1, 333, 2, 2, 128, "causal", 0.5, False, 1.0, 0),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c))
def test_parity(env, case):
    B, S, Hq, Hkv, D, kind, cap, biased, std, pad = case
    print("attn_mod", case, flush=True)
    rng, x = inputs(100 + S, B, S, Hq, Hkv, D, std)
    mask = make_mask(kind, B, S, rng)
    slopes = slopes_of(Hq) if biased else None
    scale = 1.0 / math.sqrt(D)
    got = run_gpu(env, x, Hkv, D, scale, mask, cap, slopes, pad=pad)
    heads = None if B * Hq * S * S < 4e7 else {(0, 0), (B - 1, Hkv - 1)}
    print({k: round(v, 3) for k, v in check(got, x, Hkv, scale, mask, cap, slopes, heads).items()}, flush=True)


@pytest.mark.parametrize("seed", range(8))
def test_parity_of_drawn_shapes(env, seed):
    rng = np.random.Generator(np.random.PCG64(900 + seed))
    S = int(np.exp(rng.uniform(0, np.log(450))))
    Hkv = int(rng.choice([1, 2, 3, 8]))
    Hq, D, B = Hkv * int(rng.choice([1, 2, 4])), int(rng.choice([64, 128])), int(rng.integers(1, 4))
    kind = str(rng.choice(["causal", "full", "docs", "docs_full", "prefix", "pad", "window", "wild"]))
    cap, biased = float(rng.choice([0.0, 0.0, 15.0, 50.0])), bool(rng.integers(0, 2))
    print("attn_mod drawn", seed, B, S, Hq, Hkv, D, kind, cap, biased, flush=True)
    _, x = inputs(seed, B, S, Hq, Hkv, D, 1.5)
    mask = make_mask(kind, B, S, rng)
    slopes = slopes_of(Hq) if biased else None
    got = run_gpu(env, x, Hkv, D, 0.1, mask, cap, slopes, pad=8 * int(rng.integers(0, 3)))
    check(got, x, Hkv, 0.1, mask, cap, slopes)


@pytest.mark.parametrize("B,S,Hq,Hkv,D,kind,cap,biased,std", [
    (2, 700, 48, 16, 64, "prefix", 30.0, True, 2.0), (1, 1400, 56, 8, 128, "window", 0.0, False, 1.0),
    (1, 1400, 56, 8, 128, "causal", 20.0, False, 1.0)])
def test_tiles_of_two_sizes(env, B, S, Hq, Hkv, D, kind, cap, biased, std):
    """More than 512 workgroups of 128 queries, the last few of them in halves: 2 x 48 heads of 6 tiles, 56 of 11."""
    print("two sizes", B, S, Hq, Hkv, D, kind, cap, biased, std, flush=True)
    rng, x = inputs(500 + S, B, S, Hq, Hkv, D, std)
    mask, slopes = make_mask(kind, B, S, rng), slopes_of(Hq) if biased else None
    got = run_gpu(env, x, Hkv, D, 1 / math.sqrt(D), mask, cap, slopes)
    check(got, x, Hkv, 1 / math.sqrt(D), mask, cap, slopes, {(0, 0), (B - 1, Hkv - 1)})


def test_every_key_hidden(env):
    """No query sees anything: zeros, -inf, and nothing read from the scores."""
    rng, x = inputs(7, 2, 100, 2, 2, 64)
    mask = (np.full((2, 100), 50, np.int32), np.full((2, 100), 50, np.int32), 0)
    got = run_gpu(env, x, 2, 64, 0.125, mask, 0.0, None)
    assert np.all(got["LSE"] == -np.inf)
    for n in ("O", "dQ", "dK", "dV"):
        assert np.all(got[n] == 0), n


def test_gradient_by_differences(env):
    """Directional derivatives of sum(O dO) by central differences of the GPU's own forward.

    The step moves an input by e u with |u| of one FP16 value each (u = +-1 on Q); the difference quotient's
    error is its third-order term and the forward's rounding, 2^-11 |O| |dO| summed in quadrature / e."""
    B, S, Hq, Hkv, D, scale, cap = 1, 96, 2, 1, 64, 0.125, 8.0
    rng, x = inputs(11, B, S, Hq, Hkv, D)
    # on a grid of 2^-6, so that +-e is exact
    for n in "QKV":
        x[n] = (np.round(x[n].astype(np.float32) * 64) / 64).astype(np.float16)
    mask, slopes, e = make_mask("docs", B, S, rng), slopes_of(Hq), 1.0 / 16
    got = run_gpu(env, x, Hkv, D, scale, mask, cap, slopes)
    for n, g in (("Q", "dQ"), ("K", "dK"), ("V", "dV")):
        u = rng.choice([-1.0, 1.0], size=x[n].shape)
        f = []
        for sign in (1, -1):
            y = dict(x)
            y[n] = (x[n].astype(np.float64) + sign * e * u).astype(np.float16)
            o = run_gpu(env, y, Hkv, D, scale, mask, cap, slopes, bwd=False)["O"].astype(np.float64)
            f.append((o * x["dO"]).sum())
        num, ana = (f[0] - f[1]) / (2 * e), float((got[g].astype(np.float64) * u).sum())
        ref = []                                     # the exact function's quotient bounds the third-order term
        for sign in (1, -1):
            y = {m: x[m].astype(np.float64) for m in x}
            y[n] = y[n] + sign * e * u
            l, h = oracle.intervals(S, mask[0][0], None, True)
            ref.append(sum((oracle.attn_mod_head(y["Q"][0, :, a], y["K"][0, :, 0], y["V"][0, :, 0], scale, l, h, cap,
                                                 float(slopes[a]))["o"] * y["dO"][0, :, a]).sum() for a in range(Hq)))
        third = abs((ref[0] - ref[1]) / (2 * e) - ana)
        noise = 6 * 2 * H * math.sqrt(float((np.abs(got["O"].astype(np.float64) * x["dO"]) ** 2).sum())) / (2 * e)
        back = 6 * 2 * H * math.sqrt(float((got[g].astype(np.float64) ** 2).sum()))
        print(n, num, ana, third, noise, flush=True)
        assert abs(num - ana) <= third + noise + back
        assert third <= 0.05 * max(abs(ana), 5.0)


def test_results_repeat_bitwise(env):
    rng, x = inputs(13, 1, 600, 8, 2, 128)
    mask = make_mask("docs", 1, 600, rng)
    a = run_gpu(env, x, 2, 128, 0.09, mask, 30.0, slopes_of(8))
    b = run_gpu(env, x, 2, 128, 0.09, mask, 30.0, slopes_of(8))
    for n in a:
        assert np.array_equal(a[n].view(np.uint8), b[n].view(np.uint8)), n


BAD = [float("nan"), float("inf"), -float("inf")]


@pytest.mark.parametrize("B,S,Hq,Hkv,D,cap,biased", [(2, 200, 2, 1, 64, 0.0, False), (1, 700, 4, 4, 128, 20.0, True),
                                                    (1, 333, 16, 2, 128, 0.0, True), (6, 450, 64, 64, 64, 0.0, False)])
@pytest.mark.parametrize("bad", BAD, ids=str)
def test_non_finite_padding_takes_no_part(env, B, S, Hq, Hkv, D, cap, biased, bad):
    """What no query sees, and queries that see nothing, may hold anything."""
    print("non-finite padding", B, S, Hq, Hkv, D, cap, biased, bad, flush=True)
    rng, x = inputs(50 + S, B, S, Hq, Hkv, D)
    mask = make_mask("pad", B, S, rng)
    n = mask[1].max(1)
    for b in range(B):
        for name in ("Q", "K", "V", "dO"):
            x[name][b, n[b]:] = bad
    slopes = slopes_of(Hq) if biased else None
    got = run_gpu(env, x, Hkv, D, 0.1, mask, cap, slopes)
    check(got, x, Hkv, 0.1, mask, cap, slopes, None if B < 4 else {(0, 0), (1, 1), (B - 1, Hkv - 1)})
    for b in range(B):
        assert np.all(got["dK"][b, n[b]:] == 0) and np.all(got["dV"][b, n[b]:] == 0)


@pytest.mark.parametrize("B,S,Hq,Hkv,D,cap,biased,first,last", [
    (1, 300, 2, 2, 64, 0.0, False, 100, 140), (2, 600, 8, 2, 128, 30.0, False, 257, 259),
    (1, 1100, 16, 16, 128, 0.0, True, 40, 700), (3, 130, 3, 1, 64, 15.0, True, 0, 64)])
def test_non_finite_document_stays_to_itself(env, B, S, Hq, Hkv, D, cap, biased, first, last):
    """One document of NaN and infinities: the others have the results of their own values."""
    print("non-finite document", B, S, Hq, Hkv, D, cap, biased, first, last, flush=True)
    rng, x = inputs(60 + S, B, S, Hq, Hkv, D)
    lo = np.zeros((B, S), np.int32)
    lo[:, first:] = first
    lo[:, last:] = last
    mask, slopes = (lo, None, 1), slopes_of(Hq) if biased else None
    clean = {k: v.copy() for k, v in x.items()}
    for k in clean:
        clean[k][:, first:last] = 0
    want = run_gpu(env, clean, Hkv, D, 0.1, mask, cap, slopes)
    for name in ("Q", "K", "V", "dO"):
        x[name][:, first:last] = rng.choice(np.array(BAD + [1.0], np.float16), size=x[name][:, first:last].shape)
    x["Q"][:, first:last, :, 0] = np.nan
    got = run_gpu(env, x, Hkv, D, 0.1, mask, cap, slopes)
    assert np.isnan(got["O"][:, first:last].astype(np.float32)).all(-1).all()
    for name in got:                                 # compare the other documents
        if name == "LSE":
            got[name][:, :, first:last] = want[name][:, :, first:last]
        else:
            got[name][:, first:last] = want[name][:, first:last]
    check(got, clean, Hkv, 0.1, mask, cap, slopes)


def test_non_finite_value_reaches_those_who_see_it(env):
    """An infinite V element under a causal mask: that feature of the queries from there on, nothing else."""
    B, S, H_, D = 1, 150, 2, 64
    rng, x = inputs(71, B, S, H_, H_, D)
    x["V"][0, 70, 1, 5] = np.inf
    clean = dict(x, V=x["V"].copy())
    clean["V"][0, 70, 1, 5] = 0
    mask = (None, None, 1)
    got = run_gpu(env, x, H_, D, 0.1, mask, 0.0, None, bwd=False)
    want = run_gpu(env, clean, H_, D, 0.1, mask, 0.0, None, bwd=False)
    o = got["O"]
    assert np.all(np.isposinf(o[0, 70:, 1, 5]))
    o[0, 70:, 1, 5] = want["O"][0, 70:, 1, 5]
    check(got, clean, H_, 0.1, mask, 0.0, None)


@pytest.mark.parametrize("S,Hq,Hkv,D,cap,biased", [(333, 6, 2, 64, 0.0, True), (700, 8, 8, 128, 30.0, False)])
def test_separate_buffers(env, S, Hq, Hkv, D, cap, biased):
    """Q, K, V, O and the gradients in buffers of their own, every row stride different: the same bits as
    in the fused buffers.  One of the slopes is zero."""
    torch, lt = env
    rng, x = inputs(5 + S, 2, S, Hq, Hkv, D)
    mask = make_mask("prefix", 2, S, rng)
    slopes = slopes_of(Hq) if biased else None
    if biased:
        slopes[1] = 0.0
    want = run_gpu(env, x, Hkv, D, 0.11, mask, cap, slopes)
    check(want, x, Hkv, 0.11, mask, cap, slopes, {(1, Hkv - 1)})

    def rows(a, pad):
        t = torch.full((2 * S, a.shape[2] * D + pad), float("nan"), dtype=torch.float16, device="cuda")
        t[:, :a.shape[2] * D] = torch.from_numpy(a.reshape(2 * S, -1)).cuda()
        return t
    up = lambda a: None if a is None else torch.from_numpy(a).cuda()
    lo, hi, sl = up(mask[0]), up(mask[1]), up(slopes)
    Q, K, V, dO = rows(x["Q"], 8), rows(x["K"], 24), rows(x["V"], 24), rows(x["dO"], 40)
    O, dQ, dK, dV = torch.empty_like(dO), rows(0 * x["Q"], 56), rows(0 * x["K"], 72), rows(0 * x["V"], 72)
    LSE = torch.empty(2, Hq, S, device="cuda")
    lt.lt_attn_mod_fwd(Q, K, V, Q.stride(0), K.stride(0), O, O.stride(0), LSE, lo, hi, sl, cap, 2, S, Hq, Hkv, D, 0.11,
                       mask[2])
    n = lt.lt_attn_mod_bwd_workspace_size(2, S, Hq, Hkv, D, mask[2])
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    lt.lt_attn_mod_bwd(Q, K, V, Q.stride(0), K.stride(0), O, dO, O.stride(0), LSE, lo, hi, sl, cap, dQ, dK, dV,
                       dQ.stride(0), dK.stride(0), ws, n, 2, S, Hq, Hkv, D, 0.11, mask[2])
    for name, t, h in (("O", O, Hq), ("dQ", dQ, Hq), ("dK", dK, Hkv), ("dV", dV, Hkv)):
        got = t[:, :h * D].cpu().numpy()
        assert np.array_equal(got.view(np.uint16), want[name].reshape(2 * S, -1).view(np.uint16)), name
        if name != "O":
            assert bool(torch.isnan(t[:, h * D:]).all()), name
    assert np.array_equal(LSE.cpu().numpy(), want["LSE"])


@pytest.mark.parametrize("kind,cap,std", [("window", 50.0, 3.0), ("causal", 0.0, 3.0)])
def test_gradients_of_concentrated_softmax(env, kind, cap, std):
    """Scores of deviation 9, so that rows rest on a few keys and dP - D cancels.  dQ and dK carry two
    independent FP16 roundings (dS, the output), each at most 2^-11 / sqrt(3) of the value in the mean square:
    sqrt(2 / 3) 2^-11 = 4.0e-4 of the norm."""
    B, S, Hq, Hkv, D = 1, 768, 2, 2, 128
    rng, x = inputs(81, B, S, Hq, Hkv, D, std)
    mask, scale = make_mask(kind, B, S, rng), 1 / math.sqrt(D)
    got = run_gpu(env, x, Hkv, D, scale, mask, cap, None)
    l, h_ = oracle.intervals(S, None if mask[0] is None else mask[0][0], None, True)
    for h in range(Hq):
        r = oracle.attn_mod_head(*(x[n][0, :, h] for n in "QKV"), scale, l, h_, cap, 0.0, x["dO"][0, :, h])
        for n, m in (("dQ", "dq"), ("dK", "dk")):
            e = np.linalg.norm(got[n][0, :, h].astype(np.float64) - r[m]) / np.linalg.norm(r[m])
            print(kind, h, n, e, flush=True)
            assert e <= math.sqrt(2 / 3) * H


@pytest.mark.parametrize("S,D,cap", [(1, 64, 0.0), (40, 128, 0.0), (400, 64, 30.0), (600, 128, 0.0)])
def test_rows_of_one_key_have_no_gradient(env, S, D, cap):
    """Every query sees itself alone: P = 1 and D = dP, so dQ = dK = 0, however large the score.  V and dO are
    small integers, so that dP is exact in any order; then D = (p dP) / p is off by two roundings,
    |dP - D| <= 2^-23 |dP|, P by less than 2^-10, and dS gains half an FP16 step or subnormal step.  A D that
    took sum P for 1 would be off by the rounding of the LSE, 2^-20 for the largest scores here."""
    rng, x = inputs(70 + S, 1, S, 2, 1, D, 6.0)
    for n in ("V", "dO"):
        x[n] = rng.integers(-8, 9, size=x[n].shape).astype(np.float16)
    i = np.arange(S, dtype=np.int32)[None]
    scale = 1 / math.sqrt(D)
    got = run_gpu(env, x, 1, D, scale, (i, None, 1), cap, None)
    dk = np.zeros((S, D))
    for h in range(2):
        q, k, v, do = (x[n][0, :, m].astype(np.float64) for n, m in (("Q", h), ("K", 0), ("V", 0), ("dO", h)))
        ds = (2.0 ** -23 * np.abs((do * v).sum(1)) * (1 + 2.0 ** -10) * (1 + H) + SUB)[:, None] * scale
        assert np.array_equal(got["O"][0, :, h], x["V"][0, :, 0])
        assert np.all(np.abs(got["dQ"][0, :, h]) <= ds * np.abs(k) * (1 + 2 * H) + SUB)
        dk += ds * np.abs(q)
    assert np.all(np.abs(got["dK"][0, :, 0]) <= dk * (1 + 2 * H) + SUB)


@pytest.mark.parametrize("B,S,Hq,Hkv,D,kind,slope,cap", [
    (1, 1500, 2, 2, 128, "causal", 1.0, 0.0), (1, 1300, 4, 1, 64, "full", 0.5, 0.0), (2, 900, 4, 2, 128, "docs", 2.0, 20.0),
    (1, 2100, 2, 1, 64, "prefix", 0.3, 0.0), (1, 1000, 8, 1, 128, "window", 4.0, 0.0), (1, 1200, 2, 2, 64, "wild", 0.7, 0.0)])
def test_steep_bias(env, B, S, Hq, Hkv, D, kind, slope, cap):
    """Slopes that leave most pairs without weight, next to flat heads: tiles that end after their scores."""
    print("steep bias", B, S, Hq, Hkv, D, kind, slope, cap, flush=True)
    rng, x = inputs(90 + S, B, S, Hq, Hkv, D)
    mask = make_mask(kind, B, S, rng)
    slopes = np.array([slope * (1.0 if h % 2 == 0 else 0.01) for h in range(Hq)], np.float32)
    got = run_gpu(env, x, Hkv, D, 0.1, mask, cap, slopes)
    check(got, x, Hkv, 0.1, mask, cap, slopes, {(B - 1, Hkv - 1)})
    again = run_gpu(env, x, Hkv, D, 0.1, mask, cap, slopes)
    for n in got:
        assert np.array_equal(got[n].view(np.uint8), again[n].view(np.uint8)), n


def test_bias_that_grows_with_distance(env):
    """A negative slope: the farthest keys weigh most."""
    rng, x = inputs(99, 1, 800, 2, 1, 64)
    mask, slopes = make_mask("causal", 1, 800, rng), np.array([-0.5, 0.25], np.float32)
    got = run_gpu(env, x, 1, 64, 0.125, mask, 0.0, slopes)
    check(got, x, 1, 0.125, mask, 0.0, slopes)


def test_chunks_of_heads(env):
    """dS blocks of more than 8 GiB: the pairs of batch row and kv head go in chunks."""
    torch, lt = env
    B, S, Hq, Hkv, D = 33, 1024, 128, 16, 64
    rng = np.random.Generator(np.random.PCG64(3))
    mask = make_mask("docs_full", B, S, rng)
    n32 = S // 32
    assert lt.lt_attn_mod_bwd_workspace_size(B, S, Hq, Hkv, D, 0) < B * Hq * n32 * n32 * 2048   # chunks
    g = torch.Generator()
    g.manual_seed(5)
    x = {n: torch.randn(B, S, h, D, generator=g).half().numpy() for n, h in
         (("Q", Hq), ("K", Hkv), ("V", Hkv), ("dO", Hq))}
    got = run_gpu(env, x, Hkv, D, 0.125, mask, 0.0, None)
    check(got, x, Hkv, 0.125, mask, 0.0, None, {(0, 0), (16, 7), (16, 8), (32, 15)})
