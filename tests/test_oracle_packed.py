"""Pins of the packed-sequence oracle: finite differences, brute force over
single elements, and agreement with the oracles it generalises."""

import math

import numpy as np
import pytest

import oracle


def _rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def _numeric(f, x, eps=1e-6):
    g = np.zeros_like(x)
    for idx in np.ndindex(*x.shape):
        old = x[idx]
        x[idx] = old + eps
        hi = f()
        x[idx] = old - eps
        lo = f()
        x[idx] = old
        g[idx] = (hi - lo) / (2 * eps)
    return g


MASKS = {
    "causal": (None, None, True),
    "docs": ([0, 0, 0, 3, 3, 5, 5], None, True),
    "prefix": ([0, 0, 0, 0, 4, 4, 4], [3, 3, 3, 4, 6, 6, 7], False),
    "pad": (None, [4, 4, 4, 4, 0, 0, 0], False),
    "beyond": ([-5, 9, 2, 0, 0, 6, 3], [99, 2, 1, 3, -1, 7, 99], False),
}


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("cap,slope", [(0.0, 0.0), (1.5, 0.0), (0.0, 0.3), (1.5, 0.3)])
def test_attention_gradient_by_differences(mask, cap, slope):
    lo, hi, causal = MASKS[mask]
    S, D, scale = 7, 4, 0.6
    g = _rng(1)
    q, k, v, do = (g.standard_normal((S, D)) for _ in range(4))
    lo, hi = oracle.intervals(S, lo, hi, causal)
    r = oracle.attn_mod_head(q, k, v, scale, lo, hi, cap, slope, do)
    f = lambda: float((oracle.attn_mod_head(q, k, v, scale, lo, hi, cap, slope)["o"] * do).sum())
    for name, x in (("dq", q), ("dk", k), ("dv", v)):
        assert np.max(np.abs(r[name] - _numeric(f, x))) < 1e-7, name


@pytest.mark.parametrize("mask", MASKS)
def test_attention_by_single_elements(mask):
    lo, hi, causal = MASKS[mask]
    S, D, scale, cap, slope = 7, 4, 0.6, 2.0, 0.1
    g = _rng(2)
    q, k, v = (g.standard_normal((S, D)) for _ in range(3))
    l, h = oracle.intervals(S, lo, hi, causal)
    r = oracle.attn_mod_head(q, k, v, scale, l, h, cap, slope)
    for i in range(S):
        seen = [j for j in range(S) if (lo is None or j >= lo[i]) and (hi is None or j < hi[i]) and
                not (causal and j > i)]
        if not seen:
            assert np.all(r["o"][i] == 0) and r["lse"][i] == -math.inf
            continue
        z = [cap * math.tanh(scale * sum(q[i][f] * k[j][f] for f in range(D)) / cap) - slope * abs(i - j)
             for j in seen]
        tot = sum(math.exp(x) for x in z)
        assert abs(r["lse"][i] - math.log(tot)) < 1e-12
        for f in range(D):
            assert abs(r["o"][i][f] - sum(math.exp(x) * v[j][f] for x, j in zip(z, seen)) / tot) < 1e-12


def test_attention_without_modification_is_the_plain_one():
    g = _rng(3)
    q, k, v, do = (g.standard_normal((9, 8)) for _ in range(4))
    r = oracle.attn_mod_head(q, k, v, 0.3, *oracle.intervals(9, causal=True), do=do)
    o, lse, _ = oracle.attn_head_fwd(q, k, v, 0.3)
    b = oracle.attn_head_bwd(q, k, v, do, 0.3)
    for x, y in ((r["o"], o), (r["lse"], lse), (r["dq"], b["dq"]), (r["dk"], b["dk"]), (r["dv"], b["dv"])):
        assert np.max(np.abs(x - y)) < 1e-13


def test_nan_in_places_that_nobody_sees_takes_no_part():
    g = _rng(4)
    q, k, v, do = (g.standard_normal((6, 4)) for _ in range(4))
    lo, hi = oracle.intervals(6, None, [4, 4, 4, 4, 0, 0])
    a = oracle.attn_mod_head(q, k, v, 0.5, lo, hi, do=do)
    for x in (q, k, v, do):
        x[4:] = np.nan
    b = oracle.attn_mod_head(q, k, v, 0.5, lo, hi, do=do)
    for name in ("o", "dq", "dk", "dv"):
        assert np.array_equal(a[name], b[name]), name


def test_qknorm_gradient_by_differences():
    g = _rng(5)
    T, hq, n, D = 3, 2, 3, 8
    x, dy = g.standard_normal((T, n, D)), g.standard_normal((T, n, D))
    wq, wk = 1 + 0.1 * g.standard_normal(D), 1 + 0.1 * g.standard_normal(D)
    pos = [0, 5, 1000]
    _, _, dx, dwq, dwk = oracle.qknorm_rope(x, wq, wk, hq, pos, 100.0, 1e-3, dy)
    f = lambda: float((oracle.qknorm_rope(x, wq, wk, hq, pos, 100.0, 1e-3)[0] * dy).sum())
    for a, b in ((dx, x), (dwq, wq), (dwk, wk)):
        assert np.max(np.abs(a - _numeric(f, b))) < 1e-7


def test_qknorm_is_the_norm_then_the_rotation():
    g = _rng(6)
    B, S, n, D = 2, 5, 3, 16
    x = g.standard_normal((B * S, n, D))
    w = 1 + 0.1 * g.standard_normal(D)
    y, r = oracle.qknorm_rope(x, w, w, 2, np.tile(np.arange(S), B), 10000.0, 1e-6)
    u, rstd = oracle.rmsnorm_fwd(x.reshape(-1, D), w, 1e-6)
    assert np.max(np.abs(r.reshape(-1) - rstd)) < 1e-13
    assert np.max(np.abs(y.reshape(B, S, n, D) - oracle.rope_fwd(u.reshape(B, S, n, D), 10000.0))) < 1e-13


def test_embedding_gradient_by_differences():
    g = _rng(7)
    w, dy = g.standard_normal((5, 3)), g.standard_normal((6, 3))
    ids = [2, -1, 4, 2, 7, 0]
    f = lambda: float((oracle.embed_fwd(ids, w, 1.7) * dy).sum())
    assert np.max(np.abs(oracle.embed_bwd(ids, dy, 1.7, 5) - _numeric(f, w))) < 1e-8
    assert np.all(oracle.embed_fwd(ids, w, 1.7)[[1, 4]] == 0)
