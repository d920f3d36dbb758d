"""Performance cases of the packed-sequence operators.

Three operators that a training program calls next to the decoder layer when
its batches are packed (several documents laid end to end in one sequence):

  embed   the token embedding: row lookup with scaling, and its gradient, a sum
          over the tokens of each row of the table;
  qkn     RMSNorm of every query and key head with the rotary embedding in the
          same pass, at positions that restart with each document, and its
          gradient;
  attn    attention in which every query sees an interval of keys (a document,
          a prefix, a window, a padded batch), with scores that may be capped by
          a tanh and may get a bias linear in the distance, and its gradient.

A case with ``train`` is one pass forth and back, as a training step makes it;
without, the forward alone (evaluation).  With ``own`` false, ``run`` computes
the operators in elementary torch operations in 32 bits; with ``own`` true it
makes the library's calls.
"""

import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-6


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # the repository's smallest layer (its smoke check) on a packed batch:
        # launches and fixed costs
        dict(name="attn_tiny_docs", kind="attn", B=1, S=256, Hq=4, Hkv=4, D=64, mask="docs", docs=3, cap=0.0,
             alibi=False, train=True),
        # short padded encoder batch: full attention in each sequence, rows of
        # padding that see nothing
        dict(name="attn_pad_short", kind="attn", B=4, S=333, Hq=16, Hkv=16, D=64, mask="pad", docs=1, cap=0.0,
             alibi=False, train=True),
        # evaluation of a prefix model with capped scores, odd length
        dict(name="attn_prefix_eval", kind="attn", B=2, S=1237, Hq=32, Hkv=32, D=128, mask="prefix", docs=2,
             cap=50.0, alibi=False, train=False),
        # grouped queries (Qwen2.5-32B's heads), capped scores, a sliding window
        dict(name="attn_cap_gqa_2k", kind="attn", B=1, S=2048, Hq=40, Hkv=8, D=128, mask="window", docs=1, cap=50.0,
             alibi=False, train=True),
        # Baichuan2-13B's heads with the distance bias that model trains with
        dict(name="attn_alibi_4k", kind="attn", B=1, S=4096, Hq=40, Hkv=40, D=128, mask="causal", docs=1, cap=0.0,
             alibi=True, train=True),
        # LLaMA-2-70B's heads on a long packed batch
        dict(name="attn_docs_8k", kind="attn", B=1, S=8192, Hq=64, Hkv=8, D=128, mask="docs", docs=6, cap=0.0,
             alibi=False, train=True),
        # the smallest layer's heads
        dict(name="qkn_tiny", kind="qkn", B=1, S=256, Hq=4, Hkv=4, D=64, docs=3, train=True),
        # a packed micro-batch at Qwen2.5-32B's heads
        dict(name="qkn_4k", kind="qkn", B=1, S=4096, Hq=40, Hkv=8, D=128, docs=5, train=True),
        # evaluation of two sequences at LLaMA-2-70B's heads
        dict(name="qkn_70b_eval", kind="qkn", B=2, S=4096, Hq=64, Hkv=8, D=128, docs=1, train=False),
        # a small vocabulary and a short sequence
        dict(name="embed_tiny", kind="embed", T=256, V=1000, H=256, pad=True, scaled=True, train=True),
        # LLaMA-2-7B's table
        dict(name="embed_7b", kind="embed", T=4096, V=32000, H=4096, pad=False, scaled=False, train=True),
        # a large table (152k rows, Qwen2.5-32B's width) and an odd number of tokens
        dict(name="embed_152k", kind="embed", T=8191, V=152064, H=5120, pad=True, scaled=True, train=True),
    ]


def _log_int(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi + step)))
    return max(lo, min(hi, int(v) // step * step))


def _draw_once(rng):
    kind = rng.choice(("attn", "attn", "qkn", "embed"))
    if kind == "attn":
        Hkv = rng.choice((1, 2, 4, 8, 16, 32))
        S = _log_int(rng, 1, 8192)
        return dict(kind=kind, B=rng.choice((1, 1, 2, 3, 8)), S=S, Hq=Hkv * rng.choice((1, 1, 2, 5, 8)), Hkv=Hkv,
                    D=rng.choice((64, 128, 128)), mask=rng.choice(("causal", "docs", "docs", "prefix", "pad", "window")),
                    docs=min(S, rng.choice((1, 2, 3, 7, 20))), cap=rng.choice((0.0, 0.0, 20.0, 30.0, 50.0)),
                    alibi=rng.random() < 0.35, train=rng.random() < 0.7)
    if kind == "qkn":
        Hkv = rng.choice((1, 2, 4, 8, 32))
        S = _log_int(rng, 1, 8192)
        return dict(kind=kind, B=rng.choice((1, 1, 2, 3)), S=S, Hq=Hkv * rng.choice((1, 2, 5, 8)), Hkv=Hkv,
                    D=rng.choice((64, 96, 128, 128, 256)), docs=min(S, rng.choice((1, 2, 5, 9))),
                    train=rng.random() < 0.7)
    return dict(kind=kind, T=_log_int(rng, 1, 16384), V=_log_int(rng, 32, 152064), H=_log_int(rng, 64, 8192, 8),
                pad=rng.random() < 0.5, scaled=rng.random() < 0.5, train=rng.random() < 0.7)


def draw(rng):
    """One more case of the listed ranges that costs no more than the largest listed one of its kind."""
    big = {c["kind"]: c for c in listed()}          # the last listed case of a kind is its largest
    big["qkn"] = next(c for c in listed() if c["name"] == "qkn_4k")
    while True:
        c = _draw_once(rng)
        if work(c)["flops"] > work(big[c["kind"]])["flops"] or work(c)["bytes"] > work(big[c["kind"]])["bytes"]:
            continue
        if c["kind"] == "attn" and c["B"] * c["Hq"] * c["S"] ** 2 > 64 * 8192 ** 2:
            continue
        return c


# ---------------------------------------------------------------- masks and positions
def _lengths(c, row):
    """Document lengths of one batch row, by the case alone: uneven, a length of one among them."""
    S, n = c["S"], min(c["docs"], c["S"])
    rng = random.Random(f"{S} {n} {row}")
    cuts = sorted(rng.sample(range(1, S), n - 1)) if n > 1 else []
    return [b - a for a, b in zip([0] + cuts, cuts + [S])]


def _intervals(c):
    """(LO, HI) as [B, S] int32 arrays or None: query i sees the keys LO[i] <= j < HI[i], and of those
    only j <= i where the case is causal."""
    B, S, mask = c["B"], c["S"], c["mask"]
    if mask == "causal":
        return None, None
    i = np.arange(S)
    lo, hi = np.zeros((B, S), np.int32), np.zeros((B, S), np.int32)
    for b in range(B):
        if mask == "window":
            lo[b] = np.maximum(0, i - (S // 3 + 1) + 1)
            continue
        if mask == "pad":                            # this row's length; the rest is padding
            n = max(1, S - (S * b) // (2 * B) - (S > 8) * 5)
            lo[b], hi[b] = 0, np.where(i < n, n, 0)
            continue
        lens = _lengths(c, b)
        start = np.repeat(np.cumsum([0] + lens[:-1]), lens)
        lo[b] = start
        if mask == "prefix":                         # a third of each document is its prefix
            hi[b] = np.maximum(i + 1, start + np.repeat(np.array(lens) // 3, lens))
    return lo, (hi if mask in ("pad", "prefix") else None)


def _causal(c):
    return c["mask"] in ("causal", "docs", "window")


def _pairs(c):
    """(query, key) pairs that one head's mask keeps, over the batch."""
    B, S = c["B"], c["S"]
    lo, hi = _intervals(c)
    i = np.arange(S, dtype=np.int64)[None, :]
    lo = np.zeros((B, S), np.int64) if lo is None else lo.astype(np.int64)
    hi = np.full((B, S), S, np.int64) if hi is None else hi.astype(np.int64)
    if _causal(c):
        hi = np.minimum(hi, i + 1)
    return int(np.maximum(hi - lo, 0).sum())


def _positions(c):
    """Position of every token within its document, [B, S] int32."""
    return np.stack([np.concatenate([np.arange(n) for n in _lengths(c, b)])
                     for b in range(c["B"])]).astype(np.int32)


# ---------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _rnd(g, *shape, std=1.0, mean=0.0):
    return (torch.randn(*shape, generator=g, device=DEV) * std + mean).half()


def _slopes(n):
    """Slopes of the distance bias: a geometric series, for head counts that are no power of two the
    series of the next lower one, then every other slope of the next higher one."""
    def series(m):
        return [2.0 ** (-8.0 * (k + 1) / m) for k in range(m)]
    p = 1 << (n.bit_length() - 1)
    s = series(p)
    if p < n:
        s += series(2 * p)[0::2][:n - p]
    return s


def _inputs(c, seed):
    g = _gen(seed)
    if c["kind"] == "embed":
        T, V, H = c["T"], c["V"], c["H"]
        # token ids as text has them: the share of an id falls with its rank
        u = torch.rand(T, generator=g, device=DEV, dtype=torch.float64)
        ids = (torch.exp(u * math.log(V + 1.0)) - 1.0).long().clamp_(0, V - 1)
        if c["pad"]:
            ids[torch.rand(T, generator=g, device=DEV) < 0.05] = -1
        return dict(ids=ids, W=_rnd(g, V, H, std=0.02), dY=_rnd(g, T, H))
    B, S, Hq, Hkv, D = (c[n] for n in ("B", "S", "Hq", "Hkv", "D"))
    T, row = B * S, (Hq + 2 * Hkv) * D
    if c["kind"] == "qkn":
        a = (torch.arange(S, dtype=torch.float64, device=DEV)[:, None] *
             1000000.0 ** (-2.0 * torch.arange(D // 2, dtype=torch.float64, device=DEV) / D))
        return dict(QKV=_rnd(g, T, row, std=2.0), wq=_rnd(g, D, std=0.1, mean=1.0), wk=_rnd(g, D, std=0.1, mean=1.0),
                    dY=_rnd(g, T, (Hq + Hkv) * D), CS=torch.stack([torch.cos(a), torch.sin(a)], -1).float(),
                    POS=torch.from_numpy(_positions(c)).to(DEV).view(T))
    QKV = _rnd(g, T, row)
    if c["cap"] > 0:                                 # scores that reach the cap
        QKV[:, :(Hq + Hkv) * D] *= 3.0
    lo, hi = _intervals(c)
    up = lambda x: None if x is None else torch.from_numpy(x).to(DEV)
    return dict(QKV=QKV, dO=_rnd(g, T, Hq * D), LO=up(lo), HI=up(hi),
                slopes=torch.tensor(_slopes(Hq), device=DEV) if c["alibi"] else None)


def _empty(*shape, dtype=torch.float16):
    return torch.empty(*shape, dtype=dtype, device=DEV)


def prepare(case, seed):
    c = case
    s = dict(case=c, **_inputs(c, seed))
    if not own:
        return s
    from paper_2606_10415_amd import lt
    f32 = torch.float32
    if c["kind"] == "embed":
        s["Y"] = _empty(c["T"], c["H"])
        if c["train"]:
            s["dW"], s["n"] = _empty(c["V"], c["H"]), lt.lt_embed_bwd_workspace_size(c["T"], c["H"], c["V"])
    else:
        B, S, Hq, Hkv, D = (c[n] for n in ("B", "S", "Hq", "Hkv", "D"))
        T = B * S
        if c["kind"] == "qkn":
            s.update(Y=_empty(T, (Hq + Hkv) * D), RSTD=_empty(T, Hq + Hkv, dtype=f32))
            if c["train"]:
                s.update(dX=_empty(T, (Hq + Hkv) * D), dwq=_empty(D), dwk=_empty(D))
                s["n"] = lt.lt_qknorm_rope_bwd_workspace_size(B, S, Hq, Hkv, D)
        else:
            s.update(O=_empty(T, Hq * D), LSE=_empty(B, Hq, S, dtype=f32))
            if c["train"]:
                s["dQKV"] = _empty(T, (Hq + 2 * Hkv) * D)
                s["n"] = lt.lt_attn_mod_bwd_workspace_size(B, S, Hq, Hkv, D, int(_causal(c)))
    if c["train"]:
        s["ws"] = _empty(max(s["n"], 256), dtype=torch.uint8)
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    return globals()[("_own_" if own else "_plain_") + s["case"]["kind"]](s)


def _scale(c):
    return math.sqrt(c["H"]) if c["scaled"] else 1.0


def _own_embed(s):
    from paper_2606_10415_amd import lt
    c = s["case"]
    T, V, H = c["T"], c["V"], c["H"]
    lt.lt_embed_fwd(s["ids"], s["W"], H, _scale(c), s["Y"], H, T, H, V)
    if not c["train"]:
        return [s["Y"]]
    lt.lt_embed_bwd(s["ids"], s["dY"], H, _scale(c), 0, s["dW"], H, s["ws"], s["n"], T, H, V)
    return [s["Y"], s["dW"]]


def _own_qkn(s):
    from paper_2606_10415_amd import lt
    c = s["case"]
    B, S, Hq, Hkv, D = (c[n] for n in ("B", "S", "Hq", "Hkv", "D"))
    row, qk = (Hq + 2 * Hkv) * D, (Hq + Hkv) * D
    lt.lt_qknorm_rope_fwd(s["QKV"], row, s["wq"], s["wk"], s["CS"], S, s["POS"], s["Y"], qk, s["RSTD"], B, S, Hq,
                          Hkv, D, EPS)
    if not c["train"]:
        return [s["Y"], s["RSTD"]]
    lt.lt_qknorm_rope_bwd(s["dY"], qk, s["QKV"], row, s["wq"], s["wk"], s["RSTD"], s["CS"], S, s["POS"], s["dX"], qk,
                          s["dwq"], s["dwk"], s["ws"], s["n"], B, S, Hq, Hkv, D)
    return [s["Y"], s["RSTD"], s["dX"], s["dwq"], s["dwk"]]


def _own_attn(s):
    from paper_2606_10415_amd import lt
    c = s["case"]
    B, S, Hq, Hkv, D = (c[n] for n in ("B", "S", "Hq", "Hkv", "D"))
    row, hd, scale, ca = (Hq + 2 * Hkv) * D, Hq * D, 1.0 / math.sqrt(D), int(_causal(c))

    def heads(t):
        p = t.data_ptr()
        return p, p + 2 * hd, p + 2 * (hd + Hkv * D)

    q, k, v = heads(s["QKV"])
    lt.lt_attn_mod_fwd(q, k, v, row, row, s["O"], hd, s["LSE"], s["LO"], s["HI"], s["slopes"], c["cap"], B, S, Hq,
                       Hkv, D, scale, ca)
    if not c["train"]:
        return [s["O"], s["LSE"]]
    dq, dk, dv = heads(s["dQKV"])
    lt.lt_attn_mod_bwd(q, k, v, row, row, s["O"], s["dO"], hd, s["LSE"], s["LO"], s["HI"], s["slopes"], c["cap"], dq,
                       dk, dv, row, row, s["ws"], s["n"], B, S, Hq, Hkv, D, scale, ca)
    return [s["O"], s["LSE"], s["dQKV"]]


# ---- the plain forms: elementary operations in 32 bits
def _plain_embed(s):
    c = s["case"]
    ids, scale = s["ids"], _scale(c)
    seen = (ids >= 0) & (ids < c["V"])
    rows = torch.where(seen, ids, torch.zeros_like(ids))
    Y = (s["W"][rows].float() * scale * seen[:, None]).half()
    if not c["train"]:
        return [Y]
    dW = torch.zeros(c["V"], c["H"], dtype=torch.float32, device=DEV)
    dW.index_add_(0, rows, s["dY"].float() * seen[:, None])
    return [Y, (dW * scale).half()]


def _rot(x, co, si):
    h = x.shape[-1] // 2
    a, b = x[..., :h], x[..., h:]
    return torch.cat([a * co - b * si, b * co + a * si], -1)


def _plain_qkn(s):
    c = s["case"]
    B, S, Hq, Hkv, D = (c[n] for n in ("B", "S", "Hq", "Hkv", "D"))
    T, n = B * S, Hq + Hkv
    x = s["QKV"][:, :n * D].float().view(T, n, D)
    w = torch.cat([s["wq"].float().expand(Hq, D), s["wk"].float().expand(Hkv, D)])
    cs = s["CS"][s["POS"].long()]
    co, si = cs[:, None, :, 0], cs[:, None, :, 1]
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
    Y = _rot(x * r * w, co, si).half().view(T, n * D)
    if not c["train"]:
        return [Y, r.view(T, n)]
    g = _rot(s["dY"].float().view(T, n, D), co, -si)
    gw = g * w
    dX = r * gw - r * r * r * x * (gw * x).mean(-1, keepdim=True)
    dw = (g * x * r).sum(0)
    return [Y, r.view(T, n), dX.half().view(T, n * D), dw[:Hq].sum(0).half(), dw[Hq:].sum(0).half()]


def _visible(c, lo, hi, b):
    """[S, S] truth values of one batch row: which keys (columns) each query (row) sees."""
    S = c["S"]
    j = torch.arange(S, device=DEV)[None, :]
    ok = torch.ones(S, S, dtype=torch.bool, device=DEV)
    if lo is not None:
        ok &= j >= lo[b][:, None]
    if hi is not None:
        ok &= j < hi[b][:, None]
    if _causal(c):
        ok &= j <= j.t()
    return ok


def _plain_attn(s):
    c = s["case"]
    B, S, Hq, Hkv, D = (c[n] for n in ("B", "S", "Hq", "Hkv", "D"))
    G, scale, cap = Hq // Hkv, 1.0 / math.sqrt(D), c["cap"]
    x = s["QKV"].view(B, S, Hq + 2 * Hkv, D)
    O = torch.empty(B, S, Hq, D, dtype=torch.float16, device=DEV)
    LSE = torch.empty(B, Hq, S, dtype=torch.float32, device=DEV)
    dx = torch.empty_like(x) if c["train"] else None
    pos = torch.arange(S, device=DEV, dtype=torch.float32)
    dist = (pos[:, None] - pos[None, :]).abs() if c["alibi"] else None
    step = max(1, 2 ** 28 // (G * S * S))            # kv heads at a time
    for b in range(B):
        see = _visible(c, s["LO"], s["HI"], b)
        for k0 in range(0, Hkv, step):
            nk = min(step, Hkv - k0)
            nq = nk * G
            q = x[b, :, k0 * G:k0 * G + nq].float().transpose(0, 1).contiguous()
            k, v = (x[b, :, o + k0:o + k0 + nk].float().transpose(0, 1).repeat_interleave(G, 0).contiguous()
                    for o in (Hq, Hq + Hkv))
            z = torch.bmm(q, k.transpose(1, 2).contiguous()) * scale
            if cap > 0:
                t = torch.tanh(z / cap)
                z = t * cap
            if dist is not None:
                z = z - s["slopes"][k0 * G:k0 * G + nq, None, None] * dist
            z = z.masked_fill_(~see, -math.inf)
            m = z.amax(-1, keepdim=True)
            m = torch.where(m == -math.inf, torch.zeros_like(m), m)
            z = torch.exp(z - m)
            l = z.sum(-1, keepdim=True)
            p = z / torch.where(l > 0, l, torch.ones_like(l))
            o = torch.bmm(p, v)
            O[b, :, k0 * G:k0 * G + nq] = o.transpose(0, 1).half()
            LSE[b, k0 * G:k0 * G + nq] = (m + torch.log(l)).squeeze(-1)
            if dx is None:
                continue
            g = s["dO"].view(B, S, Hq, D)[b, :, k0 * G:k0 * G + nq].float().transpose(0, 1).contiguous()
            ds = torch.bmm(g, v.transpose(1, 2).contiguous())
            ds = p * (ds - (g * o).sum(-1, keepdim=True)) * scale
            if cap > 0:
                ds = ds * (1.0 - t * t)
            dq = torch.bmm(ds, k)
            dk = torch.bmm(ds.transpose(1, 2).contiguous(), q).view(nk, G, S, D).sum(1)
            dv = torch.bmm(p.transpose(1, 2).contiguous(), g).view(nk, G, S, D).sum(1)
            dx[b, :, k0 * G:k0 * G + nq] = dq.transpose(0, 1).half()
            dx[b, :, Hq + k0:Hq + k0 + nk] = dk.transpose(0, 1).half()
            dx[b, :, Hq + Hkv + k0:Hq + Hkv + k0 + nk] = dv.transpose(0, 1).half()
    T = B * S
    return [O.view(T, Hq * D), LSE] + ([dx.view(T, -1)] if c["train"] else [])


# ---------------------------------------------------------------- its cost
def work(c):
    if c["kind"] == "embed":
        T, V, H = c["T"], c["V"], c["H"]
        # the rows of the table that the tokens name are at most T; of ids distributed as _inputs draws
        # them, the expected number of different ones
        rank = np.arange(1, V + 1, dtype=np.float64)
        share = (np.log(rank + 1) - np.log(rank)) / math.log(V + 1.0)
        rows = float((1.0 - (1.0 - share) ** (T * (0.95 if c["pad"] else 1.0))).sum())
        by = 8 * T + 2 * H * (rows + T) + (2 * H * (T + V) if c["train"] else 0)
        return dict(bytes=int(by), flops=T * H * (2 if c["train"] else 1))
    B, S, Hq, Hkv, D = (c[n] for n in ("B", "S", "Hq", "Hkv", "D"))
    T, n = B * S, Hq + Hkv
    if c["kind"] == "qkn":
        by = T * n * (4 * D + 4) + 4 * T + 4 * max(_lengths(c, 0)) * D
        if c["train"]:
            by += T * n * 4 * D                      # dY in, dX out
        return dict(bytes=by + 4 * D, flops=T * n * D * (20 if c["train"] else 7))
    p = Hq * _pairs(c)
    by = 2 * T * ((Hq + 2 * Hkv) * D + Hq * D) + 4 * T * Hq
    if c["train"]:
        by += 2 * T * ((Hq + 2 * Hkv) * D + Hq * D)
    # per pair: q.k and p.v forth; dp, dv, dq and dk back
    return dict(bytes=by, flops=(12 if c["train"] else 4) * D * p)


# ---------------------------------------------------------------- 64-bit results
def exact(case, seed):
    c, x = case, _inputs(case, seed)
    return globals()["_exact_" + c["kind"]](c, x)


def _exact_embed(c, x):
    V, H, ids, scale = c["V"], c["H"], x["ids"], _scale(c)
    Y = torch.zeros(c["T"], H, dtype=torch.float64, device=DEV)
    good = torch.nonzero((ids >= 0) & (ids < V)).flatten()
    Y[good] = x["W"].index_select(0, ids[good]).double() * scale
    if not c["train"]:
        return [Y]
    # tokens in the order of their rows, then the difference of running sums at the rows' ends
    order = good[torch.sort(ids[good], stable=True).indices]
    run = torch.cumsum(x["dY"].index_select(0, order).double(), 0)
    last = torch.searchsorted(ids[order].contiguous(), torch.arange(V, device=DEV), right=True)
    run = torch.cat([torch.zeros(1, H, dtype=torch.float64, device=DEV), run])
    ends = run[last]
    dW = ends.clone()
    dW[1:] -= ends[:-1]
    return [Y, dW * scale]


def _exact_qkn(c, x):
    B, S, Hq, Hkv, D = (c[n] for n in ("B", "S", "Hq", "Hkv", "D"))
    T, h = B * S, D // 2
    theta = 1000000.0 ** (-torch.arange(h, dtype=torch.float64, device=DEV) * 2.0 / D)
    turn = torch.polar(torch.ones(T, h, dtype=torch.float64, device=DEV), x["POS"].double()[:, None] * theta)
    outs, grads, dws = [], [], []
    rstd = torch.empty(T, Hq + Hkv, dtype=torch.float64, device=DEV)
    for n in range(Hq + Hkv):
        w = (x["wq"] if n < Hq else x["wk"]).double()
        v = x["QKV"][:, n * D:(n + 1) * D].double()
        r = (v.square().mean(1) + EPS).rsqrt()
        rstd[:, n] = r
        u = v * r[:, None] * w
        y = torch.complex(u[:, :h].contiguous(), u[:, h:].contiguous()) * turn
        outs.append(torch.cat([y.real, y.imag], 1))
        if c["train"]:
            d = x["dY"][:, n * D:(n + 1) * D].double()
            d = torch.complex(d[:, :h].contiguous(), d[:, h:].contiguous()) * turn.conj()
            d = torch.cat([d.real, d.imag], 1)
            unit = v * r[:, None]
            dws.append((d * unit).sum(0))
            d = d * w
            grads.append(r[:, None] * (d - unit * (d * unit).mean(1, keepdim=True)))
    if not c["train"]:
        return [torch.cat(outs, 1), rstd]
    return [torch.cat(outs, 1), rstd, torch.cat(grads, 1), sum(dws[:Hq]), sum(dws[Hq:])]


def _exact_attn(c, x):
    B, S, Hq, Hkv, D = (c[n] for n in ("B", "S", "Hq", "Hkv", "D"))
    if B * Hq * S * S > 64 * 8192 ** 2:
        return None
    G, cap = Hq // Hkv, c["cap"]
    X = x["QKV"].double().view(B, S, Hq + 2 * Hkv, D)
    O = torch.zeros(B, S, Hq, D, dtype=torch.float64, device=DEV)
    LSE = torch.full((B, Hq, S), -math.inf, dtype=torch.float64, device=DEV)
    dX = torch.zeros_like(X) if c["train"] else None
    i = torch.arange(S, device=DEV)
    for b in range(B):
        lo = x["LO"][b].long() if x["LO"] is not None else torch.zeros_like(i)
        hi = x["HI"][b].long() if x["HI"] is not None else torch.full_like(i, S)
        if _causal(c):
            hi = torch.minimum(hi, i + 1)
        hidden = (i[None, :] < lo[:, None]) | (i[None, :] >= hi[:, None])
        rows = torch.nonzero(lo < hi).flatten()      # queries that see something
        hidden = hidden[rows]
        for h in range(Hq):
            kv = h // G
            q, k, v = X[b, rows, h], X[b, :, Hq + kv].contiguous(), X[b, :, Hq + Hkv + kv].contiguous()
            raw = q @ k.t().contiguous() / math.sqrt(D)
            s = torch.tanh(raw / cap) * cap if cap > 0 else raw
            slope = torch.ones_like(s)
            if cap > 0:
                slope = 1.0 / torch.cosh(raw / cap).square()
            if x["slopes"] is not None:
                s = s - x["slopes"][h].double() * (rows[:, None] - i[None, :]).abs()
            s = s.masked_fill(hidden, -math.inf)
            lse = torch.logsumexp(s, 1)
            p = torch.exp(s - lse[:, None])
            O[b, rows, h] = p @ v
            LSE[b, h, rows] = lse
            if dX is None:
                continue
            g = x["dO"].view(B, S, Hq, D)[b, rows, h].double()
            dp = g @ v.t().contiguous()
            ds = p * (dp - (p * dp).sum(1, keepdim=True)) * slope / math.sqrt(D)
            dX[b, rows, h] = ds @ k
            dX[b, :, Hq + kv] += ds.t().contiguous() @ q
            dX[b, :, Hq + Hkv + kv] += p.t().contiguous() @ g
    T = B * S
    return [O.view(T, Hq * D), LSE] + ([dX.view(T, -1)] if c["train"] else [])
