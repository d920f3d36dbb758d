"""The packed-sequence operators as the layers use them: DecoderLayer and Stage with a masked, capped or
biased attention, QK norm and a token embedding, against a float64 autograd of the same layer on the CPU; HIP
graphs; other streams.

Bars: as the other chained-layer tests (FP16 intermediates on the GPU, float64 in the reference): relative
Frobenius error 5e-3 for one layer, 1e-2 for a stage of several.
"""

import math
from dataclasses import replace

import numpy as np
import pytest

from paper_2606_10415_amd import packing
from paper_2606_10415_amd.synth import NormInputs, Workload, layer_inputs, normal_f16
from conftest import rel_f

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available(), "GPU tests need a ROCm device"
    return t


def norms(w, seed, qk=True, rope=10000.0):
    one = lambda s, n: (1.0 + normal_f16(s, (n,), 0.1).astype(np.float32)).astype(np.float16)
    return NormInputs(one(seed, w.H), one(seed + 1, w.H), 1e-5, rope, None,
                      one(seed + 2, w.D) if qk else None, one(seed + 3, w.D) if qk else None)


def reference_layer(torch, w, X, p, norm, att):
    """One layer in float64 torch operations (differentiable); X [T, H], p and norm leaf tensors."""
    B, S, D = w.B, w.S, w.D
    T = B * S

    def rms(x, wt, eps):
        return wt * x * (x.square().mean(-1, keepdim=True) + eps).rsqrt()

    x = rms(X, norm["wn1"], norm["eps"]) if norm else X
    qkv = (x @ p["Wqkv"].t()).view(B, S, -1, D)
    q, k, v = qkv[:, :, :w.Hq], qkv[:, :, w.Hq:w.Hq + w.Hkv], qkv[:, :, w.Hq + w.Hkv:]
    if norm and norm.get("wq") is not None:
        q, k = rms(q, norm["wq"], norm["eps"]), rms(k, norm["wk"], norm["eps"])
    if norm and norm["base"] is not None:
        pos = torch.arange(S).expand(B, S) if att is None or att.pos is None or norm.get("wq") is None \
            else torch.from_numpy(att.pos)
        a = pos.double()[..., None] * norm["base"] ** (-2.0 * torch.arange(D // 2).double() / D)
        c, s = a.cos()[:, :, None], a.sin()[:, :, None]
        rot = lambda z: torch.cat([z[..., :D // 2] * c - z[..., D // 2:] * s, z[..., D // 2:] * c + z[..., :D // 2] * s], -1)
        q, k = rot(q), rot(k)
    G = w.Hq // w.Hkv
    z = torch.einsum("bihd,bjhd->bhij", q, k.repeat_interleave(G, 2)) / math.sqrt(D)
    i, j = torch.arange(S)[:, None], torch.arange(S)[None, :]
    see = torch.ones(B, S, S, dtype=torch.bool)
    if att is None or att.causal:
        see &= j <= i
    if att is not None:
        if att.cap:
            z = att.cap * torch.tanh(z / att.cap)
        if att.slopes is not None:
            z = z - torch.from_numpy(att.slopes).double()[None, :, None, None] * (i - j).abs()
        if att.lo is not None:
            see &= j >= torch.from_numpy(att.lo)[:, :, None]
        if att.hi is not None:
            see &= j < torch.from_numpy(att.hi)[:, :, None]
    z = z.masked_fill(~see[:, None], -1e30)
    pr = torch.softmax(z, -1) * see[:, None]
    o = torch.einsum("bhij,bjhd->bihd", pr, v.repeat_interleave(G, 2)).reshape(T, -1)
    H1 = X + o @ p["Wo"].t()
    h = rms(H1, norm["wn2"], norm["eps"]) if norm else H1
    gu = h @ p["Wgu"].t()
    A = torch.nn.functional.silu(gu[:, :w.F]) * gu[:, w.F:]
    return H1 + A @ p["Wd"].t()


def leaves(torch, arrays):
    return {k: torch.from_numpy(v.astype(np.float64)).requires_grad_() for k, v in arrays.items()}


def norm_leaves(torch, n):
    if n is None:
        return None
    d = leaves(torch, {k: getattr(n, k) for k in ("wn1", "wn2", "wq", "wk") if getattr(n, k) is not None})
    return dict(d, eps=n.eps, base=n.rope_base)


W = Workload("packed", 20, B=2, S=168, H=256, Hq=4, Hkv=2, D=64, F=344)


def attention(kind):
    if kind == "docs+cap":
        return packing.documents([[50, 1, 90], [168]], 168, cap=20.0)
    if kind == "prefix":
        return packing.documents([[100, 68], [33, 77]], 168, prefixes=[[30, 68], [0, 10]])
    if kind == "alibi":
        return packing.Attention(slopes=packing.alibi_slopes(4))
    if kind == "padded":
        return packing.padded([168, 101], 168)
    return packing.window(2, 168, 37)


@pytest.mark.parametrize("kind,qk,rope", [("docs+cap", True, 10000.0), ("prefix", True, 500000.0),
                                         ("alibi", False, None), ("padded", False, 10000.0), ("window", True, 10000.0),
                                         (None, True, 10000.0)])
def test_layer_against_autograd(torch, kind, qk, rope):
    from paper_2606_10415_amd.layer import DecoderLayer
    print("packed layer", kind, qk, rope, flush=True)
    p, n = layer_inputs(W), norms(W, 700, qk, rope)
    att = attention(kind) if kind else None
    L = DecoderLayer(W, p, norm=n, attention=att)
    L.step()
    torch.cuda.synchronize()
    ref, rn = leaves(torch, p), norm_leaves(torch, n)
    Y = reference_layer(torch, W, ref["X"], ref, rn, att)
    (Y * ref["dY"].detach()).sum().backward()
    c = lambda t: t.float().cpu().numpy()
    err = {"Y": rel_f(c(L.Y), Y.detach().numpy())}
    for name, leaf in [("dX", ref["X"])] + [("d" + k, ref[k]) for k in ("Wqkv", "Wo", "Wgu", "Wd")] + \
            [("dWn1", rn["wn1"]), ("dWn2", rn["wn2"])] + ([("dWq", rn["wq"]), ("dWk", rn["wk"])] if qk else []):
        err[name] = rel_f(c(getattr(L, name)), leaf.grad.numpy())
    print("  errors: " + ", ".join(f"{k} {v:.3e}" for k, v in err.items()), flush=True)
    for k, v in err.items():
        assert v <= 5e-3, k


@pytest.mark.parametrize("normed", [False, True], ids=["two micro-batches", "normed"])
def test_stage_with_embedding_against_autograd(torch, normed):
    """Token ids in, table gradient out, through two layers of packed attention."""
    from paper_2606_10415_amd.stage import Stage
    w = Workload("packed-stage", 21, B=1, S=200, H=128, Hq=4, Hkv=1, D=64, F=264)
    V, L, scale = 300, 2, math.sqrt(128)
    att = packing.documents([[70, 100, 20]], 200, cap=15.0)      # ten tokens of padding
    n = norms(w, 800) if normed else None
    qkv = (w.Hq + 2 * w.Hkv) * w.D
    weights = [{"Wqkv": normal_f16(900 + 10 * l, (qkv, w.H), 0.02), "Wo": normal_f16(901 + 10 * l, (w.H, w.Hq * w.D), 0.02),
                "Wgu": normal_f16(902 + 10 * l, (2 * w.F, w.H), 0.02), "Wd": normal_f16(903 + 10 * l, (w.H, w.F), 0.02)}
               for l in range(L)]
    table = normal_f16(950, (V, w.H), 0.1)
    rng = np.random.Generator(np.random.PCG64(5))
    ids = [np.minimum(rng.geometric(0.03, size=w.T) - 1, V - 1).astype(np.int64) for _ in range(1 if normed else 2)]
    for x in ids:
        x[190:] = -1
    dys = [normal_f16(960 + m, (w.T, w.H)) for m in range(len(ids))]
    for dy in dys:
        dy[190:] = 0
    res = {}
    for act in ("full", "ckpt"):
        st = Stage(w, L, act=act, weights=weights, norm=n, attention=att, embed=table, embed_scale=scale)
        for rep in range(2):                                     # the second step overwrites the first
            st.step([torch.from_numpy(x).cuda() for x in ids], [torch.from_numpy(y).cuda() for y in dys])
        torch.cuda.synchronize()
        res[act] = [st.dWe.cpu().numpy()] + [getattr(l, k).cpu().numpy() for l in st.layers
                                             for k in ("dWqkv", "dWo", "dWgu", "dWd")]
    for a, b in zip(res["full"], res["ckpt"]):
        assert np.array_equal(a.view(np.uint16), b.view(np.uint16))
    te = torch.from_numpy(table.astype(np.float64)).requires_grad_()
    lw, rn = [leaves(torch, p) for p in weights], norm_leaves(torch, n)
    for x, dy in zip(ids, dys):
        x = torch.from_numpy(x)
        h = te[x.clamp(min=0)] * (x >= 0)[:, None] * scale
        for p in lw:
            h = reference_layer(torch, w, h, p, rn, att)
        (h * torch.from_numpy(dy.astype(np.float64))).sum().backward()
    err = {"dWe": rel_f(res["full"][0], te.grad.numpy())}
    for i, (l, k) in enumerate((l, k) for l in range(L) for k in ("Wqkv", "Wo", "Wgu", "Wd")):
        err[f"d{k}{l}"] = rel_f(res["full"][1 + i], lw[l][k].grad.numpy())
    print("  errors: " + ", ".join(f"{k} {v:.3e}" for k, v in err.items()), flush=True)
    assert max(err.values()) <= 1e-2, err
    absent = np.setdiff1d(np.arange(V), np.concatenate(ids))
    assert len(absent) and np.all(res["full"][0][absent] == 0)
    with pytest.raises(ValueError):
        st.forward(torch.zeros(w.T, dtype=torch.int32, device="cuda"))


def test_stage_refusals(torch):
    from paper_2606_10415_amd.layer import DecoderLayer
    from paper_2606_10415_amd.stage import Stage
    p = layer_inputs(W)
    with pytest.raises(ValueError):
        DecoderLayer(W, p, attention=packing.window(2, 100, 5))                       # another length
    with pytest.raises(ValueError):
        DecoderLayer(W, p, attention=packing.Attention(slopes=packing.alibi_slopes(5)))
    with pytest.raises(ValueError):
        DecoderLayer(W, p, norm=norms(W, 1, True, None))                              # QK norm without a rotary base
    n = norms(W, 1)
    for bad in (replace(n, wk=None), replace(n, wq=None), replace(n, wk=n.wk[:-8])):
        with pytest.raises(ValueError):
            DecoderLayer(W, p, norm=bad)
    with pytest.raises(ValueError):
        Stage(W, 1, embed=np.zeros((10, 128), np.float16))


def test_shared_activations_of_layers_with_and_without_qk_norm(torch):
    """A layer without QK norm that shares the activations of one with it rotates Q and K in QKV."""
    from paper_2606_10415_amd.layer import DecoderLayer
    p = layer_inputs(W)
    plain, qk = norms(W, 5, False), norms(W, 5)
    with pytest.raises(ValueError):
        DecoderLayer(W, p, norm=qk, share_acts=DecoderLayer(W, p, norm=plain))
    res = []
    for share in (None, DecoderLayer(W, p, norm=qk)):
        l = DecoderLayer(W, p, norm=plain, share_acts=share)
        l.forward()
        l.backward()
        res.append((l.Y.cpu(), l.dX.cpu(), l.dWqkv.cpu()))
    assert all(torch.equal(a, b) for a, b in zip(*res))


def test_step_graph_replays_match_eager(torch):
    """Embedding, two normed layers of packed attention and their backward in one HIP graph: every replay
    equals the eager step bit for bit, with eager work and synchronisations in between."""
    from paper_2606_10415_amd.stage import Stage
    w = Workload("packed-graph", 22, B=2, S=260, H=256, Hq=8, Hkv=2, D=128, F=344)
    att = packing.documents([[100, 160], [37, 200]], 260, cap=30.0, slopes=packing.alibi_slopes(8))
    st = Stage(w, 2, norm=norms(w, 810), attention=att, embed=5000, embed_scale=2.0)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    ids = torch.randint(-1, 5000, (w.T,), generator=g, device="cuda")
    dy = torch.randn(w.T, w.H, generator=g, device="cuda").half()
    outs = lambda: [st.dWe, st.layers[1].Y, st.layers[0].dWq, st.layers[1].dWk] + \
        [getattr(l, k) for l in st.layers for k in ("dWqkv", "dWn1", "O", "LSE")]
    st.step([ids], [dy])
    torch.cuda.synchronize()
    ref = [t.clone() for t in outs()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        st.step([ids], [dy])
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st.step([ids], [dy])
    torch.cuda.synchronize()
    for r in range(4):
        assert torch.randn(1 << 16, device="cuda").square().sum().item() > 0
        for t in outs():
            t.fill_(float("nan"))
        for l in st.layers[:1]:
            l.ws.fill_(0xff)
        st.embed_ws.fill_(0xff)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(outs(), ref)):
            assert torch.equal(a.view(torch.int16 if a.dtype == torch.float16 else torch.int32),
                               b.view(torch.int16 if b.dtype == torch.float16 else torch.int32)), (r, i)


def test_two_streams_at_once(torch):
    """The same calls on two streams with buffers of their own give what they give alone."""
    from paper_2606_10415_amd.layer import DecoderLayer
    p, n, att = layer_inputs(W), norms(W, 820), attention("docs+cap")
    alone = DecoderLayer(W, p, norm=n, attention=att)
    alone.step()
    torch.cuda.synchronize()
    pair = [DecoderLayer(W, p, norm=n, attention=att) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for rep in range(5):
        for L, s in zip(pair, streams):
            L.step(stream=s)
    torch.cuda.synchronize()
    for L in pair:
        for k in ("Y", "dX", "dWqkv", "dWq", "dQKV"):
            assert torch.equal(getattr(L, k).view(torch.int16), getattr(alone, k).view(torch.int16)), k
