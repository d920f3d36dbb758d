"""GPU parity of lt_embed_fwd / lt_embed_bwd against the float64 oracle, element by element.

Bounds: y is one FP32 product rounded once (h = 2^-11 of the value, 2^-25 below the normal
range).  dW of a row of n tokens: FP32 sums, 2^-24 (n + 3) scale sum |dy|, one rounding.
"""

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


def draw_ids(kind, rng, T, V):
    if kind == "zipf":
        ids = np.minimum(np.exp(rng.random(T) * np.log(V + 1.0)).astype(np.int64) - 1, V - 1)
    elif kind == "one":
        ids = np.full(T, V - 1, np.int64)
    elif kind == "two":
        ids = np.where(rng.random(T) < 0.9, 0, V // 2).astype(np.int64)
    elif kind == "pads":
        return np.where(rng.random(T) < 0.5, -1, V).astype(np.int64)
    else:
        ids = rng.integers(0, V, size=T).astype(np.int64)
    if kind != "one" and T > 3:
        ids[rng.random(T) < 0.05] = -1
        ids[T // 2] = V
        ids[T // 3] = -2 ** 62
        ids[T - 1] = 2 ** 40 + 1
    return ids


CASES = [
    (1, 1, 8, "flat"), (1, 40, 64, "flat"), (7, 3, 8, "zipf"), (64, 1, 72, "one"), (100, 50, 2056, "zipf"),
    (255, 1000, 256, "zipf"), (256, 5000, 4096, "zipf"), (1000, 257, 520, "flat"), (1025, 32000, 1024, "zipf"),
    (3000, 2, 128, "two"), (2500, 700, 64, "one"), (4097, 300, 264, "zipf"), (777, 100, 8192, "two"),
    (50, 20, 64, "pads"), (20000, 3000, 48, "zipf"), (33, 70000, 64, "flat"),
    (300, 40000, 8, "flat"), (20, 50000, 136, "zipf"), (9000, 600, 2568, "one"),
]


@pytest.mark.parametrize("T,V,Hd,kind", CASES)
@pytest.mark.parametrize("scale,pad", [(1.0, 0), (11.3, 8)])
def test_parity(env, T, V, Hd, kind, scale, pad):
    torch, lt = env
    print("embed", T, V, Hd, kind, scale, pad, flush=True)
    rng = np.random.Generator(np.random.PCG64(17 + T + V))
    ids, w, dy = draw_ids(kind, rng, T, V), f16(rng, V, Hd + pad), f16(rng, T + 1, Hd + pad)
    dw0 = f16(rng, V + 1, Hd + pad, std=4.0)
    cu = lambda a: torch.from_numpy(a).cuda()
    I, W, dY = cu(ids), cu(w), cu(dy)
    Y = torch.full((T + 1, Hd + pad), 9.0, dtype=torch.float16, device="cuda")
    lt.lt_embed_fwd(I, W, Hd + pad, scale, Y, Hd + pad, T, Hd, V)
    n = lt.lt_embed_bwd_workspace_size(T, Hd, V)
    ws = torch.full((n + 256,), 0xff, dtype=torch.uint8, device="cuda")
    over = torch.full((V + 1, Hd + pad), float("nan"), dtype=torch.float16, device="cuda")
    lt.lt_embed_bwd(I, dY, Hd + pad, scale, 0, over, Hd + pad, ws, n, T, Hd, V)
    acc = cu(dw0)
    lt.lt_embed_bwd(I, dY, Hd + pad, scale, 1, acc, Hd + pad, ws, n, T, Hd, V)
    torch.cuda.synchronize()
    assert bool((ws[n:] == 0xff).all())
    y, over, acc = Y.cpu().numpy(), over.cpu().numpy(), acc.cpu().numpy()
    assert np.all(y[T] == 9.0) and np.all(y[:, Hd:] == 9.0)
    scale = float(np.float32(scale))
    ry = oracle.embed_fwd(ids, w[:, :Hd], scale)
    assert np.all(abs(y[:T, :Hd] - ry) <= (H + 2.0 ** -24) * abs(ry) + SUB)
    ref = oracle.embed_bwd(ids, dy[:T, :Hd], scale, V)
    mag = oracle.embed_bwd(ids, abs(dy[:T, :Hd]), scale, V)
    ok = (ids >= 0) & (ids < V)
    cnt = np.bincount(ids[ok], minlength=V)
    tol = 2.0 ** -24 * (cnt + 3)[:, None] * mag
    assert np.all(np.isnan(over[V])) and np.all(np.isnan(over[:, Hd:]))
    assert np.all(abs(over[:V, :Hd] - ref) <= tol + H * abs(ref) + SUB)
    assert np.all(over[:V, :Hd][cnt == 0] == 0)
    ref = ref + dw0[:V, :Hd]
    tol = tol + 2.0 ** -24 * abs(ref)
    assert np.all(abs(acc[:V, :Hd] - ref) <= tol + H * abs(ref) + SUB)
    assert np.array_equal(acc[:V][cnt == 0].view(np.uint16), dw0[:V][cnt == 0].view(np.uint16))
    assert np.array_equal(acc[V].view(np.uint16), dw0[V].view(np.uint16))
    assert np.array_equal(acc[:, Hd:].view(np.uint16), dw0[:, Hd:].view(np.uint16))


def test_no_tokens(env):
    torch, lt = env
    V, Hd = 100, 64
    n = lt.lt_embed_bwd_workspace_size(0, Hd, V)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    dW = torch.full((V, Hd), float("nan"), dtype=torch.float16, device="cuda")
    lt.lt_embed_bwd(None, None, Hd, 1.0, 1, dW, Hd, ws, n, 0, Hd, V)
    assert bool(torch.isnan(dW).all())
    lt.lt_embed_bwd(None, None, Hd, 1.0, 0, dW, Hd, ws, n, 0, Hd, V)
    lt.lt_embed_fwd(None, dW, Hd, 1.0, dW, Hd, 0, Hd, V)
    assert bool((dW == 0).all())


def test_non_finite_gradient_stays_in_its_row(env):
    torch, lt = env
    T, V, Hd = 500, 40, 64
    rng = np.random.Generator(np.random.PCG64(5))
    ids = rng.integers(0, V, size=T).astype(np.int64)
    ids[7] = -1
    dy = f16(rng, T, Hd)
    dy[ids == 3] = np.nan
    dy[7] = np.inf
    n = lt.lt_embed_bwd_workspace_size(T, Hd, V)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    dW = torch.empty(V, Hd, dtype=torch.float16, device="cuda")
    lt.lt_embed_bwd(torch.from_numpy(ids).cuda(), torch.from_numpy(dy).cuda(), Hd, 1.0, 0, dW, Hd, ws, n, T, Hd, V)
    nan = torch.isnan(dW).any(1).cpu().numpy()
    assert np.array_equal(nan, np.arange(V) == 3) and bool(torch.isfinite(dW[4:]).all())


def test_results_repeat_bitwise(env):
    torch, lt = env
    T, V, Hd = 6000, 900, 512
    rng = np.random.Generator(np.random.PCG64(6))
    I, dY = torch.from_numpy(draw_ids("zipf", rng, T, V)).cuda(), torch.from_numpy(f16(rng, T, Hd)).cuda()
    n = lt.lt_embed_bwd_workspace_size(T, Hd, V)
    outs = []
    for _ in range(3):
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        dW = torch.empty(V, Hd, dtype=torch.float16, device="cuda")
        lt.lt_embed_bwd(I, dY, Hd, 1.0, 0, dW, Hd, ws, n, T, Hd, V)
        outs.append(dW.cpu().numpy().view(np.uint16))
    assert np.array_equal(outs[0], outs[1]) and np.array_equal(outs[0], outs[2])
