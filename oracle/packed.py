"""Oracle of the packed-sequence operators (test infrastructure only).

* Attention in which query i sees the keys lo_i <= j < hi_i, with scores
      s = scale q.k,  capped: cap tanh(s / cap),  biased: s - slope |i - j|,
  P = row softmax over the keys seen, O = P V; a query that sees nothing has
  O = 0 and LSE = -inf.  Gradient of sum(O * dO):
      dP = dO V^T,  dZ = P (dP - sum_k P_ik dP_ik),  dS = dZ (1 - tanh^2),
      dq = scale dS K,  dk = scale dS^T Q,  dv = P^T dO.
* RMSNorm of a head (Zhang & Sennrich, 2019) followed by the rotate-half rotary
  embedding (Su et al., 2021) at a given position.
* Embedding y_t = scale W[id_t] and its gradient; ids outside the table are
  padding: a zero row, no gradient.

Everything is float64, one head (or one table) at a time, full score matrices.
"""

import numpy as np

f64 = np.float64


def intervals(S, lo=None, hi=None, causal=False):
    """(lo, hi) int arrays [S] of the keys each query sees, clamped; nothing: (0, 0)."""
    i = np.arange(S)
    lo = np.zeros(S, dtype=np.int64) if lo is None else np.maximum(np.asarray(lo, dtype=np.int64), 0)
    hi = np.full(S, S) if hi is None else np.minimum(np.asarray(hi, dtype=np.int64), S)
    if causal:
        hi = np.minimum(hi, i + 1)
    none = lo >= hi
    return np.where(none, 0, lo), np.where(none, 0, hi)


def attn_mod_head(q, k, v, scale, lo, hi, cap=0.0, slope=0.0, do=None):
    """One head: q [S, D], k, v [S, D], lo, hi [S].  Returns a dict with o, lse, p, see and, given do,
    dq, dk, dv, dp, delta, ds and the cap's derivative w."""
    q, k, v = (np.asarray(x, dtype=f64) for x in (q, k, v))
    S = q.shape[0]
    i, j = np.arange(S)[:, None], np.arange(S)[None, :]
    see = (j >= lo[:, None]) & (j < hi[:, None])
    # what no query sees, and what queries that see nothing hold, takes no part
    k, v = np.where(see.any(0)[:, None], k, 0.0), np.where(see.any(0)[:, None], v, 0.0)
    q = np.where(see.any(1)[:, None], q, 0.0)
    s = float(scale) * (q @ k.T)
    w = np.ones_like(s)
    if cap > 0:
        t = np.tanh(s / cap)
        s, w = cap * t, 1.0 - t * t
    s = s - float(slope) * np.abs(i - j)
    s = np.where(see, s, -np.inf)
    some = see.any(1)
    m = np.where(some, s.max(1), 0.0)
    e = np.exp(s - m[:, None])
    l = e.sum(1)
    p = e / np.where(some, l, 1.0)[:, None]
    with np.errstate(divide="ignore"):
        lse = np.where(some, m + np.log(np.where(some, l, 1.0)), -np.inf)
    r = dict(o=p @ v, lse=lse, p=p, see=see)
    if do is not None:
        do = np.where(some[:, None], np.asarray(do, dtype=f64), 0.0)
        dp = do @ v.T
        delta = (p * dp).sum(1)
        ds = p * (dp - delta[:, None]) * w
        r.update(dp=dp, delta=delta, ds=ds, w=w, dq=scale * (ds @ k), dk=scale * (ds.T @ q), dv=p.T @ do)
    return r


def qknorm_rope(x, wq, wk, hq, pos, base, eps, dy=None):
    """x [T, heads, D], pos [T].  Returns (y, r) or, given dy, (y, r, dx, dwq, dwk)."""
    x = np.asarray(x, dtype=f64)
    T, n, D = x.shape
    h = D // 2
    w = np.where((np.arange(n) < hq)[:, None], np.asarray(wq, dtype=f64), np.asarray(wk, dtype=f64))
    a = np.asarray(pos, dtype=f64)[:, None] * float(base) ** (-2.0 * np.arange(h) / D)
    c, s = np.cos(a)[:, None, :], np.sin(a)[:, None, :]
    r = 1.0 / np.sqrt(np.mean(x * x, axis=2) + eps)
    u = w * x * r[:, :, None]
    y = np.concatenate([u[..., :h] * c - u[..., h:] * s, u[..., h:] * c + u[..., :h] * s], axis=2)
    if dy is None:
        return y, r
    dy = np.asarray(dy, dtype=f64)
    g = np.concatenate([dy[..., :h] * c + dy[..., h:] * s, dy[..., h:] * c - dy[..., :h] * s], axis=2)
    dx = r[:, :, None] * w * g - (r ** 3)[:, :, None] * x * np.mean(g * w * x, axis=2, keepdims=True)
    dw = np.sum(g * x * r[:, :, None], axis=0)
    return y, r, dx, dw[:hq].sum(0), dw[hq:].sum(0)


def embed_fwd(ids, w, scale):
    w = np.asarray(w, dtype=f64)
    y = np.zeros((len(ids), w.shape[1]))
    for t, v in enumerate(ids):
        if 0 <= v < w.shape[0]:
            y[t] = scale * w[v]
    return y


def embed_bwd(ids, dy, scale, V):
    dy = np.asarray(dy, dtype=f64)
    dw = np.zeros((V, dy.shape[1]))
    for t, v in enumerate(ids):
        if 0 <= v < V:
            dw[v] += scale * dy[t]
    return dw
