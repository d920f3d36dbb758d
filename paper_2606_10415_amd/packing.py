"""Which keys the queries of a batch see, for the layers' attention.

``Attention`` is what ``DecoderLayer`` and ``Stage`` take; its arrays are those
of ``lt_attn_mod_fwd`` and of the positions of ``lt_qknorm_rope_fwd``.  The
functions below build it for common batches, on the host, once per batch; every
layer then uses the same device arrays.
"""

from dataclasses import dataclass

import numpy as np


@dataclass
class Attention:
    """Intervals of visible keys and score modification (include/lt.h, lt_attn_mod_fwd).

    lo, hi: int32 [B, S] or None; causal: only keys up to the query; cap: tanh cap of the
    scores, 0 for none; slopes: distance bias per query head, or None; pos: int32 [B, S]
    positions for the rotary embedding with QK norm, None for 0 .. S - 1 per row.  The rotation
    without QK norm is by 0 .. S - 1: scores depend on the distance of two positions only.
    """
    lo: object = None
    hi: object = None
    causal: int = 1
    cap: float = 0.0
    slopes: object = None
    pos: object = None


def documents(lengths, S, prefixes=None, **mod):
    """A packed batch: ``lengths[b]`` are the document lengths of batch row b, end to end; tokens
    behind the last document are padding, which sees nothing and is seen by nothing.  Attention is
    causal within each document; with ``prefixes`` (the same nesting) the first so many tokens of a document
    are seen by all of it.  Positions restart with each document.  ``mod``: cap, slopes."""
    B = len(lengths)
    i = np.arange(S, dtype=np.int32)
    lo, hi, pos = (np.zeros((B, S), np.int32) for _ in range(3))
    for b, lens in enumerate(lengths):
        at = 0
        for d, n in enumerate(lens):
            if n < 1 or at + n > S:
                raise ValueError(f"documents of batch row {b} do not fit {S} tokens: {list(lens)}")
            p = prefixes[b][d] if prefixes is not None else 0
            if not 0 <= p <= n:
                raise ValueError(f"prefix {p} of a document of {n} tokens")
            lo[b, at:at + n] = at
            hi[b, at:at + n] = np.maximum(i[at:at + n] + 1, at + p)
            pos[b, at:at + n] = i[:n]
            at += n
    # causal halves the workspace of the backward
    return Attention(lo=lo, hi=hi, causal=0 if prefixes is not None else 1, pos=pos, **mod)


def padded(lengths, S, causal=0, **mod):
    """A padded batch: row b holds ``lengths[b]`` tokens, then padding that takes no part."""
    i = np.arange(S, dtype=np.int32)
    if min(lengths) < 0 or max(lengths) > S:
        raise ValueError(f"lengths outside 0 .. {S}: {list(lengths)}")
    hi = np.stack([np.where(i < n, n, 0) for n in lengths]).astype(np.int32)
    return Attention(hi=hi, causal=causal, **mod)


def window(B, S, width, **mod):
    """A causal sliding window: every query sees itself and the ``width - 1`` keys before it."""
    if width < 1:
        raise ValueError("width must be >= 1")
    lo = np.maximum(np.arange(S, dtype=np.int64) - width + 1, 0).astype(np.int32)
    return Attention(lo=np.broadcast_to(lo, (B, S)).copy(), **mod)


def alibi_slopes(heads):
    """Slopes of the linear distance bias (Press et al., 2022): 2^(-8 (k + 1) / n) for a power of two n of
    heads; otherwise those of the next lower power, then every other one of the next higher."""
    def series(n):
        return [2.0 ** (-8.0 * (k + 1) / n) for k in range(n)]
    p = 1 << (heads.bit_length() - 1)
    s = series(p)
    if p < heads:
        s += series(2 * p)[0::2][:heads - p]
    return np.array(s, dtype=np.float32)
