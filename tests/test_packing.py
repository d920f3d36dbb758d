"""CPU checks of the packed-batch descriptions (packing.py)."""

import numpy as np
import pytest

from paper_2606_10415_amd import packing


def sees(a, b, S):
    i, j = np.arange(S)[:, None], np.arange(S)[None, :]
    m = np.ones((S, S), bool)
    if a.lo is not None:
        m &= j >= a.lo[b][:, None]
    if a.hi is not None:
        m &= j < a.hi[b][:, None]
    return m & (j <= i) if a.causal else m


def test_documents():
    a = packing.documents([[3, 2], [6]], 7)
    doc = [[0, 0, 0, 1, 1, -1, -2], [0] * 6 + [-1]]
    for b in range(2):
        want = np.array([[doc[b][i] == doc[b][j] and doc[b][i] >= 0 and j <= i for j in range(7)] for i in range(7)])
        assert np.array_equal(sees(a, b, 7), want)
    assert a.pos.tolist() == [[0, 1, 2, 0, 1, 0, 0], [0, 1, 2, 3, 4, 5, 0]]
    p = packing.documents([[4, 3]], 7, prefixes=[[2, 0]], cap=30.0)
    assert p.hi.tolist() == [[2, 2, 3, 4, 5, 6, 7]] and p.lo.tolist() == [[0, 0, 0, 0, 4, 4, 4]] and p.cap == 30.0


def test_padded_and_window():
    a = packing.padded([2, 0, 4], 4)
    assert a.hi.tolist() == [[2, 2, 0, 0], [0, 0, 0, 0], [4, 4, 4, 4]] and a.causal == 0
    w = packing.window(2, 5, 2)
    assert w.causal == 1 and w.lo.tolist() == [[0, 0, 1, 2, 3]] * 2


def test_slopes():
    assert np.allclose(packing.alibi_slopes(8), [2.0 ** -k for k in range(1, 9)])
    s = packing.alibi_slopes(12)
    assert len(s) == 12 and np.allclose(s[8:], [2.0 ** (-0.5 * k) for k in (1, 3, 5, 7)])


@pytest.mark.parametrize("f,a", [(packing.documents, ([[3, 5]], 7)), (packing.documents, ([[0, 5]], 7)),
                                 (packing.documents, ([[3]], 7, [[4]])), (packing.padded, ([8], 7)),
                                 (packing.window, (1, 7, 0))])
def test_refusals(f, a):
    with pytest.raises(ValueError):
        f(*a)
