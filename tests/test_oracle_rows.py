"""The sets of keys of oracle/rows.py against each other: a node of a tree sees what the last row of a chain of its own
ancestors sees."""
import numpy as np
import pytest

from oracle import rows


@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (1, 1), (2, 0), (3, 4), (5, 1), (5, 30), (11, 0), (12, 2), (40, 3), (64, 64)])
@pytest.mark.parametrize("L,Tq", [(40, 12), (12, 12), (5, 12), (1, 1), (13, 12)])
def test_a_chain_as_a_tree(window, sinks, L, Tq):
    bits = np.tril(np.ones((Tq, Tq), dtype=bool))
    n = min(L, Tq)
    got = rows.tree(L, Tq, L + 2, bits, None, window, sinks)
    assert np.array_equal(got[:n], rows.chain(L, n, L + 2, window, sinks))
    assert not got[n:].any()


@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (2, 3), (4, 0), (6, 17), (9, 1), (30, 2)])
@pytest.mark.parametrize("L,Tq,drafted", [(30, 14, None), (30, 14, 9), (14, 14, 14), (9, 14, 20), (100, 40, 33)])
@pytest.mark.parametrize("shuffled", [False, True])
def test_every_path_is_a_chain(window, sinks, L, Tq, drafted, shuffled):
    """Also where a node lies before its ancestors."""
    rng = np.random.default_rng(L + Tq + window)
    n = min(L, Tq, drafted or Tq)
    bits = np.zeros((Tq, Tq), dtype=bool)
    bits[:n, :n] = rows.random_tree(n, rng, reach=1)
    order = rng.permutation(n) if shuffled else np.arange(n)
    bits[:n, :n] = bits[:n, :n][np.ix_(order, order)]
    got, base = rows.tree(L, Tq, L, bits, drafted, window, sinks), L - n
    depth = bits[:n].sum(axis=1)
    assert depth.max() > 3
    for t in range(n):
        path = sorted(np.flatnonzero(bits[t]), key=lambda m: depth[m])  # root first, the node last
        want = np.zeros(L, dtype=bool)
        chain = rows.chain(base + len(path), 1, base + len(path), window, sinks)[0]
        want[:base] = chain[:base]
        want[[base + m for m in path]] = chain[base:]
        assert np.array_equal(got[t], want), t
