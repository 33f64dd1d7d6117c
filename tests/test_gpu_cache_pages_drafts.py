"""Verification and compaction of the same drafted rows, with draft_lens longer than the tree."""
import numpy as np
import pytest
import torch

from oracle import pages as ref_pages, rows
from test_gpu_cache_pages import DEV, _ints, plx  # noqa: F401
from test_gpu_decode_rows import _check, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page", [0, 16])
def test_drafts_longer_than_the_tree(plx, page):
    """draft_lens above Tq: the tree's nodes are the last Tq cached tokens, and with max_draft = Tq compaction moves those."""
    Tq, cap, lens, drafted = 6, 96, [90, 40, 3], [20, 6, 9]
    bits = np.tril(np.ones((Tq, Tq), dtype=bool))
    x = _inputs(3, 4, 2, 64, Tq, cap, seed=1)
    k, v, table = x["k"], x["v"], None
    if page:
        order = np.random.default_rng(4).permutation(3 * (cap // page))
        table = _ints(order.reshape(3, -1).tolist())
        k, v = (torch.empty(3 * (cap // page), 2, page, 64, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        for pool, rows_ in ((k, x["k"]), (v, x["v"])):
            pool[torch.as_tensor(order, device=DEV)] = rows_.reshape(3, 2, -1, page, 64).transpose(1, 2).reshape(-1, 2, page, 64)
    more = {} if table is None else dict(block_table=table)
    got = plx.parallax_decode_tree(x["q"], x["r"], k, v, x["scale"], torch.from_numpy(rows.words(bits)).to(DEV),
                                   seq_lens=_ints(lens), draft_lens=_ints(drafted), **more)
    _check(got, x, [rows.tree(L, Tq, cap, bits, n) for L, n in zip(lens, drafted)])
    accepted, count = [[0, 2, 5], [3, 4, 5], [1, 2, -1]], [3, 3, 2]
    place = (lambda b, key: (int(table[b, key // page]), slice(None), key % page)) if page else (lambda b, key: (b, slice(None), key))
    want = [p.float().cpu().numpy() for p in (k, v)]
    for w in want:
        new = ref_pages.compact(w, place, lens, [min(n, Tq) for n in drafted], accepted, count)
    assert new == [87, 37, 2]
    got = plx.parallax_cache_compact(k, v, _ints(lens), _ints(drafted), _ints(accepted), _ints(count), max_draft=Tq, **more)
    assert got.tolist() == new
    for p, w in zip((k, v), want):
        np.testing.assert_array_equal(p.float().cpu().numpy(), w)
