"""The plain bookkeeping of oracle/pages.py: what holds after any run of calls."""
import numpy as np
import pytest

from oracle.pages import Pages


@pytest.mark.parametrize("seed", range(6))
def test_every_new_token_has_a_page(seed):
    rng = np.random.default_rng(seed)
    sequences, width, page, num_pages = 6, 8, int(rng.choice([1, 3, 4, 16])), 40
    o = Pages([[-1] * width for _ in range(sequences)], [0] * sequences, [0] * num_pages, rng.permutation(num_pages).tolist(), page)
    for _ in range(200):
        pick = rng.permutation(sequences)[: int(rng.integers(1, 4))].tolist()
        kind = rng.choice(["extend", "extend", "fork", "free", "window"])
        if kind == "extend":
            before, to = list(o.lens), [o.lens[s] + int(rng.integers(0, 2 * page + 1)) for s in pick]
            missing, _ = o.extend(pick, to)
            for s in pick if missing == 0 else []:
                assert all(o.table[s][token // page] >= 0 for token in range(before[s], o.lens[s]))
        elif kind == "fork":
            o.fork(pick, rng.permutation(sequences)[: len(pick)].tolist())
        else:
            first = [int(rng.integers(0, o.lens[s] + 1)) for s in pick]
            o.release(pick, first, None if kind == "free" else [f + int(rng.integers(0, 4 * page)) for f in first])
        named = [x for row in o.table for x in row if x >= 0]
        assert all(o.refs[x] == named.count(x) for x in range(num_pages))
        assert sorted(o.free + sorted(set(named))) == list(range(num_pages))
