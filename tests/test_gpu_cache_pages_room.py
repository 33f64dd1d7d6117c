"""Room in a cache: after parallax_cache_extend every new token has a page, also where pages had been given back."""
import numpy as np
import pytest
import torch

from test_gpu_cache_pages import DEV, _ints, _same, _state, plx  # noqa: F401

pytestmark = pytest.mark.gpu


def _every_token_has_a_page(t, s, first, end):
    row = t.block_table[s].tolist()
    for token in range(first, end):
        assert row[token // t.page_size] >= 0, (s, token, row)


@pytest.mark.parametrize("shared", [False, True])
def test_room_where_the_last_page_was_given_back(plx, shared):
    """A sequence whose end was moved into a range that had been given back has no last page: extend hands one out."""
    rng = np.random.default_rng(1)
    t, o = _state(plx, 4, 12, 60, 4, rng)
    k, v = (torch.randn(60, 2, 4, 64, device=DEV).to(torch.bfloat16) for _ in range(2))
    for seqs, to in (([0, 1], [40, 38]),):
        plx.parallax_cache_extend(t, _ints(seqs), _ints(to), k, v)
        o.extend(seqs, to)
    plx.parallax_cache_free(t, _ints([0, 1]), _ints([4, 8]), _ints([32, 30]))  # behind the sinks, in front of the window
    o.release([0, 1], [4, 8], [32, 30])
    plx.parallax_cache_free(t, _ints([0, 1]), _ints([13, 18]))  # the ends drop into it
    o.release([0, 1], [13, 18])
    _same(t, o, "freed")
    assert t.seq_lens.tolist()[:2] == [13, 18] and t.block_table[0, 3] == -1 and t.block_table[1, 4] == -1
    if shared:
        plx.parallax_cache_fork(t, _ints([0]), _ints([2]))
        o.fork([0], [2])
    seqs, to = [2, 1, 0, 3], [15, 27, 16, 5]
    missing, src, dst, moved = plx.parallax_cache_extend(t, _ints(seqs), _ints(to))
    lacking, moves = o.extend(seqs, to)
    assert missing.tolist() == [lacking] == [0]
    assert list(zip(src.tolist(), dst.tolist(), moved.tolist())) == moves
    _same(t, o, "extended")
    before = [13 if shared else 0, 18, 13, 0]
    for s, first, end in zip(seqs, before, to):
        assert t.seq_lens[s] == end
        _every_token_has_a_page(t, s, first, end)


def test_lacking_pages_count_the_last_one_too(plx):
    t, o = _state(plx, 1, 8, 8, 4, np.random.default_rng(2))
    plx.parallax_cache_extend(t, _ints([0]), _ints([32]))
    o.extend([0], [32])
    plx.parallax_cache_free(t, _ints([0]), _ints([8]), _ints([28]))
    plx.parallax_cache_free(t, _ints([0]), _ints([10]))
    o.release([0], [8], [28])
    o.release([0], [10])
    t.free_count.fill_(2)  # (two of the six free ones)
    o.free = o.free[:2]
    before = [x.clone() for x in (t.block_table, t.seq_lens, t.page_refs, t.free_pages, t.free_count)]
    assert plx.parallax_cache_extend(t, _ints([0]), _ints([17]))[0].tolist() == [1]  # tokens 10 .. 16: pages 2, 3, 4
    for a, b in zip(before, (t.block_table, t.seq_lens, t.page_refs, t.free_pages, t.free_count)):
        assert torch.equal(a, b)
    assert plx.parallax_cache_extend(t, _ints([0]), _ints([16]))[0].tolist() == [0]
    _every_token_has_a_page(t, 0, 10, 16)


@pytest.mark.parametrize("seed", range(4))
def test_every_new_token_has_a_page(plx, seed):
    """Random calls; after an extend that lacks nothing each listed sequence has a page for every token it grew by."""
    rng = np.random.default_rng(50 + seed)
    sequences, width, page = 7, 9, int(rng.choice([3, 4, 16]))
    t, o = _state(plx, sequences, width, 90, page, rng)
    grown = 0
    for step in range(60):
        pick = rng.permutation(sequences)[: int(rng.integers(1, 5))].tolist()
        if step % 3 != 2:
            before = t.seq_lens.tolist()
            to = [min(before[s] + int(rng.integers(0, 2 * page + 1)), width * page) for s in pick]
            missing = plx.parallax_cache_extend(t, _ints(pick), _ints(to))[0].tolist()
            assert missing == [o.extend(pick, to)[0]]
            if missing == [0]:
                for s, end in zip(pick, to):
                    assert t.seq_lens[s] == end
                    _every_token_has_a_page(t, s, before[s], end)
                    grown += end - before[s]
        else:
            first = [int(rng.integers(0, max(o.lens[s], 1))) for s in pick]
            last = [f + int(rng.integers(0, 4 * page)) for f in first] if step % 2 else None
            plx.parallax_cache_free(t, _ints(pick), _ints(first), None if last is None else _ints(last))
            o.release(pick, first, last)
        _same(t, o, step)
    assert grown > 100
