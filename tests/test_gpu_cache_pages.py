"""The pages of a paged cache on the device (fork, extend, free, copy, compact) against the plain ones of oracle/pages.py, and a
run of them together with the attention that reads the cache."""
import numpy as np
import pytest
import torch

from oracle import masked, pages as ref_pages, rows
from parity import BF16_REL_L2, host, rel_l2

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def plx():
    from paper_2605_29157_amd import binding

    binding.load_library()
    assert torch.cuda.is_available()
    return binding


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _state(plx, sequences, width, num_pages, page, rng, stride=None):
    """An empty table with its free list shuffled, and the oracle of it."""
    t = plx.PageTable.empty(sequences, width, num_pages, page, device=DEV)
    order = rng.permutation(num_pages).astype(np.int32)
    t.free_pages.copy_(torch.from_numpy(order))
    if stride:
        table = torch.full((sequences, stride), 77, dtype=torch.int32, device=DEV)
        table[:, :width] = -1
        t = plx.PageTable(table[:, :width], t.seq_lens, t.page_refs, t.free_pages, t.free_count, page)
    o = ref_pages.Pages([[-1] * width for _ in range(sequences)], [0] * sequences, [0] * num_pages, order.tolist(), page)
    return t, o


def _same(t, o, info=()):
    assert t.block_table.tolist() == o.table, info
    assert t.seq_lens.tolist() == o.lens, info
    assert t.page_refs.tolist() == o.refs, info
    assert t.free_count.tolist() == [len(o.free)], info
    assert t.free_pages.tolist()[: len(o.free)] == o.free, info
    named = [x for row in o.table for x in row if x >= 0]
    assert all(o.refs[x] == named.count(x) for x in range(len(o.refs))), info
    assert sorted(o.free + sorted(set(named))) == list(range(len(o.refs))), info


@pytest.mark.parametrize("sequences,width,num_pages,page,stride,seed", [
    (6, 5, 40, 4, None, 0), (9, 7, 60, 1, 11, 1), (40, 33, 900, 16, None, 2), (3, 1, 2, 64, None, 3),
    (130, 300, 20000, 5, 301, 4), (1, 3000, 5000, 2, None, 5)])
def test_random_life_of_a_cache(plx, sequences, width, num_pages, page, stride, seed):
    """Random calls in a row, each compared with the oracle: lists with repeats, with entries outside, with too few pages."""
    rng = np.random.default_rng(seed)
    t, o = _state(plx, sequences, width, num_pages, page, rng, stride)
    for step in range(24):
        n = int(rng.integers(1, min(2 * sequences, 200) + 1))
        pick = rng.integers(-1, sequences + 1, n).tolist()
        kind = rng.choice(["extend", "extend", "fork", "free", "end", "window"]) if step else "extend"
        if kind == "extend":
            to = [int(rng.integers(0, width * page + 3)) if rng.random() < 0.3 else
                  (o.lens[s] if 0 <= s < sequences else 0) + int(rng.integers(0, 3 * page + 1)) for s in pick]
            missing, src, dst, moved = plx.parallax_cache_extend(t, _ints(pick), _ints(to))
            lacking, moves = o.extend(pick, to)
            assert missing.tolist() == [lacking], (step, kind)
            assert list(zip(src.tolist(), dst.tolist(), moved.tolist())) == moves, (step, kind)
        elif kind == "fork":
            children = rng.integers(-1, sequences + 1, n).tolist()
            plx.parallax_cache_fork(t, _ints(pick), _ints(children))
            o.fork(pick, children)
        elif kind == "end":
            plx.parallax_cache_free(t, _ints(pick))
            o.release(pick)
        else:
            first = rng.integers(-2, width * page + 2, n).tolist()
            last = None if kind == "free" else [f + int(rng.integers(0, 5 * page)) for f in first]
            plx.parallax_cache_free(t, _ints(pick), _ints(first), None if last is None else _ints(last))
            o.release(pick, first, last)
        _same(t, o, (step, kind))
    if stride:
        assert (t.block_table.as_strided((sequences, stride - width), (stride, 1), width) == 77).all()


def test_empty_lists_and_all_or_nothing(plx):
    rng = np.random.default_rng(7)
    t, o = _state(plx, 4, 8, 10, 4, rng)
    none = _ints([])
    assert plx.parallax_cache_extend(t, none, none)[0].tolist() == [0]
    plx.parallax_cache_fork(t, none, none)
    plx.parallax_cache_free(t, none)
    _same(t, o)
    missing = plx.parallax_cache_extend(t, _ints([0, 1]), _ints([32, 32]))[0]
    assert missing.tolist() == [6] and o.extend([0, 1], [32, 32])[0] == 6
    _same(t, o)


def test_most_sequences(plx):
    """1024 sequences in one extend, all of them in one fork and one free."""
    rng = np.random.default_rng(8)
    t, o = _state(plx, 2048, 3, 6200, 4, rng)
    seqs = rng.permutation(1024).tolist()
    to = rng.integers(0, 12, 1024).tolist()
    plx.parallax_cache_extend(t, _ints(seqs), _ints(to))
    o.extend(seqs, to)
    _same(t, o)
    plx.parallax_cache_fork(t, _ints(list(range(1024))), _ints(list(range(1024, 2048))))
    o.fork(list(range(1024)), list(range(1024, 2048)))
    _same(t, o)
    both = rng.permutation(2048)[:1024].tolist()
    to = [min(o.lens[s] + 3, 12) for s in both]
    plx.parallax_cache_extend(t, _ints(both), _ints(to))
    o.extend(both, to)
    _same(t, o)
    plx.parallax_cache_free(t, _ints(list(range(2048))))
    o.release(list(range(2048)))
    _same(t, o)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads,page,d,gap", [(8, 16, 128, 0), (1, 64, 576, 0), (3, 5, 64, 8), (2, 1, 8, 0)])
def test_copy(plx, dtype, heads, page, d, gap):
    pools = [torch.randn(20, heads, page, d + gap, device=DEV).to(dtype)[..., :d] for _ in range(2)]
    src, dst, n = [0, 3, -1, 19, 5, 6, 25, 4], [1, 7, 2, 8, -1, 6, 9, 11], [1, page, 1, 0, 2, 3, 1, page + 9]
    for rows_ in (None, n):
        for k, v in ((pools[0], pools[1]), (pools[0], None)):
            want = [p.clone() for p in pools]
            for p, there in zip(want, (True, v is not None)):
                for a, b, c in zip(src, dst, n):
                    if there and 0 <= a < 20 and 0 <= b < 20:
                        m = page if rows_ is None else min(c, page)
                        p[b, :, :m] = p[a, :, :m].clone()
            plx.parallax_cache_copy(k, v, _ints(src), _ints(dst), None if rows_ is None else _ints(rows_))
            assert torch.equal(pools[0], want[0]) and torch.equal(pools[1], want[1])
    if heads == 1:  # a pool without a head dimension
        want = pools[0].clone()
        want[2] = want[3]
        plx.parallax_cache_copy(pools[0][:, 0], None, _ints([3]), _ints([2]))
        assert torch.equal(pools[0], want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page", [0, 16, 5])
@pytest.mark.parametrize("Tq,most", [(1, 1), (5, 3), (64, 64), (200, 130)])
def test_compact(plx, dtype, page, Tq, most):
    rng = np.random.default_rng(Tq + page)
    lens = [300, 7, 0, 205, 64, 1]
    drafted = [Tq, Tq, Tq, max(Tq // 2, 1), 0, 1]
    paths = []
    for n, m in zip(lens, drafted):
        m = min(n, m)
        paths.append(sorted(rng.choice(m, int(rng.integers(0, min(m, most) + 1)), replace=False).tolist()) if m else [])
    accepted = [p + [-5] * (most - len(p)) for p in paths]
    count = [len(p) for p in paths]
    B, Hkv, d, cap = len(lens), 3, 64, 300
    if page:
        per = 60 if page == 5 else 19
        table = rng.permutation(B * per).reshape(B, per)
        shape, table_t = (B * per, Hkv, page, d), _ints(table.tolist())

        def place(b, key):
            return table[b, key // page], slice(None), key % page
    else:
        shape, table_t = (B, Hkv, cap, d), None

        def place(b, key):
            return b, slice(None), key
    pools = [torch.randn(shape, device=DEV).to(dtype) for _ in range(2)]
    want = [host(p) for p in pools]
    for w in want:
        new = ref_pages.compact(w, place, lens, drafted, accepted, count)
    got = plx.parallax_cache_compact(pools[0], pools[1], _ints(lens), _ints(drafted), _ints(accepted), _ints(count),
                                     block_table=table_t)
    assert got.tolist() == new
    for p, w in zip(pools, want):
        np.testing.assert_array_equal(host(p), w)


def test_compact_leaves_rows_without_a_page(plx):
    """Table entries that are no page (-1, past the pool): nothing moves from or to them, the other rows do."""
    page, n_pages, cap = 4, 6, 20
    pools = [torch.randn(n_pages, 2, page, 64, device=DEV).to(torch.bfloat16) for _ in range(2)]
    want = [p.clone() for p in pools]
    table = [[0, 2, -1, 3, n_pages], [5, 4, -1, -1, -1]]
    lens, drafted, accepted = [cap, 6], [cap, 5], [[1, 4, 5, 6, 9, 13, 17], [1, 3, -1, -1, -1, -1, -1]]
    base = [n - m for n, m in zip(lens, drafted)]
    new = plx.parallax_cache_compact(pools[0], pools[1], _ints(lens), _ints(drafted), _ints(accepted), _ints([7, 2]),
                                     block_table=_ints(table))
    assert new.tolist() == [7, 3]
    for w in want:
        old = w.clone()
        for b, count in ((0, 7), (1, 2)):
            for i in range(count):
                src, dst = (divmod(base[b] + x, page) for x in (accepted[b][i], i))
                src, dst = (table[b][src[0]], src[1]), (table[b][dst[0]], dst[1])
                if 0 <= src[0] < n_pages and 0 <= dst[0] < n_pages:
                    w[dst[0], :, dst[1]] = old[src[0], :, src[1]]
    for p, w in zip(pools, want):
        assert torch.equal(p, w)


def test_serving_with_drafts(plx):
    """A cache from its first prompt on: extend, fork, drafted trees, verification, acceptance, and pages behind the window given
    back; after every step the attention equals the oracle's over the tokens that the sequence is made of."""
    rng = np.random.default_rng(11)
    Hq, Hkv, d, page, Tq = 8, 4, 64, 16, 6
    t, o = _state(plx, 4, 12, 40, page, rng)
    k, v = (torch.full((40, Hkv, page, d), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    truth = {s: ([], []) for s in range(4)}  # rows of K, V per token
    window, sinks, scale = 40, 5, d ** -0.5

    def write(s, at, n):
        """n new rows of sequence s from token `at` on"""
        del truth[s][0][at:], truth[s][1][at:]
        for j in range(at, at + n):
            for pool, kept in zip((k, v), truth[s]):
                row = torch.randn(Hkv, d).to(torch.bfloat16)
                pool[t.block_table[s, j // page].long(), :, j % page] = row.to(DEV)
                kept.append(row.float().numpy())

    def extend(seqs, to):
        missing = plx.parallax_cache_extend(t, _ints(seqs), _ints(to), k, v)
        assert missing.tolist() == [0] and o.extend(seqs, to)[0] == 0

    def check(got, q, r, see_of):
        for s in range(4):
            if not truth[s][0]:
                assert (got[s] == 0).all()
                continue
            K, V = (np.stack(x, 1)[None] for x in truth[s])
            see = see_of(s, K.shape[2])
            want = masked.masked_forward(host(q)[s:s + 1], host(r)[s:s + 1], K, V, scale, see[None, None])
            assert rel_l2(host(got)[s:s + 1], want) <= BF16_REL_L2, s

    extend([0, 1], [70, 33])
    write(0, 0, 70)
    write(1, 0, 33)
    for step in range(6):
        if step == 1:
            plx.parallax_cache_fork(t, _ints([0, 1]), _ints([2, 3]))
            o.fork([0, 1], [2, 3])
            for a, b in ((0, 2), (1, 3)):
                truth[b] = (list(truth[a][0]), list(truth[a][1]))
        live = [s for s in range(4) if o.lens[s]]
        base = list(o.lens)
        drafted = [int(rng.integers(1, Tq + 1)) if s in live else 0 for s in range(4)]
        extend(live, [base[s] + drafted[s] for s in live])
        for s in live:
            write(s, base[s], drafted[s])
        _same(t, o, step)
        bits = np.stack([rows.random_tree(Tq, rng) for _ in range(4)])
        q, r = (torch.randn(4, Hq, Tq, d, device=DEV).to(torch.bfloat16) for _ in range(2))
        got = plx.parallax_decode_tree(q, r, k, v, scale, torch.from_numpy(rows.words(bits)).to(DEV), seq_lens=t.seq_lens,
                                       draft_lens=_ints(drafted), block_table=t.block_table, window=window, sinks=sinks)
        check(got, q, r, lambda s, n: rows.tree(n, Tq, n, bits[s], drafted[s], window, sinks))
        # accept a path of every tree: the last node and its ancestors
        paths = [np.flatnonzero(bits[s][drafted[s] - 1][: drafted[s]]).tolist() if s in live else [] for s in range(4)]
        accepted = _ints([p + [-1] * (Tq - len(p)) for p in paths])
        lens = plx.parallax_cache_compact(k, v, t.seq_lens, _ints(drafted), accepted, _ints([len(p) for p in paths]),
                                          block_table=t.block_table)
        for s in live:
            for kept in truth[s]:
                kept[base[s]:] = [kept[base[s] + m] for m in paths[s]]
        assert lens.tolist() == [base[s] + len(paths[s]) for s in range(4)]
        plx.parallax_cache_free(t, _ints(list(range(4))), lens)  # the rejected ones
        o.release(list(range(4)), lens.tolist())
        behind = [max(o.lens[s] - window, 0) for s in range(4)]
        plx.parallax_cache_free(t, _ints(list(range(4))), _ints([sinks] * 4), _ints(behind))
        o.release(list(range(4)), [sinks] * 4, behind)
        _same(t, o, step)
        k[t.free_pages[: int(t.free_count)].long()] = float("nan")  # nobody reads what is free
        v[t.free_pages[: int(t.free_count)].long()] = float("inf")
        q, r = (torch.randn(4, Hq, 1, d, device=DEV).to(torch.bfloat16) for _ in range(2))
        got = plx.parallax_decode(q, r, k, v, scale, seq_lens=t.seq_lens, block_table=t.block_table, window=window, sinks=sinks)
        check(got, q, r, lambda s, n: rows.chain(n, 1, n, window, sinks))
    plx.parallax_cache_free(t, _ints([0, 1, 2, 3]))
    o.release([0, 1, 2, 3])
    _same(t, o)
    assert len(o.free) == 40


def test_captured_calls(plx):
    """Fork, extend and free in a graph, replayed with eager work between the replays; on another stream too."""
    rng = np.random.default_rng(12)
    t, o = _state(plx, 6, 9, 60, 4, rng)
    k, v = (torch.randn(60, 2, 4, 64, device=DEV).to(torch.bfloat16) for _ in range(2))
    plx.parallax_cache_extend(t, _ints([0, 1, 2]), _ints([9, 14, 3]), k, v)
    o.extend([0, 1, 2], [9, 14, 3])
    parents, children, seqs = _ints([0, 1, 2]), _ints([3, 4, 5]), _ints([3, 4, 5, 0, 1, 2])
    first, to = _ints([0, 0, 0, 9, 14, 3]), _ints([12, 20, 4, 10, 15, 9])

    def cycle():
        plx.parallax_cache_free(t, seqs, first)
        plx.parallax_cache_fork(t, parents, children)
        return plx.parallax_cache_extend(t, seqs, to, k, v)

    def expect():
        o.release(seqs.tolist(), first.tolist())
        o.fork(parents.tolist(), children.tolist())
        return o.extend(seqs.tolist(), to.tolist())[0]

    cycle()
    expect()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        missing = cycle()
    for new in ([12, 20, 4, 10, 15, 9], [30, 36, 1, 36, 36, 36], [36] * 6, [12, 20, 4, 9, 14, 3]):
        to.copy_(_ints(new))
        graph.replay()
        torch.cuda.synchronize()
        assert missing.tolist() == [expect()]
        _same(t, o, new)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        cycle()
    side.synchronize()
    expect()
    _same(t, o)
