"""Trees of drafted nodes behind a sliding window that is shorter than the draft: a node sees what a decode of its own path,
token after token, would see (through the C ABI, against the masked CPU oracle)."""
import numpy as np
import pytest
import torch

from oracle import rows
from test_gpu_decode_rows import DEV, _check, _inputs, _paged, plx  # noqa: F401

pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _path_sees(L, Tq, cap, bits, drafted, window, sinks):
    """rows.chain of every node's own path, the drafted keys put where the nodes lie."""
    n = min(L, Tq, drafted)
    base, see = L - n, np.zeros((Tq, cap), dtype=bool)
    depth = bits[:n, :n].sum(axis=1)
    for t in range(n):
        path = sorted(np.flatnonzero(bits[t, :n]), key=lambda m: depth[m])
        chain = rows.chain(base + len(path), 1, base + len(path), window, sinks)[0]
        see[t, :base] = chain[:base]
        see[t, [base + m for m in path]] = chain[base:]
    return see


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads,d,Tq", [((4, 2), 128, 7), ((4, 4), 64, 16), ((4, 2), 64, 25), ((8, 2), 128, 40), ((4, 1), 64, 150)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (3, 2), (6, 400), (6, 0)])
def test_a_chain_as_a_tree(plx, dtype, heads, d, Tq, window, sinks):
    """... gives what the decode over the last Tq positions with the same window gives."""
    lens = (420, Tq + 1, Tq)
    x = _inputs(3, *heads, d, Tq, 420, seed=Tq + window, dtype=dtype)
    see = [rows.chain(L, Tq, 420, window, sinks) for L in lens]
    mask = torch.from_numpy(rows.words(np.tril(np.ones((Tq, Tq), dtype=bool)))).to(DEV)
    for splits in (0, 1, 3):
        got = plx.parallax_decode_tree(x["q"], x["r"], x["k"], x["v"], x["scale"], mask, seq_lens=_ints(lens), window=window,
                                       sinks=sinks, num_splits=splits)
        _check(got, x, see, dtype, (window, sinks, splits, "tree"))
    if sinks:
        got = plx.parallax_decode(x["q"], x["r"], x["k"], x["v"], x["scale"], seq_lens=_ints(lens), window=window, sinks=sinks)
        _check(got, x, see, dtype, (window, sinks, "chain"))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page", [0, 16, 24])
@pytest.mark.parametrize("heads,d,Tq", [((4, 2), 128, 8), ((8, 2), 64, 30), ((8, 2), 128, 70), ((2, 1), 128, 256)])
@pytest.mark.parametrize("window,sinks", [(2, 0), (5, 9), (9, 300)])
def test_every_path(plx, dtype, page, heads, d, Tq, window, sinks):
    """Trees deeper than the window, also with nodes that lie before their ancestors; sinks that reach the drafted keys."""
    lens, drafted, cap = (600, Tq + 3, Tq // 2, 0), (Tq, Tq - 1, Tq, 1), 600
    rng = np.random.default_rng(Tq + window)
    bits = np.stack([rows.random_tree(Tq, rng, reach=1) for _ in lens])
    n = drafted[1]  # (the second one's nodes in any order)
    order = rng.permutation(n)
    bits[1, :n, :n] = bits[1, :n, :n][np.ix_(order, order)]
    bits[1, n:] = False
    see = [_path_sees(L, Tq, cap, bits[b], drafted[b], window, sinks) for b, L in enumerate(lens)]
    x = _inputs(4, *heads, d, Tq, cap, seed=Tq + page, dtype=dtype)
    y, more = x, {}
    if page:
        y = _paged(x, page, seed=page)
        more = dict(block_table=y["block_table"], max_len=cap)
    for splits in (0, 2):
        got = plx.parallax_decode_tree(y["q"], y["r"], y["k"], y["v"], y["scale"], torch.from_numpy(rows.words(bits)).to(DEV),
                                       seq_lens=_ints(lens), draft_lens=_ints(drafted), window=window, sinks=sinks, num_splits=splits, **more)
        _check(got, x, see, dtype, (page, splits))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_ancestors_behind_the_window_hold_anything(plx, dtype):
    """A drafted key that has left a node's window does not reach it, whatever its row holds."""
    for heads, Tq in (((4, 2), 8), ((8, 2), 40)):
        L, cap, window = 300, 310, 4
        x = _inputs(1, *heads, 64, Tq, cap, seed=Tq, dtype=dtype)
        mask = torch.from_numpy(rows.words(np.tril(np.ones((Tq, Tq), dtype=bool)))).to(DEV)
        see = rows.chain(L, Tq, cap, window)[None]
        free = [t for t in range(Tq) if t < 2 or t >= 2 + window]  # nodes that do not see node 2
        z = dict(x, q=x["q"][:, :, free], r=x["r"][:, :, free])
        for bad in (float("nan"), float("inf")):
            y = dict(x, k=x["k"].clone(), v=x["v"].clone())
            y["k"][:, :, L - Tq + 2] = bad
            y["v"][:, :, L - Tq + 2] = bad
            for splits in (1, 3):
                got = plx.parallax_decode_tree(y["q"], y["r"], y["k"], y["v"], y["scale"], mask, seq_lens=_ints([L]), window=window,
                                               num_splits=splits)
                _check(got[:, :, free], z, see[:, free], dtype, (heads, bad, splits))
                for t in range(2, 2 + window):
                    assert not torch.isfinite(got[:, :, t]).all(), (t, bad)


@pytest.mark.parametrize("d,page", [(36, 0), (64, 16), (132, 7), (200, 0), (256, 0), (256, 5)])
@pytest.mark.parametrize("heads,Tq", [((6, 2), 5), ((2, 2), 20), ((4, 1), 100)])
def test_f32_head_dimensions(plx, d, page, heads, Tq):
    lens, drafted, cap, window, sinks = (333, Tq + 20), (Tq, Tq - 2), 333, 3, 7
    rng = np.random.default_rng(d + Tq)
    bits = np.stack([rows.random_tree(Tq, rng, reach=1) for _ in lens])
    see = [_path_sees(L, Tq, cap, bits[b], drafted[b], window, sinks) for b, L in enumerate(lens)]
    x = _inputs(2, *heads, d, Tq, cap, seed=d, dtype=torch.float32)
    y, more = x, {}
    if page:
        y = _paged(x, page, seed=page)
        more = dict(block_table=y["block_table"], max_len=cap)
    mask = torch.from_numpy(rows.words(bits)).to(DEV)
    for use_r in (True, False):
        z = x if use_r else dict(x, r=torch.zeros_like(x["r"]))
        for splits in (0, 3):
            got = plx.parallax_decode_tree(y["q"], y["r"] if use_r else None, y["k"], y["v"], y["scale"], mask, seq_lens=_ints(lens),
                                           draft_lens=_ints(drafted), window=window, sinks=sinks, use_r=use_r, num_splits=splits, **more)
            _check(got, z, see, torch.float32, (d, page, use_r, splits))


def test_captured_with_new_drafts(plx):
    """The window is shorter than some of the drafts that a captured call is replayed with."""
    Tq, cap, window = 30, 500, 6
    rng = np.random.default_rng(5)
    for dtype in (torch.bfloat16, torch.float32):
        x = _inputs(2, 8, 4, 64, Tq, cap, seed=3, dtype=dtype)
        mask = torch.from_numpy(rows.words(np.stack([rows.random_tree(Tq, rng, reach=1) for _ in range(2)]))).to(DEV)
        lens, drafted = _ints([500, 300]), _ints([30, 5])
        call = lambda: plx.parallax_decode_tree(x["q"], x["r"], x["k"], x["v"], x["scale"], mask, seq_lens=lens, draft_lens=drafted,
                                                window=window, sinks=2)
        call()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = call()
        for new_lens, new_drafted in (([500, 300], [30, 5]), ([31, 6], [30, 6]), ([3, 0], [7, 7]), ([400, 129], [0, 30])):
            bits = np.stack([rows.random_tree(Tq, rng, reach=1) for _ in range(2)])
            mask.copy_(torch.from_numpy(rows.words(bits)))
            lens.copy_(_ints(new_lens))
            drafted.copy_(_ints(new_drafted))
            want = call()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want), new_lens
            _check(out, x, [_path_sees(L, Tq, cap, bits[b], new_drafted[b], window, 2) for b, L in enumerate(new_lens)], dtype, new_lens)
