"""More than 16 columns (rows x heads of a group): long caches, values that are not finite, the softmax-only twin, gaps, splits of every
count and shapes at random, against the masked CPU oracle."""
import numpy as np
import pytest
import torch

from oracle import rows
from test_gpu_decode_rows import DEV, _check, _inputs, _normal, _paged, plx  # noqa: F401

pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("page", [0, 16, 48, 24])
@pytest.mark.parametrize("heads,d,Tq", [((2, 1), 128, 20), ((8, 1), 128, 20), ((4, 1), 64, 12), ((8, 1), 64, 33)])
def test_one_split_over_a_long_cache(plx, heads, d, Tq, page):
    """More tiles than page addresses are looked up for at a time (64 tiles of 64 or 128 keys)."""
    lens, cap = (9001, 130, 8192 + 128), 9001
    x = _inputs(3, *heads, d, Tq, cap, seed=page + Tq)
    bits = rows.random_tree(Tq, np.random.default_rng(page))
    see = [rows.tree(L, Tq, cap, bits) for L in lens]
    more = {}
    y = x
    if page:
        y = _paged(x, page, seed=page)
        more = dict(block_table=y["block_table"], max_len=cap)
    mask = torch.from_numpy(rows.words(bits)).to(DEV)
    for splits in (1, 2):
        got = plx.parallax_decode_tree(y["q"], y["r"], y["k"], y["v"], y["scale"], mask, seq_lens=_ints(lens), num_splits=splits, **more)
        _check(got, x, see, info=(heads, d, page, splits))


@pytest.mark.parametrize("heads,d,Tq", [((4, 2), 128, 25), ((8, 2), 64, 40), ((8, 2), 128, 40), ((8, 1), 128, 70)])
def test_values_that_are_not_finite(plx, heads, d, Tq):
    """They reach the nodes that see their key, in whichever of the column groups these are, and no other node."""
    L, cap, node = 300, 330, 9
    bits = rows.random_tree(Tq, np.random.default_rng(Tq))
    bits[:, node] = False
    bits[node, node] = bits[Tq - 1, node] = True  # (the last node is in another column group or wave)
    x = _inputs(1, *heads, d, Tq, cap, seed=d + Tq)
    see = rows.tree(L, Tq, cap, bits)[None]
    mask, lens = torch.from_numpy(rows.words(bits)).to(DEV), _ints([L])
    hit = [node, Tq - 1]
    others = [t for t in range(Tq) if t not in hit]
    z = dict(x, q=x["q"][:, :, others], r=x["r"][:, :, others])
    for bad in (float("nan"), float("inf"), float("-inf")):
        for names in (("k",), ("v",), ("k", "v")):
            y = dict(x, k=x["k"].clone(), v=x["v"].clone())
            for n in names:
                y[n][:, :, L - Tq + node, ::3] = bad
                y[n][:, :, L:] = bad
            for splits in (1, 2, 5):
                got = plx.parallax_decode_tree(y["q"], y["r"], y["k"], y["v"], y["scale"], mask, seq_lens=lens, num_splits=splits)
                _check(got[:, :, others], z, see[:, others], info=(bad, names, splits))
                for t in hit:
                    assert not torch.isfinite(got[:, :, t]).all(), (t, bad, names, splits)
    # a committed key: every node sees it
    y = dict(x, v=x["v"].clone())
    y["v"][:, :, 100] = float("nan")
    got = plx.parallax_decode_tree(y["q"], y["r"], y["k"], y["v"], y["scale"], mask, seq_lens=lens)
    assert torch.isnan(got).all()


def test_twin_and_gaps(plx):
    Tq, lens, cap = 30, (400, 333), 400
    bits = np.stack([rows.random_tree(Tq, np.random.default_rng(b)) for b in range(2)])
    mask, lens_t = torch.from_numpy(rows.words(bits)).to(DEV), _ints(lens)
    see = [rows.tree(L, Tq, cap, bits[b]) for b, L in enumerate(lens)]
    for heads in ((4, 2), (16, 2)):
        for d in (64, 128):
            x = _inputs(2, *heads, d, Tq, cap, seed=d)
            got = plx.parallax_decode_tree(x["q"], None, x["k"], x["v"], x["scale"], mask, seq_lens=lens_t, use_r=False)
            _check(got, dict(x, r=torch.zeros_like(x["r"])), see, info=(heads, d, "twin"))
            y = dict(x, k=_normal((2, cap, 2, d + 8), 5, torch.bfloat16)[..., :d].transpose(1, 2),
                     v=_normal((2, 2, cap, d + 16), 6, torch.bfloat16)[..., 8:d + 8])
            got = plx.parallax_decode_tree(y["q"], y["r"], y["k"], y["v"], y["scale"], mask, seq_lens=lens_t)
            _check(got, y, see, info=(heads, d, "gaps"))


@pytest.mark.parametrize("splits", [2, 3, 4, 5, 8, 9, 33, 128])
def test_every_merge(plx, splits):
    """More splits than tiles as well: records of splits without keys."""
    Tq, lens, cap = 18, (700, 40, 0), 700
    x = _inputs(3, 8, 4, 128, Tq, cap, seed=splits)
    see = [rows.chain(L, Tq, cap, 300, 5) for L in lens]
    got = plx.parallax_decode(x["q"], x["r"], x["k"], x["v"], x["scale"], seq_lens=_ints(lens), window=300, sinks=5, num_splits=splits)
    _check(got, x, see, info=splits)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Tq", [5, 20, 70])
def test_the_largest_window_and_sinks(plx, dtype, Tq):
    """2^31 - 1: all keys, also for rows in front of the first token."""
    lens, cap, most = (200, 3, 0), 200, 2**31 - 1
    x = _inputs(3, 4, 2, 64, Tq, cap, seed=Tq, dtype=dtype)
    see = [rows.chain(L, Tq, cap) for L in lens]
    bits = rows.random_tree(Tq, np.random.default_rng(Tq))
    for window, sinks in ((most, 0), (most, 4), (most, most), (1, most), (cap, cap)):
        if sinks:
            got = plx.parallax_decode(x["q"], x["r"], x["k"], x["v"], x["scale"], seq_lens=_ints(lens), window=window, sinks=sinks)
            _check(got, x, see, dtype, (window, sinks))
        got = plx.parallax_decode_tree(x["q"], x["r"], x["k"], x["v"], x["scale"], torch.from_numpy(rows.words(bits)).to(DEV),
                                       seq_lens=_ints(lens), window=window, sinks=sinks)
        _check(got, x, [rows.tree(L, Tq, cap, bits) for L in lens], dtype, (window, sinks, "tree"))


def test_captured_with_new_masks(plx):
    """A captured call is replayed with other masks, lengths and drafts, eager work of the same kind in between."""
    Tq, cap = 40, 900
    rng = np.random.default_rng(8)
    x = _inputs(2, 8, 2, 128, Tq, cap, seed=91)
    mask = torch.from_numpy(rows.words(np.stack([rows.random_tree(Tq, rng) for _ in range(2)]))).to(DEV)
    lens, drafted = _ints([900, 500]), _ints([40, 13])
    call = lambda: plx.parallax_decode_tree(x["q"], x["r"], x["k"], x["v"], x["scale"], mask, seq_lens=lens, draft_lens=drafted)
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for new_lens, new_drafted in (([900, 500], [40, 13]), ([70, 41], [0, 40]), ([1, 0], [1, 5]), ([64, 128], [40, 40])):
        bits = np.stack([rows.random_tree(Tq, rng) for _ in range(2)])
        mask.copy_(torch.from_numpy(rows.words(bits)))
        lens.copy_(_ints(new_lens))
        drafted.copy_(_ints(new_drafted))
        want = call()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), new_lens
        _check(out, x, [rows.tree(L, Tq, cap, bits[b], new_drafted[b]) for b, L in enumerate(new_lens)], info=new_lens)


@pytest.mark.parametrize("seed", range(24))
def test_shapes_at_random(plx, seed):
    rng = np.random.default_rng(1000 + seed)
    B, Hkv, d = int(rng.integers(1, 6)), int(rng.choice([1, 2, 3, 8])), int(rng.choice([64, 128]))
    G = int(rng.choice([1, 2, 3, 5, 8, 16]))
    tree = bool(rng.integers(2))
    Tq = int(rng.integers(max(17 // G, 1), 90))
    cap = int(np.exp(rng.uniform(np.log(Tq), np.log(2500))))
    lens = [int(rng.integers(0, cap + 1)) for _ in range(B)]
    lens[0] = cap
    window = int(rng.integers(1, 400)) if not tree or rng.integers(2) else 0
    sinks = int(rng.choice([1, 4, 70, 130])) if window else 0
    page = int(rng.choice([0, 16, 64, 7]))
    x = _inputs(B, Hkv * G, Hkv, d, Tq, cap, seed=seed)
    y, more = x, dict(seq_lens=_ints(lens), window=window, sinks=sinks)
    if page:
        y = _paged(x, page, seed)
        more.update(block_table=y["block_table"], max_len=cap)
    info = (seed, B, Hkv, G, d, Tq, cap, window, sinks, page, tree)
    if tree:
        drafted = [int(rng.integers(0, Tq + 1)) for _ in range(B)]
        bits = np.stack([rows.random_tree(Tq, rng) for _ in range(B)])
        see = [rows.tree(L, Tq, cap, bits[b], drafted[b], window, sinks) for b, L in enumerate(lens)]
        got = plx.parallax_decode_tree(y["q"], y["r"], y["k"], y["v"], y["scale"], torch.from_numpy(rows.words(bits)).to(DEV),
                                       draft_lens=_ints(drafted), **more)
    else:
        see = [rows.chain(L, Tq, cap, window, sinks) for L in lens]
        got = plx.parallax_decode(y["q"], y["r"], y["k"], y["v"], y["scale"], **more)
    _check(got, x, see, info=info)
