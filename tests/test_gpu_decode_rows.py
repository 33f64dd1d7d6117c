"""GPU parity of the decode of rows whose key sets differ (through the C ABI) against the masked CPU oracle: a sliding window
with sinks (parallax_decode(..., sinks=)) and trees of drafted nodes (parallax_decode_tree)."""
import numpy as np
import pytest
import torch

from oracle import masked, rows
from parity import BF16_REL_L2, F32_MAX_REL, host, max_rel, rel_l2

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def plx():
    from paper_2605_29157_amd import binding

    binding.load_library()
    assert torch.cuda.is_available()
    return binding


def _normal(shape, seed, dtype):
    gen = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=gen).to(dtype).to(DEV)


def _inputs(B, Hq, Hkv, d, Tq, cap, seed, dtype=torch.bfloat16):
    return dict(q=_normal((B, Hq, Tq, d), seed, dtype), r=_normal((B, Hq, Tq, d), seed + 1, dtype),
                k=_normal((B, Hkv, cap, d), seed + 2, dtype), v=_normal((B, Hkv, cap, d), seed + 3, dtype),
                scale=d ** -0.5)


def _paged(x, page, seed):
    """Pools of shuffled pages that hold the caches of x, and their block table."""
    B, Hkv, cap, d = x["k"].shape
    per = -(-cap // page)
    order = np.random.default_rng(seed).permutation(B * per + 3)[: B * per]
    out = dict(x, block_table=torch.tensor(order.reshape(B, per), dtype=torch.int32, device=DEV), max_len=cap)
    for n in ("k", "v"):
        pool = torch.full((B * per + 3, Hkv, page, d), float("nan"), dtype=x[n].dtype, device=DEV)
        padded = torch.full((B, Hkv, per * page, d), float("nan"), dtype=x[n].dtype, device=DEV)
        padded[:, :, :cap] = x[n]
        pool[torch.as_tensor(order, device=DEV)] = padded.reshape(B, Hkv, per, page, d).transpose(1, 2).reshape(
            B * per, Hkv, page, d)
        out[n] = pool
    return out


def _check(got, x, see, dtype=torch.bfloat16, info=()):
    """see [B, Tq, cap]"""
    see = np.asarray(see)
    mask = see[:, None]
    # (keys nobody sees may hold anything: the oracle multiplies by zero, so they are cleared for it)
    used = see.any(axis=1)[:, None, :, None]
    q, r = host(x["q"]), host(x["r"])
    k, v = (np.where(used, np.nan_to_num(host(x[n])), 0.0) for n in ("k", "v"))
    ref = masked.masked_forward(q, r, k, v, x["scale"], mask)
    got = host(got).astype(np.float64)
    assert np.isfinite(got).all(), info
    none = ~see.any(axis=2)
    if none.any():
        assert (got.transpose(0, 2, 1, 3)[none] == 0).all(), info
    if dtype == torch.float32:
        assert max_rel(got, ref) <= F32_MAX_REL, info
    else:
        if np.linalg.norm(ref) > 0:
            assert rel_l2(got, ref) <= BF16_REL_L2, info
        bound = rows.bf16_bound(q, r, k, v, x["scale"], mask)
        assert (np.abs(got - ref) <= bound).all(), info + (float((np.abs(got - ref) - bound).max()),)


# ---- window and sinks ----------------------------------------------------------------------------------

SINK_CASES = [  # lengths, Tq, window, sinks
    ((1,), 1, 1, 1), ((2, 1, 0), 1, 1, 1), ((5, 3), 1, 2, 1), ((33, 32, 31), 1, 16, 4), ((100, 64), 1, 31, 32),
    ((700, 129, 1), 1, 100, 33), ((700, 130, 300), 2, 100, 70), ((3000, 1500), 1, 257, 4), ((3000, 20), 4, 64, 130),
    ((900, 7, 64), 9, 33, 5), ((2100, 800), 20, 500, 31), ((300, 299), 1, 5000, 4), ((300, 299), 1, 10, 5000),
    ((256, 128), 1, 128, 128), ((257, 129), 3, 127, 1), ((40, 3), 8, 1, 2), ((5000,), 1, 1024, 4),
]


@pytest.mark.parametrize("lens,Tq,window,sinks", SINK_CASES)
@pytest.mark.parametrize("heads,d", [((4, 2), 128), ((6, 6), 64), ((8, 1), 128), ((32, 2), 64)])
def test_sinks_contiguous(plx, lens, Tq, window, sinks, heads, d):
    cap = max(lens) + 3
    x = _inputs(len(lens), *heads, d, Tq, cap, seed=cap + window, dtype=torch.bfloat16)
    see = [rows.chain(L, Tq, cap, window, sinks) for L in lens]
    lens_t = torch.tensor(lens, dtype=torch.int32, device=DEV)
    for splits in (0, 1, 3):
        got = plx.parallax_decode(x["q"], x["r"], x["k"], x["v"], x["scale"], seq_lens=lens_t, window=window,
                                  sinks=sinks, num_splits=splits)
        _check(got, x, see, info=(lens, Tq, window, sinks, heads, splits))


@pytest.mark.parametrize("page", [16, 24, 64, 5, 1])
@pytest.mark.parametrize("lens,Tq,window,sinks", [((700, 129, 1), 1, 100, 33), ((2100, 800), 20, 500, 31),
                                                  ((257, 129, 0), 3, 127, 1), ((5000, 4000), 1, 1024, 4)])
def test_sinks_paged(plx, lens, Tq, window, sinks, page):
    cap = max(lens)
    x = _inputs(len(lens), 8, 4, 128, Tq, cap, seed=cap + page)
    see = [rows.chain(L, Tq, cap, window, sinks) for L in lens]
    p = _paged(x, page, seed=page)
    got = plx.parallax_decode(p["q"], p["r"], p["k"], p["v"], p["scale"], block_table=p["block_table"], max_len=cap,
                              seq_lens=torch.tensor(lens, dtype=torch.int32, device=DEV), window=window, sinks=sinks)
    _check(got, x, see, info=(lens, page))


def test_sinks_freed_pages(plx):
    """Pages between the sinks and the window are gone: their table entries are negative, the pages others'."""
    lens, window, sinks, page, cap = (1000, 640), 130, 20, 16, 1000
    x = _inputs(2, 8, 4, 128, 1, cap, seed=77)
    see = [rows.chain(L, 1, cap, window, sinks) for L in lens]
    p = _paged(x, page, seed=5)
    table = p["block_table"].clone()
    for b, L in enumerate(lens):
        for n in range(table.shape[1]):
            if n * page >= sinks and (n + 1) * page <= L - window:
                for pool in (p["k"], p["v"]):
                    pool[table[b, n]] = float("inf")
                table[b, n] = -1
    got = plx.parallax_decode(p["q"], p["r"], p["k"], p["v"], p["scale"], block_table=table, max_len=cap,
                              seq_lens=torch.tensor(lens, dtype=torch.int32, device=DEV), window=window, sinks=sinks)
    _check(got, x, see)


@pytest.mark.parametrize("d", [64, 36, 128, 200, 256])
@pytest.mark.parametrize("lens,Tq,window,sinks", SINK_CASES[1:12])
def test_sinks_f32(plx, d, lens, Tq, window, sinks):
    cap = max(lens) + 1
    x = _inputs(len(lens), 6, 2, d, Tq, cap, seed=cap + d, dtype=torch.float32)
    see = [rows.chain(L, Tq, cap, window, sinks) for L in lens]
    lens_t = torch.tensor(lens, dtype=torch.int32, device=DEV)
    for splits in (0, 1, 3):
        got = plx.parallax_decode(x["q"], x["r"], x["k"], x["v"], x["scale"], seq_lens=lens_t, window=window,
                                  sinks=sinks, num_splits=splits)
        _check(got, x, see, torch.float32, (lens, splits))
    p = _paged(x, 24, seed=d)
    got = plx.parallax_decode(p["q"], p["r"], p["k"], p["v"], p["scale"], block_table=p["block_table"], max_len=cap,
                              seq_lens=lens_t, window=window, sinks=sinks)
    _check(got, x, see, torch.float32, (lens, "paged"))


# ---- trees ---------------------------------------------------------------------------------------------

TREE_CASES = [  # lengths, drafted, Tq
    ((1,), None, 1), ((5, 3, 0), (2, 3, 1), 4), ((40, 41), None, 8), ((100, 33, 64), (8, 0, 5), 8),
    ((700, 301), (31, 17), 31), ((1500, 64), None, 64), ((900, 70), (65, 70), 70), ((600, 10), None, 200),
    ((2000, 1023), (3, 16), 16), ((129, 128, 127), None, 33), ((3000,), None, 64),
]


@pytest.mark.parametrize("lens,drafted,Tq", TREE_CASES)
@pytest.mark.parametrize("heads,d", [((4, 2), 128), ((6, 6), 64), ((16, 2), 128), ((32, 2), 64)])
def test_tree_contiguous(plx, lens, drafted, Tq, heads, d):
    B, cap = len(lens), max(lens) + 2
    rng = np.random.default_rng(Tq + cap)
    bits = np.stack([rows.random_tree(Tq, rng) for _ in lens])
    x = _inputs(B, *heads, d, Tq, cap, seed=cap + Tq)
    see = [rows.tree(L, Tq, cap, bits[b], None if drafted is None else drafted[b]) for b, L in enumerate(lens)]
    opts = dict(seq_lens=torch.tensor(lens, dtype=torch.int32, device=DEV),
                draft_lens=None if drafted is None else torch.tensor(drafted, dtype=torch.int32, device=DEV))
    mask = torch.from_numpy(rows.words(bits)).to(DEV)
    for splits in (0, 1, 3):
        got = plx.parallax_decode_tree(x["q"], x["r"], x["k"], x["v"], x["scale"], mask, num_splits=splits, **opts)
        _check(got, x, see, info=(lens, drafted, Tq, splits))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("page", [16, 24, 1])
@pytest.mark.parametrize("lens,drafted,Tq,window,sinks", [((700, 301), (31, 17), 31, 0, 0), ((900, 70), (65, 70), 70, 40, 9),
                                                          ((600, 10, 0), (4, 5, 2), 6, 64, 33), ((400, 399), None, 8, 3, 0),
                                                          ((400, 33), None, 9, 1, 1)])
def test_tree_paged_window(plx, dtype, page, lens, drafted, Tq, window, sinks):
    B, cap = len(lens), max(lens)
    rng = np.random.default_rng(Tq + cap)
    bits = np.stack([rows.random_tree(Tq, rng) for _ in lens])
    x = _inputs(B, 8, 4, 128, Tq, cap, seed=cap + Tq, dtype=dtype)
    see = [rows.tree(L, Tq, cap, bits[b], None if drafted is None else drafted[b], window, sinks)
           for b, L in enumerate(lens)]
    p = _paged(x, page, seed=page)
    got = plx.parallax_decode_tree(
        p["q"], p["r"], p["k"], p["v"], p["scale"], torch.from_numpy(rows.words(bits)).to(DEV),
        seq_lens=torch.tensor(lens, dtype=torch.int32, device=DEV), block_table=p["block_table"], max_len=cap,
        draft_lens=None if drafted is None else torch.tensor(drafted, dtype=torch.int32, device=DEV),
        window=window, sinks=sinks)
    _check(got, x, see, dtype, (lens, page))


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 64), (torch.float32, 64), (torch.float32, 132)])
def test_tree_any_mask(plx, dtype, d):
    """Masks that are no tree: nodes that see nothing at all without committed keys, nodes that see later ones."""
    Tq, lens = 20, (20, 150)
    rng = np.random.default_rng(3)
    bits = rng.random((2, Tq, Tq)) < 0.3
    bits[:, 4] = False
    x = _inputs(2, 4, 2, d, Tq, 150, seed=8, dtype=dtype)
    see = [rows.tree(L, Tq, 150, bits[b]) for b, L in enumerate(lens)]
    got = plx.parallax_decode_tree(x["q"], x["r"], x["k"], x["v"], x["scale"], torch.from_numpy(rows.words(bits)).to(DEV),
                                   seq_lens=torch.tensor(lens, dtype=torch.int32, device=DEV))
    _check(got, x, see, dtype)
    shared = plx.parallax_decode_tree(x["q"], x["r"], x["k"], x["v"], x["scale"],
                                      torch.from_numpy(rows.words(bits[0])).to(DEV),
                                      seq_lens=torch.tensor(lens, dtype=torch.int32, device=DEV))
    _check(shared, x, [rows.tree(L, Tq, 150, bits[0]) for L in lens], dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_unseen_keys_hold_anything(plx, dtype):
    """Infinities and NaN in a drafted key reach the nodes that see it, and no other; rows behind the sequence none."""
    Tq, L, cap = 12, 90, 128
    rng = np.random.default_rng(9)
    bits = rows.random_tree(Tq, rng)
    bits[:, 7] = False
    bits[7, 7] = True  # node 7 is seen by itself only
    x = _inputs(1, 4, 2, 64, Tq, cap, seed=21, dtype=dtype)
    see = rows.tree(L, Tq, cap, bits)[None]
    at = L - Tq + 7
    lens = torch.tensor([L], dtype=torch.int32, device=DEV)
    mask = torch.from_numpy(rows.words(bits)).to(DEV)
    for bad in (float("nan"), float("inf"), float("-inf")):
        for names in (("k",), ("v",), ("k", "v")):
            y = dict(x, k=x["k"].clone(), v=x["v"].clone())
            for n in names:
                y[n][:, :, at, ::3] = bad
                y[n][:, :, L:] = bad
            for splits in (1, 3):
                got = plx.parallax_decode_tree(y["q"], y["r"], y["k"], y["v"], y["scale"], mask, seq_lens=lens,
                                               num_splits=splits)
                others = [t for t in range(Tq) if t != 7]
                z = dict(x, q=x["q"][:, :, others], r=x["r"][:, :, others])
                _check(got[:, :, others], z, see[:, others], dtype, (bad, names, splits))
                assert not torch.isfinite(got[:, :, 7]).all(), (bad, names, splits)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_chain_as_a_tree(plx, dtype):
    """The mask of a chain gives what the decode over the last Tq positions gives."""
    Tq, lens = 6, torch.tensor([500, 77], dtype=torch.int32, device=DEV)
    x = _inputs(2, 8, 4, 128, Tq, 500, seed=31, dtype=dtype)
    mask = torch.tensor([(1 << (t + 1)) - 1 for t in range(Tq)], dtype=torch.int64, device=DEV)
    a = plx.parallax_decode_tree(x["q"], x["r"], x["k"], x["v"], x["scale"], mask, seq_lens=lens)
    b = plx.parallax_decode(x["q"], x["r"], x["k"], x["v"], x["scale"], seq_lens=lens)
    assert rel_l2(host(a), host(b).astype(np.float64)) <= (BF16_REL_L2 if dtype == torch.bfloat16 else F32_MAX_REL)


def test_twin_and_strides(plx):
    """The softmax-only twin, and caches with gaps between rows and heads (row by row where they are too far apart)."""
    Tq, lens, cap = 7, (300, 200), 300
    rng = np.random.default_rng(2)
    bits = np.stack([rows.random_tree(Tq, rng) for _ in lens])
    mask, lens_t = torch.from_numpy(rows.words(bits)).to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV)
    for dtype in (torch.bfloat16, torch.float32):
        x = _inputs(2, 8, 4, 64, Tq, cap, seed=41, dtype=dtype)
        see = [rows.tree(L, Tq, cap, bits[b]) for b, L in enumerate(lens)]
        got = plx.parallax_decode_tree(x["q"], None, x["k"], x["v"], x["scale"], mask, seq_lens=lens_t, use_r=False)
        _check(got, dict(x, r=torch.zeros_like(x["r"])), see, dtype)
        wide = _normal((2, cap, 4, 72), 5, dtype)[..., :64].transpose(1, 2)
        y = dict(x, k=wide, v=_normal((2, 4, cap, 80), 6, dtype)[..., 8:72])
        got = plx.parallax_decode_tree(y["q"], y["r"], y["k"], y["v"], y["scale"], mask, seq_lens=lens_t)
        _check(got, y, see, dtype)


def test_offsets_past_32_bits(plx):
    """A pool of more than 2^32 bytes: the pages of the sequence are its last ones."""
    page, Hkv, d, n = 64, 8, 128, 40000  # 2^32.3 elements' bytes
    need = 2 * n * Hkv * page * d * 2
    if torch.cuda.mem_get_info()[0] < 1.2 * need:
        pytest.skip("needs %d GB" % (need >> 30))
    k = torch.zeros(n, Hkv, page, d, dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    cap, Tq = 150, 5
    x = _inputs(1, 16, 8, d, Tq, cap, seed=51)
    table = torch.tensor([[n - 1, n - 7, n - 3]], dtype=torch.int32, device=DEV)
    for b in range(3):
        rows_here = min(page, cap - b * page)
        for pool, name in ((k, "k"), (v, "v")):
            pool[table[0, b], :, :rows_here] = x[name][0, :, b * page: b * page + rows_here]
    bits = rows.random_tree(Tq, np.random.default_rng(1))
    got = plx.parallax_decode_tree(x["q"], x["r"], k, v, x["scale"], torch.from_numpy(rows.words(bits)).to(DEV),
                                   block_table=table, max_len=cap)
    _check(got, x, rows.tree(cap, Tq, cap, bits)[None])


def test_graph_and_stream(plx):
    """Captured calls replayed with new lengths, between eager work; a call on another stream."""
    Tq, cap = 9, 800
    bits = rows.random_tree(Tq, np.random.default_rng(4))
    mask = torch.from_numpy(rows.words(bits)).to(DEV)
    x = _inputs(2, 16, 8, 128, Tq, cap, seed=61)
    lens = torch.tensor([800, 700], dtype=torch.int32, device=DEV)
    q1, r1 = x["q"][:, :, 0].contiguous(), x["r"][:, :, 0].contiguous()

    def calls():
        return (plx.parallax_decode_tree(x["q"], x["r"], x["k"], x["v"], x["scale"], mask, seq_lens=lens),
                plx.parallax_decode(q1, r1, x["k"], x["v"], x["scale"], seq_lens=lens, window=100, sinks=4))

    calls()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = calls()
    for new in ([800, 700], [333, 10], [9, 800], [1, 0]):
        lens.copy_(torch.tensor(new, dtype=torch.int32, device=DEV))
        want = calls()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b), new
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    other = plx.parallax_decode_tree(x["q"], x["r"], x["k"], x["v"], x["scale"], mask, seq_lens=lens, stream=side)
    side.synchronize()
    assert torch.equal(other, outs[0])


def test_same_bits_every_time(plx):
    x = _inputs(3, 16, 8, 128, 5, 3000, seed=71)
    mask = torch.from_numpy(rows.words(rows.random_tree(5, np.random.default_rng(4)))).to(DEV)
    first = plx.parallax_decode_tree(x["q"], x["r"], x["k"], x["v"], x["scale"], mask)
    for _ in range(5):
        assert torch.equal(first, plx.parallax_decode_tree(x["q"], x["r"], x["k"], x["v"], x["scale"], mask))


def test_tree_mask_words(plx):
    rng = np.random.default_rng(6)
    for Tq in (1, 5, 64, 70, 200):
        parents = np.array([[int(rng.integers(max(-1, t - 9), t)) if t else -1 for t in range(Tq)] for _ in range(3)])
        bits = np.zeros((3, Tq, Tq), dtype=bool)
        for b in range(3):
            for t in range(Tq):
                if parents[b, t] >= 0:
                    bits[b, t] = bits[b, parents[b, t]]
                bits[b, t, t] = True
        got = plx.tree_mask_words(torch.from_numpy(parents).to(DEV))
        np.testing.assert_array_equal(got.cpu().numpy(), rows.words(bits))
