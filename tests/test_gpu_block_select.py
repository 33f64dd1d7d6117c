"""GPU parity of block bounds and selection (through the C ABI) against the CPU oracle, and of a whole sparse step."""
import numpy as np
import pytest
import torch

from oracle import blocks, masked, rows
from parity import host

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def plx():
    from paper_2605_29157_amd import binding

    binding.load_library()
    assert torch.cuda.is_available()
    return binding


def _normal(shape, seed, dtype=torch.bfloat16):
    gen = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=gen).to(dtype).to(DEV)


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _paged(x, page, seed, fill):
    """[B, Hkv, cap, row] -> pools of shuffled pages, block table"""
    B, Hkv, cap, row = x.shape
    per = -(-cap // page)
    order = torch.from_numpy(np.random.default_rng(seed).permutation(B * per + 3)[: B * per]).to(DEV)
    pool = torch.full((B * per + 3, Hkv, page, row), fill, dtype=x.dtype, device=DEV)
    padded = torch.full((B, Hkv, per * page, row), fill, dtype=x.dtype, device=DEV)
    padded[:, :, :cap] = x
    pool[order] = padded.reshape(B, Hkv, per, page, row).transpose(1, 2).reshape(B * per, Hkv, page, row)
    return pool, order.reshape(B, per).to(torch.int32)


def _same(a, b):
    return torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("page", [0, 16, 24, 64])
@pytest.mark.parametrize("d", [64, 128])
def test_bounds(plx, d, page, four):
    lens = (1, 63, 64, 65, 300, 0, 500)
    B, Hkv, cap = len(lens), 2, 500
    k = _normal((B, Hkv, cap, d), 1)
    for b, n in enumerate(lens):
        k[b, :, n:] = 1e30  # (rows that nobody has written)
    if four:
        cache = torch.zeros((B, Hkv, cap, blocks.row_bytes(d)), dtype=torch.uint8, device=DEV)
        plx.parallax_cache_write_q4(k, k, cache)
        k = plx.parallax_cache_read_q4(cache, d, cap)[0]
    keys = cache if four else k
    more = {}
    if page:
        keys, table = _paged(keys, page, 2, 200 if four else float("nan"))
        more = dict(block_table=table)
    n_blocks = 9
    out = torch.full((B, Hkv, n_blocks, 2, d), 7.0, dtype=torch.bfloat16, device=DEV)
    want = host(out)
    hk = host(k)
    for b, n in enumerate(lens):
        for h in range(Hkv):
            low, high = blocks.bounds(hk[b, h], n)
            if n:
                want[b, h, :len(low), 0], want[b, h, :len(low), 1] = low, high
    got = plx.parallax_cache_bounds(keys, out, _ints(lens), **more)
    assert got is out and np.array_equal(host(out), want)
    # only what is new: 70 more tokens, the other blocks stay as they are
    old = (0, 1, 0, 64, 230, 0, 431)
    out.fill_(7.0)
    plx.parallax_cache_bounds(keys, out, _ints(lens), from_lens=_ints(old), max_new=70, **more)
    for b, n in enumerate(old):
        want[b, :, : n // 64] = 7.0
        if lens[b] <= n // 64 * 64:
            want[b] = 7.0
    assert np.array_equal(host(out), want)


def test_bounds_of_not_finite_keys(plx):
    k = _normal((1, 1, 130, 64), 1)
    k[0, 0, 3, 5], k[0, 0, 70, 6], k[0, 0, 71, 7] = float("nan"), float("inf"), float("-inf")
    k[0, 0, 129, 9] = float("-nan")
    out = plx.parallax_cache_bounds(k, torch.zeros(1, 1, 3, 2, 64, dtype=torch.bfloat16, device=DEV))
    low, high = host(out)[0, 0, :, 0], host(out)[0, 0, :, 1]
    assert np.isnan(low[0, 5]) or np.isnan(high[0, 5])
    assert high[1, 6] == np.inf and low[1, 7] == -np.inf
    assert np.isnan(low[2, 9]) or np.isnan(high[2, 9])
    bad = np.zeros((3, 2, 64), dtype=bool)
    bad[0, :, 5], bad[1, :, 6], bad[1, :, 7], bad[2, :, 9] = True, True, True, True
    assert np.isfinite(np.where(bad, 0, host(out)[0, 0])).all()


SELECT = [  # lengths, Hq, Hkv, d, Tq, keep, first, recent
    ((1, 0, 64), 2, 2, 128, 1, 1, 0, 1), ((640, 641, 63), 4, 2, 64, 1, 10, 1, 2), ((5000, 2000), 16, 8, 128, 1, 12, 1, 2),
    ((5000, 3333), 4, 1, 64, 4, 7, 2, 4), ((3000,), 16, 1, 128, 1, 5, 0, 0), ((9000, 8000), 2, 2, 64, 3, 6, 2, 4),
    ((40000, 35000), 4, 2, 128, 2, 100, 1, 2), ((40000,), 3, 1, 64, 1, 1, 0, 0), ((40000,), 8, 8, 64, 1, 620, 1, 1),
]


@pytest.mark.parametrize("case", SELECT, ids=str)
def test_select(plx, case):
    lens, Hq, Hkv, d, Tq, keep, first, recent = case
    B, n_blocks = len(lens), -(-max(lens) // 64) + 1
    a = _normal((B, Hkv, n_blocks, d), 1).float()
    bounds = torch.stack([a - 2, a + 2], 3).to(torch.bfloat16)
    for b, n in enumerate(lens):
        bounds[b, :, -(-n // 64):] = float("nan")
    q = _normal((B, Hq, Tq, d), 2)
    got = plx.parallax_select_blocks(q if Tq > 1 else q[:, :, 0].contiguous(), bounds, _ints(lens), keep, first=first, recent=recent)
    assert got.shape == (B, Hkv, keep) and got.dtype == torch.int32
    hq, hb = host(q).reshape(B, Hkv, -1, d), host(bounds)
    for b, n in enumerate(lens):
        for h in range(Hkv):
            held = -(-n // 64)
            want = blocks.select(hq[b, h], hb[b, h, :held, 0], hb[b, h, :held, 1], keep, first, recent) if held else []
            assert got[b, h].tolist() == want + [-1] * (keep - len(want)), (b, h)


def test_select_ties_and_not_finite(plx):
    """Few different scores (so that the last place is shared), equal ones throughout, negative ones, NaN and infinite bounds."""
    d, n = 64, 700
    rng = np.random.default_rng(0)
    bounds = torch.zeros((6, 1, n, 2, d), dtype=torch.bfloat16, device=DEV)
    bounds[0, 0, :, 1, 0] = torch.from_numpy(rng.integers(0, 5, n)).to(DEV)
    bounds[2, 0, :, :, 0] = -torch.from_numpy(rng.integers(1, 9, n)).to(DEV).float()[:, None].to(torch.bfloat16)
    bounds[3, 0, :, 1, 0] = torch.from_numpy(rng.integers(0, 5, n)).to(DEV)
    bounds[3, 0, 77, 0, 9], bounds[3, 0, 500, 1, 3] = float("nan"), float("inf")
    bounds[4, 0, :, 1, 0] = (2.0 ** torch.from_numpy(rng.integers(-60, 60, n)).to(DEV).double()).to(torch.bfloat16)
    bounds[5, 0, :, 1, 0], bounds[5, 0, :, 1, 1] = 2.0 ** 20, torch.arange(n, device=DEV).to(torch.bfloat16) * 2.0 ** -12
    q = torch.zeros((6, 1, d), dtype=torch.bfloat16, device=DEV)
    q[:, :, 0], q[:, :, 1] = 1.0, 2.0 ** -6
    got = plx.parallax_select_blocks(q, bounds, None, 50, first=1, recent=2)
    for b in range(6):
        hb = host(bounds[b, 0])
        assert got[b, 0].tolist() == blocks.select(host(q[b]), hb[:, 0], hb[:, 1], 50, 1, 2), b


def _sees(lists, lens, Tq, cap):
    return np.stack([np.stack([rows.chain(n, Tq, cap) & blocks.listed_keys(x, n, cap) for x in lists[b]]) for b, n in enumerate(lens)])


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("page", [0, 16, 24])
def test_steps_of_a_sequence(plx, page, four):
    """Tokens appended one by one: rows written, bounds brought up to date, blocks selected, attention over them, captured into one
    graph and replayed for every token."""
    B, Hq, Hkv, d, cap, keep = 2, 4, 2, 128, 600, 4
    k, v = _normal((B, Hkv, cap, d), 1), _normal((B, Hkv, cap, d), 2)
    if four:
        rows_now = torch.zeros((B, Hkv, cap, blocks.row_bytes(d)), dtype=torch.uint8, device=DEV)
        plx.parallax_cache_write_q4(k, v, rows_now)
        k, v = plx.parallax_cache_read_q4(rows_now, d, cap)
        rows_now[:, :, 300:] = 0xff
    more, table = {}, None
    if page:
        if four:
            rows_now, table = _paged(rows_now, page, 3, 0xff)
        else:
            kp, table = _paged(k, page, 3, float("nan"))
            vp, _ = _paged(v, page, 3, float("nan"))
        more = dict(block_table=table)
    n_blocks = -(-(table.shape[1] * page if page else cap) // 64)
    bounds = torch.zeros((B, Hkv, n_blocks, 2, d), dtype=torch.bfloat16, device=DEV)
    lens, before = _ints([290, 255]), _ints([0, 0])
    keys = rows_now if four else (kp if page else k)
    plx.parallax_cache_bounds(keys, bounds, lens, **more)
    before.copy_(lens)
    new_k, new_v = torch.empty((2, B, Hkv, 1, d), dtype=torch.bfloat16, device=DEV)
    q, r = torch.empty((2, B, Hq, d), dtype=torch.bfloat16, device=DEV)
    out, names = torch.empty_like(q), torch.empty((B, Hkv, keep), dtype=torch.int32, device=DEV)
    ws = torch.empty(1 << 20, dtype=torch.float32, device=DEV)

    def step():
        if four:
            plx.parallax_cache_write_q4(new_k, new_v, rows_now, start=before, **more)
        plx.parallax_cache_bounds(keys, bounds, lens, from_lens=before, max_new=1, **more)
        plx.parallax_select_blocks(q, bounds, lens, keep, first=1, recent=1, out=names, workspace=ws[: 1 << 14])
        args = dict(seq_lens=lens, block_list=names, out=out, workspace=ws[1 << 14:], **more)
        if four:
            plx.parallax_decode_q4(q, r, rows_now, d ** -0.5, **args)
        else:
            plx.parallax_decode(q, r, *((kp, vp) if page else (k, v)), d ** -0.5, **args)
        before.copy_(lens)

    graph = None
    hk, hv = host(k), host(v)
    for n in range(6):
        lens += 1
        at = (lens - 1).tolist()
        new_k.copy_(torch.stack([k[b, :, i] for b, i in enumerate(at)])[:, :, None])
        new_v.copy_(torch.stack([v[b, :, i] for b, i in enumerate(at)])[:, :, None])
        q.copy_(_normal((B, Hq, d), 100 + n))
        r.copy_(_normal((B, Hq, d), 200 + n))
        if n < 2:
            step()
        else:
            if graph is None:
                graph = torch.cuda.CUDAGraph()
                kept = before.clone()
                with torch.cuda.graph(graph):
                    step()
                before.copy_(kept)
            graph.replay()
        torch.cuda.synchronize()
        now = lens.tolist()
        hq = host(q).reshape(B, Hkv, -1, d)
        for b in range(B):
            for h in range(Hkv):
                low, high = blocks.bounds(hk[b, h], now[b])
                got = host(bounds[b, h])
                assert np.array_equal(got[:len(low), 0], low) and np.array_equal(got[:len(low), 1], high), (n, b, h)
                assert names[b, h].tolist() == blocks.select(hq[b, h], low, high, keep, 1, 1), (n, b, h)
        see = _sees(names.tolist(), now, 1, cap)
        mask = np.repeat(see, Hq // Hkv, axis=1)
        ref = masked.masked_forward(host(q)[:, :, None], host(r)[:, :, None], hk, hv, d ** -0.5, mask)
        bound = rows.bf16_bound(host(q)[:, :, None], host(r)[:, :, None], hk, hv, d ** -0.5, mask)
        assert (np.abs(host(out)[:, :, None] - ref) <= bound).all(), n


@pytest.mark.parametrize("n", [240, 255, 256, 257])
@pytest.mark.parametrize("d", [64, 128])
def test_select_around_one_round(plx, d, n):
    """As many blocks as a workgroup scores at once, and one more; every place of a row holds the value that is not finite once."""
    B, keep = 4, 9
    a = _normal((B, 2, n, d), 7).float()
    bounds = torch.stack([a - 1.5, a + 1.5], 3).to(torch.bfloat16)
    for i, bad in enumerate((float("inf"), -float("inf"), float("nan"))):
        for h in range(2):
            bounds[i, h, 3 + 37 * h + torch.arange(4) * 50, (i + h) % 2, (torch.arange(4) * 17 + 31 * h + 5 * i) % d] = bad
    q = _normal((B, 4, d), 8)
    got = plx.parallax_select_blocks(q, bounds, None, keep, first=0, recent=1)
    hq, hb = host(q).reshape(B, 2, -1, d), host(bounds)
    for b in range(B):
        for h in range(2):
            assert got[b, h].tolist() == blocks.select(hq[b, h], hb[b, h, :, 0], hb[b, h, :, 1], keep, 0, 1), (b, h)


@pytest.mark.parametrize("four", [False, True])
def test_bounds_are_not_cut_unasked(plx, four):
    """A block table with more pages than bounds have room for is refused like a contiguous cache of that length, unless max_len says that
    no sequence is that long; pages that only round a length up are not."""
    d, page, L = 64, 16, 300
    k = _normal((1, 1, 400, d), 1)
    if four:
        keys = torch.zeros((1, 1, 400, blocks.row_bytes(d)), dtype=torch.uint8, device=DEV)
        plx.parallax_cache_write_q4(k, k, keys)
        k = plx.parallax_cache_read_q4(keys, d, 400)[0]
    else:
        keys = k
    pools, table = _paged(keys, page, 2, 200 if four else float("nan"))
    assert table.shape[1] == 25
    few = torch.full((1, 1, 5, 2, d), 7.0, dtype=torch.bfloat16, device=DEV)
    lens = _ints([L])
    for more in (dict(), dict(max_len=321), dict(max_len=0), dict(max_len=-1)):
        with pytest.raises(ValueError):
            plx.parallax_cache_bounds(pools, few, lens, block_table=table, **more)
    with pytest.raises(ValueError):
        plx.parallax_cache_bounds(keys, few, lens, max_len=401)
    assert (few == 7.0).all()
    low, high = blocks.bounds(host(k)[0, 0], L)
    for more in (dict(max_len=320), dict(max_len=L)):
        few.fill_(7.0)
        plx.parallax_cache_bounds(pools, few, lens, block_table=table, **more)
        assert np.array_equal(host(few)[0, 0, :, 0], low) and np.array_equal(host(few)[0, 0, :, 1], high)
    # 20 pages for 301 .. 320 tokens, 21 for the first of the sixth block
    plx.parallax_cache_bounds(pools, few, lens, block_table=table[:, :20].contiguous())
    assert np.array_equal(host(few)[0, 0, :, 0], low)
    with pytest.raises(ValueError):
        plx.parallax_cache_bounds(pools, few, lens, block_table=table[:, :21].contiguous())
    # a contiguous cache of which a part is looked at
    few.fill_(7.0)
    plx.parallax_cache_bounds(keys, few, lens, max_len=320)
    assert np.array_equal(host(few)[0, 0, :, 1], high)


@pytest.mark.parametrize("n_blocks", [40, 300])
@pytest.mark.parametrize("d", [64, 128])
def test_equal_sums_in_any_order_are_equal(plx, d, n_blocks):
    """Blocks whose bounds are the same numbers in other dimensions, with products up to 2^30 of each other: equal scores, so the lower
    numbers are kept."""
    rng = np.random.default_rng(d)
    x = rng.integers(128, 256, d) * np.exp2(rng.integers(-29, 1, d).astype(np.float64)) * rng.choice([-1, 1], d)
    x[0], x[1] = 255.0, 128.0 * 2.0 ** -29
    q = torch.full((1, 1, d), 255.0 / 128, dtype=torch.bfloat16, device=DEV)
    b = np.stack([rng.permutation(x) for _ in range(n_blocks)])
    bounds = torch.tensor(np.stack([b, b], 1)[None, None], dtype=torch.bfloat16, device=DEV)
    assert np.array_equal(host(bounds)[0, 0, :, 0], b)
    got = plx.parallax_select_blocks(q, bounds, None, 7, first=0, recent=0)
    assert got.flatten().tolist() == list(range(7))
