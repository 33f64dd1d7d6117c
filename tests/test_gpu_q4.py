"""GPU parity of the 4-bit cache (through the C ABI) against the CPU oracle: rows written and read back, decode over them."""
import numpy as np
import pytest
import torch

from oracle import blocks, masked, rows
from parity import BF16_REL_L2, host, rel_l2

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


def _cache(B, Hkv, cap, d, seed, spread=2):
    """A 4-bit cache of random codes whose scales lie within `spread` powers of two of each other (values about N(0, 1))."""
    rng = np.random.default_rng(seed)
    x = rng.integers(0, 256, (B, Hkv, cap, blocks.row_bytes(d)), dtype=np.uint8)
    x[..., d:] = rng.integers(127 - 1 - spread, 127, x[..., d:].shape)
    x[..., d + d // 8:] = 0
    return x


def _paged(cache, page, seed, fill=0xff):
    """numpy cache [B, Hkv, cap, row] -> pools of shuffled pages with `fill` in what no token has, block table"""
    B, Hkv, cap, row = cache.shape
    per = -(-cap // page)
    order = np.random.default_rng(seed).permutation(B * per + 3)[: B * per]
    pool = np.full((B * per + 3, Hkv, page, row), fill, dtype=np.uint8)
    padded = np.full((B, Hkv, per * page, row), fill, dtype=np.uint8)
    padded[:, :, :cap] = cache
    pool[order] = padded.reshape(B, Hkv, per, page, row).transpose(0, 2, 1, 3, 4).reshape(B * per, Hkv, page, row)
    return torch.from_numpy(pool).to(DEV), torch.tensor(order.reshape(B, per), dtype=torch.int32, device=DEV)


def _check(got, q, r, k, v, scale, see, info=()):
    """see [B, Hkv or 1, Tq, cap]"""
    B, Hq = q.shape[:2]
    see = np.broadcast_to(see, (B, k.shape[1]) + see.shape[2:])
    mask = np.repeat(see, Hq // k.shape[1], axis=1)
    used = see.any(axis=2)[..., None]
    k, v = (np.where(used, np.nan_to_num(x), 0.0) for x in (k, v))
    ref = masked.masked_forward(q, r, k, v, scale, mask)
    got = host(got).astype(np.float64).reshape(q.shape)
    assert np.isfinite(got).all(), info
    none = ~mask.any(axis=3)
    assert (got[none] == 0).all(), info
    if np.linalg.norm(ref) > 0:
        assert rel_l2(got, ref) <= BF16_REL_L2, info
    bound = rows.bf16_bound(q, r, k, v, scale, mask)
    assert (np.abs(got - ref) <= bound).all(), info + (float((np.abs(got - ref) - bound).max()),)


# ---- rows -------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_are_the_oracles(plx, d, dtype):
    """Every byte: ordinary values, halfway ones, tiny, huge, infinite and NaN ones, zeros of either sign."""
    rng = np.random.default_rng(d)
    T = 40
    x = rng.standard_normal((2, 1, 2, T, d)) * np.exp2(rng.integers(-3, 4, (2, 1, 2, T, d // 16, 1)).repeat(16, -1)).reshape(2, 1, 2, T, d)
    x[:, :, :, 1] = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -2.5, -5.0], x[:, :, :, 1].shape)
    x[:, :, :, 2] = 0.0
    x[:, :, :, 3] = -0.0
    x[:, :, :, 4] *= 2.0 ** -124
    x[:, :, :, 5] *= 2.0 ** -140
    x[:, :, :, 6] = 3.3e38 * rng.uniform(-1, 1, x[:, :, :, 6].shape)
    x[:, :, :, 7, 3] = np.inf
    x[:, :, :, 7, 17] = -np.inf
    x[:, :, :, 8, 5] = np.nan
    x[:, :, :, 9, :] = 7.0
    x[:, :, :, 10, :16] = np.nextafter(np.float32(7.0), np.float32(0))
    k, v = (torch.tensor(y).to(dtype).to(DEV) for y in x)
    cache = torch.full((1, 2, T + 3, blocks.row_bytes(d)), 0xa5, dtype=torch.uint8, device=DEV)
    start = torch.tensor([2], dtype=torch.int32, device=DEV)
    plx.parallax_cache_write_q4(k, v, cache, start=start)
    got = cache.cpu().numpy()
    assert (got[:, :, :2] == 0xa5).all() and (got[:, :, T + 2:] == 0xa5).all()
    hk, hv = (y.double().cpu().numpy() for y in (k, v))
    for h in range(2):
        for t in range(T):
            want = blocks.pack_row(hk[0, h, t], hv[0, h, t])
            assert np.array_equal(got[0, h, t + 2], want), (h, t)
    for out in (torch.bfloat16, torch.float32):
        back = plx.parallax_cache_read_q4(cache, d, T, start=start, dtype=out)
        for y, want in zip(back, blocks.unpack(got[:, :, 2: T + 2], d)):
            assert y.dtype == out and np.array_equal(y.double().cpu().numpy(), want, equal_nan=True)


@pytest.mark.parametrize("page", [0, 1, 16, 24])
@pytest.mark.parametrize("d,T", [(128, 1), (64, 1), (128, 70), (64, 33)])
def test_rows_go_where_they_belong(plx, d, T, page):
    """Ragged starts and counts, strides with gaps, positions outside the cache, entries that are no page; everything else stays."""
    B, Hkv, cap = 4, 3, 100
    wide = _normal((2, B, T, Hkv, 2 * d), 5)
    k, v = (wide[i].transpose(1, 2)[..., d // 2: d // 2 + d] for i in (0, 1))
    start = torch.tensor([0, 37, 90, -2], dtype=torch.int32, device=DEV)
    counts = torch.tensor([T, max(T - 5, 1), T, T], dtype=torch.int32, device=DEV)
    before = _cache(B, Hkv, cap, d, 3)
    if page:
        pool, table = _paged(before, page, 4)
        table[1, 40 // page] = -1
        table[0, 0] = 10 ** 6
        target, more = pool, dict(block_table=table)
        capacity = table.shape[1] * page
    else:
        target, more, capacity = torch.from_numpy(before).to(DEV), {}, cap
    want = target.cpu().numpy().copy()
    hk, hv = host(k), host(v)
    expect = np.zeros((2, B, Hkv, T, d))
    for b in range(B):
        for t in range(T):
            pos = int(start[b]) + t
            if not 0 <= pos < capacity:
                continue
            if page:
                n = int(table[b, pos // page])
                if not 0 <= n < pool.shape[0]:
                    continue
                at = (n, slice(None), pos % page)
            else:
                at = (b, slice(None), pos)
            if t < int(counts[b]):
                want[at] = np.stack([blocks.pack_row(hk[b, h, t], hv[b, h, t]) for h in range(Hkv)])
            expect[:, b, :, t] = np.nan_to_num(np.stack(blocks.unpack(want[at], d)), nan=-1)
    plx.parallax_cache_write_q4(k, v, target, start=start, counts=counts, **more)
    assert np.array_equal(target.cpu().numpy(), want)
    back = plx.parallax_cache_read_q4(target, d, T, start=start, **more)
    for i in (0, 1):
        assert np.array_equal(np.nan_to_num(back[i].double().cpu().numpy(), nan=-1), expect[i])
    lens = torch.tensor([1, 50, 95, 0], dtype=torch.int32, device=DEV)
    back = plx.parallax_cache_read_q4(target, d, T, start=start, seq_lens=lens, **more)
    inside = (start[:, None] + torch.arange(T, device=DEV) < lens[:, None]).cpu().numpy()[:, None, :, None]
    for i in (0, 1):
        assert np.array_equal(np.nan_to_num(back[i].double().cpu().numpy(), nan=-1), np.where(inside, expect[i], 0.0))


# ---- decode -----------------------------------------------------------------------------------------------

DECODE = [  # lengths, Hq, Hkv, d, Tq, window, sinks
    ((1,), 2, 2, 128, 1, 0, 0), ((1, 2, 0), 4, 2, 64, 1, 0, 0), ((31, 32, 33), 4, 4, 128, 1, 0, 0),
    ((700, 129, 1), 16, 8, 128, 1, 0, 0), ((700, 130, 300), 8, 4, 64, 2, 0, 0), ((3000, 1500), 4, 1, 128, 4, 0, 0),
    ((257, 3), 16, 1, 64, 1, 0, 0), ((900, 7, 64), 4, 2, 128, 8, 0, 0), ((2500,), 2, 2, 64, 1, 0, 0),
    ((700, 129, 1), 4, 2, 128, 1, 100, 33), ((3000, 20), 8, 2, 64, 4, 64, 130), ((900, 40), 4, 2, 128, 3, 33, 0),
    ((256, 128), 2, 1, 128, 1, 128, 128), ((300, 299), 2, 2, 64, 2, 5000, 4), ((5, 2), 4, 2, 128, 4, 2, 1),
]


@pytest.mark.parametrize("page", [0, 16, 24, 7])
@pytest.mark.parametrize("case", DECODE, ids=str)
def test_decode(plx, case, page):
    lens, Hq, Hkv, d, Tq, window, sinks = case
    B, cap = len(lens), max(lens) + 5
    cache = _cache(B, Hkv, cap, d, 11)
    for b, n in enumerate(lens):
        cache[b, :, n:] = 0xff  # (what no token has written: NaN scales)
    q, r = _normal((B, Hq, Tq, d), 1), _normal((B, Hq, Tq, d), 2)
    if page:
        target, table = _paged(cache, page, 3)
        more = dict(block_table=table, max_len=cap)
    else:
        target, more = torch.from_numpy(cache).to(DEV), {}
    seq = torch.tensor(lens, dtype=torch.int32, device=DEV)
    see = np.stack([rows.chain(n, Tq, cap, window, sinks) for n in lens])[:, None]
    k, v = blocks.unpack(cache, d)
    args = (q[:, :, 0].contiguous(), r[:, :, 0].contiguous()) if Tq == 1 else (q, r)
    for use_r, S in ((True, 0), (True, 1), (True, 5), (False, 3)):
        got = plx.parallax_decode_q4(*args, target, d ** -0.5, seq_lens=seq, use_r=use_r, num_splits=S, window=window, sinks=sinks, **more)
        hr = host(r) if use_r else np.zeros_like(host(r))
        _check(got, host(q), hr, k, v, d ** -0.5, see, (case, page, use_r, S))


@pytest.mark.parametrize("page", [0, 16, 64, 24])
@pytest.mark.parametrize("d,Tq", [(128, 1), (64, 1), (128, 4), (64, 2)])
def test_decode_over_lists(plx, d, Tq, page):
    """Entries that are no block, listed twice, out of order, at the end of a sequence; a head whose list names nothing."""
    lens = (1000, 640, 65, 64, 0, 1)
    B, Hq, Hkv, cap = len(lens), 4, 2, 1010
    cache = _cache(B, Hkv, cap, d, 21)
    for b, n in enumerate(lens):
        cache[b, :, n:] = 0xff
    lists = np.array([[0, 3, 7, 15, -1, -1, -1, -1], [15, -1, 2, 2, 5, 16, 10 ** 9, -2 ** 31]] +
                     [[0, 1, 2, 3, 4, 5, 6, 9], [-1] * 8] + [[1] + [-1] * 7, [0, 1, 2, 3, -1, -1, -1, -1]] +
                     [[0] + [0] * 7, [-5, -3, -1, 0, 0, 1, 2, 3]] + [[0] * 8] * 2 + [[0, 1, 2, 3, 4, 5, 6, 7]] * 2, dtype=np.int64)
    lists = lists.reshape(B, Hkv, 8)
    q, r = _normal((B, Hq, Tq, d), 31), _normal((B, Hq, Tq, d), 32)
    see = np.zeros((B, Hkv, Tq, cap), dtype=bool)
    for b, n in enumerate(lens):
        causal = rows.chain(n, Tq, cap)
        for h in range(Hkv):
            see[b, h] = causal & blocks.listed_keys(lists[b, h].tolist(), n, cap)
            cache[b, h, ~see[b, h].any(0)] = 0xff  # (what lies in other blocks reaches nothing)
    if page:
        target, table = _paged(cache, page, 3)
        more = dict(block_table=table, max_len=cap)
    else:
        target, more = torch.from_numpy(cache).to(DEV), {}
    seq = torch.tensor(lens, dtype=torch.int32, device=DEV)
    names = torch.tensor(lists, dtype=torch.int32, device=DEV)
    k, v = blocks.unpack(cache, d)
    for use_r, S in ((True, 0), (True, 1), (True, 3), (False, 2)):
        got = plx.parallax_decode_q4(q, r, target, d ** -0.5, seq_lens=seq, use_r=use_r, num_splits=S, block_list=names, **more)
        hr = host(r) if use_r else np.zeros_like(host(r))
        _check(got, host(q), hr, k, v, d ** -0.5, see, (page, use_r, S))
    # ... and the same over bf16 keys and values, which read NaN wherever nothing is listed
    kv = plx.parallax_cache_read_q4(torch.from_numpy(cache).to(DEV), d, cap)
    if page:
        pools = plx.parallax_cache_read_q4(target, d, page)  # (every page as a sequence of its own)
        kv = pools
    for use_r, S in ((True, 0), (True, 1), (True, 3), (False, 2)):
        got = plx.parallax_decode(q, r, *kv, d ** -0.5, seq_lens=seq, use_r=use_r, num_splits=S, block_list=names, **more)
        hr = host(r) if use_r else np.zeros_like(host(r))
        _check(got, host(q), hr, k, v, d ** -0.5, see, (page, use_r, S, "bf16"))


def test_not_finite_values_reach_who_sees_them(plx):
    """A NaN group of a key that some rows of a tile see and others do not (d = 128, rows in a chain, and a window)."""
    d, Tq, n = 128, 4, 90
    cache = _cache(1, 1, n, d, 41)
    cache[0, 0, 88, d + 8 + 2] = 255  # V, dimensions 32 .. 47, of the last key but one
    q, r = _normal((1, 2, Tq, d), 42), _normal((1, 2, Tq, d), 43)
    seq = torch.tensor([n], dtype=torch.int32, device=DEV)
    got = host(plx.parallax_decode_q4(q, r, torch.from_numpy(cache).to(DEV), d ** -0.5, seq_lens=seq))
    bad = np.zeros((1, 2, Tq, d), dtype=bool)
    bad[:, :, 2:, 32:48] = True
    assert np.array_equal(~np.isfinite(got), bad)
    cache[0, 0, 88, d + 8 + 2] = 127
    cache[0, 0, 88, d + 1] = 255  # K
    got = host(plx.parallax_decode_q4(q, r, torch.from_numpy(cache).to(DEV), d ** -0.5, seq_lens=seq))
    bad[:] = False
    bad[:, :, 2:] = True
    assert np.array_equal(np.isnan(got), bad)


def test_strides_and_one_cache_for_all(plx):
    """Rows with gaps, heads inside tokens, and a cache that all sequences share (stride 0)."""
    d, B, Hkv, cap = 128, 3, 2, 200
    cache = _cache(1, Hkv, cap, d, 51)
    q, r = _normal((B, 4, d), 52), _normal((B, 4, d), 53)
    seq = torch.tensor([200, 31, 7], dtype=torch.int32, device=DEV)
    wide = torch.full((cap, Hkv, 208), 0xff, dtype=torch.uint8, device=DEV)
    wide[..., 16:160] = torch.from_numpy(cache[0]).to(DEV).transpose(0, 1)
    view = wide[..., 16:160].transpose(0, 1)[None].expand(B, -1, -1, -1)
    got = plx.parallax_decode_q4(q, r, view, d ** -0.5, seq_lens=seq)
    want = plx.parallax_decode_q4(q, r, torch.from_numpy(np.repeat(cache, B, 0)).to(DEV), d ** -0.5, seq_lens=seq)
    assert torch.equal(got, want)
