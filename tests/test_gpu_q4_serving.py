"""4-bit caches and lists of blocks as a server uses them: guard bands, other streams, the page calls, a chunk prefilled over what a
cache holds, caches beyond 32 bits, two graphs, what the binding refuses."""
import numpy as np
import pytest
import torch

from oracle import blocks, masked, rows
from parity import BF16_REL_L2, host, rel_l2
from test_gpu_guard_bands import Guarded, plx  # noqa: F401
from test_gpu_q4 import _cache, _check, _normal, _paged
from test_gpu_streams import _noise

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("d,Hq,Hkv,Tq,L,S,page", [(128, 4, 2, 1, 301, 3, 0), (64, 4, 4, 3, 500, 2, 16), (128, 16, 1, 1, 1000, 9, 64),
                                                  (64, 2, 1, 8, 130, 1, 7), (128, 8, 2, 2, 64, 1, 0), (64, 16, 2, 1, 700, 40, 0)])
def test_guard_bands(plx, d, Hq, Hkv, Tq, L, S, page):  # noqa: F811
    """Every buffer that a call reads or writes has exactly its size."""
    g, B, keep = Guarded(), 2, 5
    n_blocks = -(-L // 64)

    def guarded(t):
        x = g.like(t)
        x.copy_(t)
        return x

    k, v = (guarded(_normal((B, Hkv, L, d), s)) for s in (1, 2))
    shape, more = (B, Hkv, L), {}
    if page:
        per = -(-L // page)
        more = dict(block_table=guarded(_ints(np.random.default_rng(1).permutation(B * per).reshape(B, per).tolist())))
        shape = (B * per, Hkv, page)
    cache = g.empty((*shape, blocks.row_bytes(d)), torch.uint8)
    cache.zero_()
    start, lens = guarded(_ints([0, 3])), guarded(_ints([L, L - 3]))
    plx.parallax_cache_write_q4(k, v, cache, start=start, counts=lens, **more)
    out = g.empty((B, Hkv, L, d), torch.bfloat16), g.empty((B, Hkv, L, d), torch.bfloat16)
    plx.parallax_cache_read_q4(cache, d, L, start=start, seq_lens=lens, out=out, **more)
    bounds = g.empty((B, Hkv, n_blocks, 2, d), torch.bfloat16)
    bounds.zero_()
    plx.parallax_cache_bounds(cache, bounds, lens, **more)
    plx.parallax_cache_bounds(k, bounds, lens, from_lens=guarded(_ints([L - 1, 0])), max_new=L)
    q, r = (guarded(_normal((B, Hq, Tq, d), s)) for s in (3, 4))
    names = g.empty((B, Hkv, keep), torch.int32)
    plx.parallax_select_blocks(q, bounds, lens, keep, out=names, workspace=g.empty((B * Hkv * n_blocks,), torch.int64))
    big = torch.randn(B, Hkv, 300, 2, d, device=DEV).to(torch.bfloat16)  # (above what one launch does)
    plx.parallax_select_blocks(q, guarded(big), None, keep, out=g.empty((B, Hkv, keep), torch.int32),
                               workspace=g.empty((B * Hkv * 300,), torch.int64))
    ws = g.empty((B * Hq * Tq * S * (2 * d + 4),), torch.float32)
    at = dict(seq_lens=lens, num_splits=S, workspace=ws)
    want = plx.parallax_decode_q4(q, r, cache, 0.1, seq_lens=lens, num_splits=S, **more)
    got = plx.parallax_decode_q4(q, r, cache, 0.1, out=g.like(q), **at, **more)
    assert torch.equal(got, want)
    plx.parallax_decode_q4(q, r, cache, 0.1, out=g.like(q), block_list=names, **at, **more)
    plx.parallax_decode(q, r, k, v, 0.1, out=g.like(q), block_list=names, **at)
    g.check((d, Hq, Hkv, Tq, L, S, page))


def test_other_stream_between_busy_memory(plx):  # noqa: F811
    d, B = 128, 2
    k, v = (_normal((B, 4, 900, d), s) for s in (1, 2))
    q, r = (_normal((B, 8, d), s) for s in (3, 4))
    cache = torch.zeros(B, 4, 900, blocks.row_bytes(d), dtype=torch.uint8, device=DEV)
    plx.parallax_cache_write_q4(k, v, cache)
    bounds = plx.parallax_cache_bounds(k, torch.zeros(B, 4, 200, 2, d, dtype=torch.bfloat16, device=DEV))
    lens = _ints([900, 700])
    names = plx.parallax_select_blocks(q, bounds, lens, 7)

    def write(stream):
        again = torch.empty_like(cache)
        torch.cuda.synchronize()
        plx.parallax_cache_write_q4(k, v, again, stream=stream)
        torch.cuda.synchronize()
        return again

    calls = dict(read=lambda s: plx.parallax_cache_read_q4(cache, d, 900, seq_lens=lens, stream=s),
                 q4=lambda s: plx.parallax_decode_q4(q, r, cache, 0.1, seq_lens=lens, num_splits=5, stream=s),
                 q4_list=lambda s: plx.parallax_decode_q4(q, r, cache, 0.1, seq_lens=lens, num_splits=2, block_list=names, stream=s),
                 blocks=lambda s: plx.parallax_decode(q, r, k, v, 0.1, seq_lens=lens, num_splits=2, block_list=names, stream=s),
                 select=lambda s: plx.parallax_select_blocks(q, bounds, lens, 7, stream=s), write=write)
    side = torch.cuda.Stream()
    for name, call in calls.items():
        want = call(None)
        torch.cuda.synchronize()
        held = _noise()
        torch.cuda._sleep(3_000_000)
        for b in held:
            b.fill_(float("nan"))
        del held, b  # free, with the writes still behind the pause
        got = call(side)
        after = _noise()
        torch.cuda.synchronize()
        for a, b in zip(want if isinstance(want, (tuple, list)) else (want,), got if isinstance(got, (tuple, list)) else (got,)):
            assert torch.equal(a, b), name
        del after


@pytest.mark.parametrize("d,page", [(128, 16), (64, 24)])
def test_pages_of_a_4_bit_cache(plx, d, page):  # noqa: F811
    """A prompt written, the sequence forked, both copies grown (the shared last page is copied), decoded; one freed."""
    B, Hkv, Hq, width, pages, T = 4, 2, 4, 8, 20, 2 * page + 5
    t = plx.PageTable.empty(B, width, pages, page, device=DEV)
    pool = torch.full((pages, Hkv, page, blocks.row_bytes(d)), 0xff, dtype=torch.uint8, device=DEV)
    k, v = (_normal((1, Hkv, T + 2, d), s) for s in (1, 2))
    other_k, other_v = (_normal((1, Hkv, 2, d), s) for s in (3, 4))
    assert plx.parallax_cache_extend(t, _ints([0]), _ints([T]), pool, None).tolist() == [0]
    plx.parallax_cache_write_q4(k[:, :, :T], v[:, :, :T], pool, block_table=t.block_table[:1])
    plx.parallax_cache_fork(t, _ints([0]), _ints([2]))
    assert plx.parallax_cache_extend(t, _ints([0, 2]), _ints([T + 2, T + 2]), pool, None).tolist() == [0]
    where = _ints([T])
    plx.parallax_cache_write_q4(k[:, :, T:], v[:, :, T:], pool, start=where, block_table=t.block_table[:1])
    plx.parallax_cache_write_q4(other_k, other_v, pool, start=where, block_table=t.block_table[2:3])
    assert t.seq_lens.tolist() == [T + 2, 0, T + 2, 0]
    q, r = (_normal((B, Hq, d), s) for s in (5, 6))
    got = plx.parallax_decode_q4(q, r, pool, d ** -0.5, seq_lens=t.seq_lens, block_table=t.block_table)
    packed = np.zeros((B, Hkv, T + 2, blocks.row_bytes(d)), dtype=np.uint8)
    hk, hv, ok, ov = (host(x) for x in (k, v, other_k, other_v))
    for h in range(Hkv):
        for i in range(T + 2):
            packed[0, h, i] = packed[2, h, i] = blocks.pack_row(hk[0, h, i], hv[0, h, i])
        for i in range(2):
            packed[2, h, T + i] = blocks.pack_row(ok[0, h, i], ov[0, h, i])
    see = np.stack([rows.chain(n, 1, T + 2) for n in (T + 2, 0, T + 2, 0)])[:, None]
    _check(got, host(q)[:, :, None], host(r)[:, :, None], *blocks.unpack(packed, d), d ** -0.5, see)
    plx.parallax_cache_free(t, _ints([0]))
    again = plx.parallax_decode_q4(q, r, pool, d ** -0.5, seq_lens=t.seq_lens, block_table=t.block_table)
    assert torch.equal(again[2], got[2]) and not again[0].any()
    # accepted drafts move as the rows of any pool do
    lens = plx.parallax_cache_compact(pool.view(torch.bfloat16), None, t.seq_lens, _ints([0, 0, 2, 0]), _ints([[0], [0], [1], [0]]),
                                      _ints([0, 0, 1, 0]), block_table=t.block_table)
    assert lens.tolist() == [0, 0, T + 1, 0]
    back = plx.parallax_cache_read_q4(pool, d, 1, start=_ints([0, 0, T, 0]), block_table=t.block_table)
    assert np.array_equal(back[0][2, :, 0].double().cpu().numpy(), blocks.unpack(packed[2, :, T + 1], d)[0])


def test_a_chunk_behind_a_4_bit_cache(plx):  # noqa: F811
    """Rows read back as the keys in front of a prefill chunk: the last row is what a decode step over the cache gives."""
    d, T, chunk = 128, 300, 40
    k, v = (_normal((1, 2, T, d), s) for s in (1, 2))
    q, r = (_normal((1, 4, chunk, d), s) for s in (3, 4))
    cache = torch.zeros(1, 2, T, blocks.row_bytes(d), dtype=torch.uint8, device=DEV)
    plx.parallax_cache_write_q4(k, v, cache)
    kk, vv = plx.parallax_cache_read_q4(cache, d, T)
    o = plx.parallax_prefill(q, r, kk, vv, d ** -0.5, causal=True)
    step = plx.parallax_decode_q4(q[:, :, -4:].contiguous(), r[:, :, -4:].contiguous(), cache, d ** -0.5)
    see = rows.chain(T, 4, T)[None, None]
    for x in (o[:, :, -4:], step):
        _check(x.contiguous(), host(q)[:, :, -4:], host(r)[:, :, -4:], *(host(y).astype(np.float64) for y in (kk, vv)), d ** -0.5, see)


@pytest.mark.parametrize("d,page", [(128, 0), (64, 0), (128, 48), (128, 64)])
def test_caches_beyond_32_bits(plx, d, page):  # noqa: F811
    """The last tokens of a sequence of 2^25 (4.8 GB of rows at d = 128): written, read, bounded, selected, decoded over."""
    L, T = 2 ** 25 + 77, 300
    row = blocks.row_bytes(d)
    more, n_pages = {}, -(-L // page) if page else 0
    if page:
        cache = torch.empty(n_pages, 1, page, row, dtype=torch.uint8, device=DEV)
        more = dict(block_table=torch.arange(n_pages, dtype=torch.int32, device=DEV)[None])
    else:
        cache = torch.empty(1, 1, L, row, dtype=torch.uint8, device=DEV)
    k, v = (_normal((1, 1, T, d), s) for s in (1, 2))
    q, r = (_normal((1, 2, d), s) for s in (3, 4))
    start, lens = _ints([L - T]), _ints([L])
    plx.parallax_cache_write_q4(k, v, cache, start=start, **more)
    kk, vv = plx.parallax_cache_read_q4(cache, d, T, start=start, **more)
    small = torch.zeros(1, 1, T, row, dtype=torch.uint8, device=DEV)
    plx.parallax_cache_write_q4(k, v, small)
    assert all(torch.equal(a, b) for a, b in zip((kk, vv), plx.parallax_cache_read_q4(small, d, T)))
    hk, hv = (host(x).astype(np.float64) for x in (kk, vv))
    got = plx.parallax_decode_q4(q, r, cache, d ** -0.5, seq_lens=lens, window=256, **more)
    see = np.zeros((1, 1, 1, T), dtype=bool)
    see[..., T - 256:] = True
    _check(got, host(q)[:, :, None], host(r)[:, :, None], hk, hv, d ** -0.5, see)
    # the last three blocks: tokens from 64 * first on
    n_blocks = -(-L // 64)
    bounds = torch.zeros(1, 1, n_blocks, 2, d, dtype=torch.bfloat16, device=DEV)
    first = n_blocks - 3
    plx.parallax_cache_bounds(cache, bounds, lens, from_lens=_ints([64 * first]), max_new=200, **more)
    skip = 64 * first - (L - T)
    low, high = blocks.bounds(hk[0, 0, skip:], T - skip)
    assert np.array_equal(host(bounds)[0, 0, first:, 0], low) and np.array_equal(host(bounds)[0, 0, first:, 1], high)
    bounds[:, :, :first] = -1000.0 * torch.sign(q[:, :1]).unsqueeze(2).unsqueeze(2)
    names = plx.parallax_select_blocks(q[:, :1].contiguous(), bounds, lens, 3, first=0, recent=1)
    assert names[0, 0].tolist() == [first, first + 1, first + 2]
    got = plx.parallax_decode_q4(q, r, cache, d ** -0.5, seq_lens=lens, block_list=names, **more)
    see = np.zeros((1, 1, 1, T), dtype=bool)
    see[..., skip:] = True
    _check(got, host(q)[:, :, None], host(r)[:, :, None], hk, hv, d ** -0.5, see)
    del cache
    if page != 48:  # ... and over bf16 rows
        shape = (n_pages, 1, page, d) if page else (1, 1, L, d)
        pool = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
        pool.view(-1, d)[L - T: L] = kk[0, 0]
        got = plx.parallax_decode(q, r, pool, pool, d ** -0.5, seq_lens=lens, block_list=names, **more)
        _check(got, host(q)[:, :, None], host(r)[:, :, None], hk, hk, d ** -0.5, see)


def test_two_graphs_with_one_workspace(plx):  # noqa: F811
    """Two captured steps share a workspace and are replayed in turn, with eager work between."""
    d, B = 64, 3
    cache = torch.from_numpy(_cache(B, 2, 700, d, 5)).to(DEV)
    lens = _ints([700, 300, 64])
    q, r = (_normal((2, B, 4, d), s) for s in (1, 2))
    ws = torch.empty(1 << 18, dtype=torch.float32, device=DEV)
    outs = [torch.empty(B, 4, d, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    want = [plx.parallax_decode_q4(q[i], r[i], cache, 0.1, seq_lens=lens, num_splits=3 + 4 * i) for i in range(2)]
    graphs = []
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            plx.parallax_decode_q4(q[i], r[i], cache, 0.1, seq_lens=lens, num_splits=3 + 4 * i, workspace=ws, out=outs[i])
    for n in range(6):
        outs[n % 2].zero_()
        graphs[n % 2].replay()
        (torch.randn(1000, device=DEV) @ torch.randn(1000, 7, device=DEV)).sum()
        torch.cuda.synchronize()
        assert torch.equal(outs[n % 2], want[n % 2]), n


def test_the_same_bits_every_time(plx):  # noqa: F811
    d = 128
    cache = torch.from_numpy(_cache(2, 2, 3000, d, 6)).to(DEV)
    q, r = (_normal((2, 4, d), s) for s in (1, 2))
    first = plx.parallax_decode_q4(q, r, cache, 0.1, num_splits=6)
    assert all(torch.equal(plx.parallax_decode_q4(q, r, cache, 0.1, num_splits=6), first) for _ in range(5))
    pool, table = _paged(cache.cpu().numpy(), 16, 3)
    assert torch.equal(plx.parallax_decode_q4(q, r, pool, 0.1, num_splits=6, block_table=table, max_len=3000), first)
    pool, table = _paged(cache.cpu().numpy(), 24, 3)
    assert torch.equal(plx.parallax_decode_q4(q, r, pool, 0.1, num_splits=6, block_table=table, max_len=3000), first)
    # a list of all blocks is all of them
    names = torch.arange(47, dtype=torch.int32, device=DEV).expand(2, 2, 47).contiguous()
    assert torch.equal(plx.parallax_decode_q4(q, r, cache, 0.1, num_splits=6, block_list=names), first)


def test_refusals_of_the_binding(plx):  # noqa: F811
    d = 64
    k = _normal((2, 2, 10, d), 1)
    cache = torch.zeros(2, 2, 20, 80, dtype=torch.uint8, device=DEV)
    q = _normal((2, 4, d), 2)
    bounds = torch.zeros(2, 2, 1, 2, d, dtype=torch.bfloat16, device=DEV)
    names = torch.zeros(2, 2, 3, dtype=torch.int32, device=DEV)
    table = torch.zeros(2, 4, dtype=torch.int32, device=DEV)
    for call in (
            lambda: plx.parallax_cache_write_q4(k, k[:, :, :5], cache), lambda: plx.parallax_cache_write_q4(k, k.float(), cache),
            lambda: plx.parallax_cache_write_q4(k[0], k[0], cache), lambda: plx.parallax_cache_write_q4(k, k, cache[:, :1]),
            lambda: plx.parallax_cache_write_q4(k, k, cache[:1]), lambda: plx.parallax_cache_write_q4(k.half(), k.half(), cache),
            lambda: plx.parallax_cache_write_q4(k, k, cache[..., :79]), lambda: plx.parallax_cache_write_q4(k, k, cache.view(torch.int8)),
            lambda: plx.parallax_cache_write_q4(k, k, torch.zeros(2, 2, 20, 144, dtype=torch.uint8, device=DEV)),
            lambda: plx.parallax_cache_write_q4(k, k, cache, start=_ints([1])), lambda: plx.parallax_cache_write_q4(k, k, cache, start=_ints([1, 2]).long()),
            lambda: plx.parallax_cache_write_q4(k, k, cache, block_table=table.long()),
            lambda: plx.parallax_cache_write_q4(k, k, cache, block_table=table[:1]),
            lambda: plx.parallax_cache_read_q4(cache, 128, 4), lambda: plx.parallax_cache_read_q4(cache, d, 4, out=(k, k)),
            lambda: plx.parallax_cache_read_q4(cache, d, 10, out=(k[:1].expand(2, -1, -1, -1), k)),
            lambda: plx.parallax_cache_read_q4(cache, d, 4, dtype=torch.float16), lambda: plx.parallax_cache_read_q4(cache, d, -1),
            lambda: plx.parallax_decode_q4(q.float(), q.float(), cache, 0.1), lambda: plx.parallax_decode_q4(q, None, cache, 0.1),
            lambda: plx.parallax_decode_q4(q, q[:, :2], cache, 0.1), lambda: plx.parallax_decode_q4(q[:1], q[:1], cache, 0.1),
            lambda: plx.parallax_decode_q4(q.transpose(1, 2), q.transpose(1, 2), cache, 0.1),
            lambda: plx.parallax_decode_q4(q, q, cache, 0.1, block_list=names.long()), lambda: plx.parallax_decode_q4(q, q, cache, 0.1, block_list=names[:1]),
            lambda: plx.parallax_decode_q4(q, q, cache, 0.1, block_list=names[..., :0]), lambda: plx.parallax_decode_q4(q, q, cache, 0.1, block_list=names, window=4),
            lambda: plx.parallax_decode_q4(q, q, cache, 0.1, sinks=4), lambda: plx.parallax_decode_q4(q, q, cache, float("nan")),
            lambda: plx.parallax_decode(q, q, k, k, 0.1, block_list=names, sinks=4, window=5),
            lambda: plx.parallax_decode(q, q, k, k, 0.1, block_list=names, window=5),
            lambda: plx.parallax_decode(q.float(), q.float(), k.float(), k.float(), 0.1, block_list=names),
            lambda: plx.parallax_decode(q, q, k, k, 0.1, block_list=names, split_counters=names),
            lambda: plx.parallax_cache_bounds(k.float(), bounds), lambda: plx.parallax_cache_bounds(k, bounds.float()),
            lambda: plx.parallax_cache_bounds(k, bounds[:, :1]), lambda: plx.parallax_cache_bounds(k, bounds, _ints([3])),
            lambda: plx.parallax_cache_bounds(_normal((2, 2, 65, d), 1), bounds), lambda: plx.parallax_cache_bounds(cache, bounds[..., :32].contiguous()),
            lambda: plx.parallax_select_blocks(q, bounds, None, 2), lambda: plx.parallax_select_blocks(q, bounds, None, 0, first=0, recent=0),
            lambda: plx.parallax_select_blocks(q, bounds[:1], None, 3), lambda: plx.parallax_select_blocks(q, bounds, None, 3, out=names[..., :2].contiguous()),
            lambda: plx.parallax_select_blocks(q, bounds, None, 3, workspace=torch.zeros(1, device=DEV)),
            lambda: plx.parallax_select_blocks(_normal((2, 4, 9, d), 1), bounds, None, 3)):
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            call()
    torch.cuda.synchronize()


@pytest.mark.parametrize("d,page", [(128, 0), (128, 24), (64, 1), (64, 64)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_many_rows_are_as_few(plx, d, page, dtype):  # noqa: F811
    """More rows than a launch takes one by one, ragged: the bytes and rows that calls over 50 tokens give."""
    B, Hkv, T, room = 3, 8, 1700, 1800
    k, v = (_normal((B, Hkv, T, d), s).to(dtype) for s in (1, 2))
    k[1, 2, 1699, 3] = float("inf")
    start, counts = _ints([0, 99, 500]), _ints([T, 1699, T])  # (of the last 400 tokens have no room)
    more, shape = {}, (B, Hkv, room)
    if page:
        per = -(-room // page)
        table = torch.from_numpy(np.random.default_rng(3).permutation(B * per).astype(np.int32).reshape(B, per)).to(DEV)
        table[0, 1] = -1
        more, shape = dict(block_table=table), (B * per, Hkv, page)
    many = torch.full((*shape, blocks.row_bytes(d)), 0x11, dtype=torch.uint8, device=DEV)
    few = many.clone()
    plx.parallax_cache_write_q4(k, v, many, start=start, counts=counts, **more)
    for t in range(0, T, 50):
        plx.parallax_cache_write_q4(k[:, :, t: t + 50], v[:, :, t: t + 50], few, start=start + t, counts=(counts - t).clamp(0, 50), **more)
    assert torch.equal(many, few)
    lens = _ints([room - 3, 1700, room])
    at = dict(seq_lens=lens, dtype=dtype, **more)
    got = plx.parallax_cache_read_q4(many, d, T, start=start, **at)
    for t in range(0, T, 50):
        part = plx.parallax_cache_read_q4(many, d, 50, start=start + t, **at)
        assert all(torch.equal(a[:, :, t: t + 50].view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, part)), t


@pytest.mark.parametrize("page", [1, 3, 7, 1000, 65535])
def test_pages_of_far_tokens(plx, page):  # noqa: F811
    """Rows around the borders of pages, up to token 2^25 + 1 of a sequence, in pages of sizes that are no powers of two."""
    d, last = 64, 2 ** 25 + 1
    n_pages = last // page + 1
    pool = torch.empty((n_pages, 1, page, 80), dtype=torch.uint8, device=DEV)
    table = torch.arange(n_pages, dtype=torch.int32, device=DEV).flip(0)[None].contiguous()
    T = 5
    k, v = (_normal((1, 1, T, d), s) for s in (1, 2))
    small = torch.zeros(1, 1, T, 80, dtype=torch.uint8, device=DEV)
    plx.parallax_cache_write_q4(k, v, small)
    for first in (0, page - 2, 1000 * page - 3, last // 2, (last // page - 1) * page - 2, last + 1 - T):
        first = max(first, 0)
        start = _ints([first])
        plx.parallax_cache_write_q4(k, v, pool, start=start, block_table=table)
        for t in range(T):
            x = first + t
            if x // page < n_pages:
                assert torch.equal(pool[n_pages - 1 - x // page, 0, x % page], small[0, 0, t]), (first, t)
        back = plx.parallax_cache_read_q4(pool, d, T, start=start, block_table=table)
        want = plx.parallax_cache_read_q4(small, d, T)
        there = (first + torch.arange(T, device=DEV) < n_pages * page)[None, None, :, None]  # (a token past the last page: zeros)
        assert all(torch.equal(a, torch.where(there, b, torch.zeros_like(b))) for a, b in zip(back, want)), first


@pytest.mark.parametrize("d", [64, 128])
def test_the_same_bits_in_pages_of_any_size(plx, d):  # noqa: F811
    """Lists, windows with sinks and whole sequences that end anywhere: pages of any size give what rows without pages give."""
    B, L = 5, 700
    cache = torch.from_numpy(_cache(B, 2, L, d, 8)).to(DEV)
    lens = _ints([700, 641, 8, 65, 0])
    q, r = (_normal((B, 8, 2, d), s) for s in (1, 2))
    names = _ints([[[0, 2, 5, 10, -1], [1, 3, 3, 4, 9]]] * B)
    for page in (1, 7, 8, 16, 40, 48, 64, 100, 128, 1000):
        pool, table = _paged(cache.cpu().numpy(), page, 3)
        for more in (dict(), dict(block_list=names), dict(window=100, sinks=70)):
            for S in (1, 3):
                want = plx.parallax_decode_q4(q, r, cache, 0.1, seq_lens=lens, num_splits=S, **more)
                got = plx.parallax_decode_q4(q, r, pool, 0.1, seq_lens=lens, num_splits=S, block_table=table, max_len=L, **more)
                assert torch.equal(got, want), (page, S, tuple(more))


@pytest.mark.parametrize("d", [64, 128])
def test_lists_over_bf16_pages_of_any_size(plx, d):  # noqa: F811
    """... and the bf16 decode over lists, whose entries may be anything."""
    B, L = 4, 700
    k, v = (_normal((B, 2, L, d), s) for s in (1, 2))
    q, r = (_normal((B, 8, 2, d), s) for s in (3, 4))
    lens = _ints([700, 641, 65, 0])
    top, low = 2 ** 31 - 1, -2 ** 31
    names = _ints([[[low, 0, 2, 5, 10, top], [1, 3, 3, 4, 9, -1]], [[0, 0, 0, 0, 0, 0], [10, 9, 8, 7, 6, 5]],
                   [[-1, 0, 1, 2, 3, 4], [top, 1, low, 0, 2, 1]], [[0, 1, 2, 3, 4, 5]] * 2])
    kept = [[[0, 2, 5, 10], [1, 3, 4, 9]], [[0], [10]], [[0, 1], [0]], [[], []]]
    for x in (0, 1, 2):  # what the entries come to
        for h in (0, 1):
            seen = np.full((1, 2, L), False)
            before = -1
            for e in names[x, h].tolist():
                if 0 <= e and e > before and e * 64 < lens[x].item():
                    seen[..., e * 64: e * 64 + 64] = True
                before = e
            assert [j for j in range(11) if seen[0, 0, j * 64]] == kept[x][h], (x, h)
    want = {}
    for page in (0, 1, 7, 8, 16, 40, 64, 100, 1000):
        kk, vv, more = k, v, {}
        if page:
            per = -(-L // page)
            order = torch.randperm(B * per, device=DEV)
            table = order.to(torch.int32).reshape(B, per)
            kk, vv = (torch.full((B * per, 2, page, d), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2))
            for pool, rows_of in ((kk, k), (vv, v)):
                padded = torch.full((B, 2, per * page, d), float("nan"), dtype=torch.bfloat16, device=DEV)
                padded[:, :, :L] = rows_of
                pool[order] = padded.reshape(B, 2, per, page, d).transpose(1, 2).reshape(B * per, 2, page, d)
            more = dict(block_table=table, max_len=L)
        for S in (1, 3):
            got = plx.parallax_decode(q, r, kk, vv, 0.1, seq_lens=lens, num_splits=S, block_list=names, **more)
            want.setdefault(S, got)
            assert torch.equal(got, want[S]), (page, S)
    held = lens.tolist()
    see = np.stack([np.stack([rows.chain(held[b], 2, L) & blocks.listed_keys(x, held[b], L) for x in kept[b]]) for b in range(B)])
    for S in (1, 3):
        _check(want[S], host(q), host(r), host(k), host(v), 0.1, see, (S,))


@pytest.mark.parametrize("kind", ["v grows", "v falls", "v of one group", "v huge", "v tiny", "u large", "u grows", "u falls", "u tiny", "all"])
@pytest.mark.parametrize("d,Hq,Tq", [(128, 2, 1), (128, 4, 1), (128, 8, 2), (64, 3, 1), (64, 8, 1), (64, 4, 4)])
def test_references_move(plx, d, Hq, Tq, kind):  # noqa: F811
    """Values of V and products rho.k whose size changes by many powers of two along the sequence, between dimensions, or is far from one."""
    L = 1500
    k, v = (_normal((1, 1, L, d), s).float() for s in (1, 2))
    q, r = (_normal((1, Hq, Tq, d), s) for s in (3, 4))
    ramp = torch.exp2(torch.linspace(-25, 25, L, device=DEV))[:, None]
    if kind in ("v grows", "all"):
        v *= ramp
    if kind == "v falls":
        v *= ramp.flip(0)
    if kind in ("v of one group", "all"):
        v[..., 16:32] *= 2.0 ** 9
    if kind == "v huge":
        v *= 2.0 ** 90
    if kind == "v tiny":
        v *= 2.0 ** -90
    if kind == "u large":
        r = (r.float() * 2.0 ** 14).to(torch.bfloat16)
    if kind == "u tiny":
        r = (r.float() * 2.0 ** -30).to(torch.bfloat16)
    if kind in ("u grows", "u falls", "all"):  # (in dimensions that q does not look at)
        half = torch.exp2(torch.linspace(-4, 12, L, device=DEV))[:, None]
        k[..., d // 2:] *= half.flip(0) if kind == "u falls" else half
        q[..., d // 2:] = 0
    cache = torch.zeros(1, 1, L, blocks.row_bytes(d), dtype=torch.uint8, device=DEV)
    plx.parallax_cache_write_q4(k, v, cache)
    hk, hv = (x.double().cpu().numpy() for x in plx.parallax_cache_read_q4(cache, d, L, dtype=torch.float32))
    see = rows.chain(L, Tq, L)[None, None]
    hq, hr = host(q).astype(np.float64), host(r).astype(np.float64)
    unit = np.abs(hv).max()  # (the bound's arithmetic is in units of one)
    for S in (1, 2, 5):
        got = plx.parallax_decode_q4(q, r, cache, d ** -0.5, num_splits=S)
        got = host(got).astype(np.float64)
        ref = masked.masked_forward(hq, hr, hk, hv, d ** -0.5, np.broadcast_to(see, (1, Hq, Tq, L)))
        assert np.isfinite(got).all()
        assert rel_l2(got, ref) <= BF16_REL_L2, (kind, S)
        bound = rows.bf16_bound(hq, hr, hk, hv / unit, d ** -0.5, np.broadcast_to(see, (1, Hq, Tq, L))) * unit
        assert (np.abs(got - ref) <= bound).all(), (kind, S, float((np.abs(got - ref) / bound).max()))


@pytest.mark.parametrize("large", [1.0, 2.0 ** 6])
@pytest.mark.parametrize("d", [64, 128])
def test_what_cancels_does_so_exactly(plx, d, large):  # noqa: F811
    """One key, or one value for all keys: the weights sum to one, so the value comes back whatever rho is (to a bf16 rounding of f32 sums
    of 2^-23 |rho.k|, which is below half of its step)."""
    L = 130
    k, v = (_normal((2, 2, L, d), s) for s in (1, 2))
    q, r = (_normal((2, 8, d), s) for s in (3, 4))
    r = (r.float() * large).to(torch.bfloat16)
    cache = torch.zeros(2, 2, L, blocks.row_bytes(d), dtype=torch.uint8, device=DEV)
    for lens, values in ((_ints([1, 1]), v), (_ints([L, 77]), v[:, :, :1].expand(-1, -1, L, -1).contiguous())):
        plx.parallax_cache_write_q4(k, values, cache)
        want = plx.parallax_cache_read_q4(cache, d, 1)[1][:, :, 0].repeat_interleave(4, 1)
        for S in (1, 3):
            got = plx.parallax_decode_q4(q, r, cache, d ** -0.5, seq_lens=lens, num_splits=S)
            assert ((got.float() - want.float()).abs() <= 2.0 ** -8 * want.float().abs()).all(), (S, "a step")
            if int(lens[0]) == 1:
                assert torch.equal(got, want), S
        names = _ints([[[0, 1, 2]] * 2] * 2)
        got = plx.parallax_decode(q, r, k, values, d ** -0.5, seq_lens=lens, block_list=names)
        want = values[:, :, 0].repeat_interleave(4, 1)
        assert ((got.float() - want.float()).abs() <= 2.0 ** -8 * want.float().abs()).all()
        if int(lens[0]) == 1:
            assert torch.equal(got, want)


@pytest.mark.parametrize("huge", [False, True])
@pytest.mark.parametrize("d,Hq", [(128, 2), (128, 8), (64, 4)])
def test_nan_in_a_value_stays_in_its_dimensions(plx, d, Hq, huge):  # noqa: F811
    """16 dimensions of V of one key are NaN: those of the rows that see it are not finite, all other ones as without it (but for where
    the references stand: both are within the rounding of the same result)."""
    L, at = 400, 333
    k, v = (_normal((1, 1, L, d), s).float() for s in (1, 2))
    q, r = (_normal((1, Hq, 2, d), s) for s in (3, 4))
    if huge:
        v *= 2.0 ** 105
    cache = torch.zeros(1, 1, L, blocks.row_bytes(d), dtype=torch.uint8, device=DEV)
    plx.parallax_cache_write_q4(k, v, cache)
    bad = v.clone()
    bad[0, 0, at, 21] = float("nan")
    other = cache.clone()
    plx.parallax_cache_write_q4(k, bad, other)
    for n, S in ((L, 1), (L, 3), (at + 1, 1), (at + 2, 2), (at, 1)):  # (the second row of two ends at n; the first one key before)
        lens = _ints([n])
        want = plx.parallax_decode_q4(q, r, cache, d ** -0.5, seq_lens=lens, num_splits=S)
        got = plx.parallax_decode_q4(q, r, other, d ** -0.5, seq_lens=lens, num_splits=S)
        assert torch.isfinite(want.float()).all()
        for t in range(2):
            sees = at < n - 1 + t
            assert torch.equal(torch.isfinite(got[:, :, t, 16:32].float()), torch.full_like(got[:, :, t, 16:32], not sees, dtype=torch.bool)), (n, S, t)
            rest = [x for x in range(d) if not 16 <= x < 32]
            assert rel_l2(host(got)[:, :, t, rest], host(want)[:, :, t, rest]) <= BF16_REL_L2, (n, S, t)
            if not sees:
                assert rel_l2(host(got)[:, :, t], host(want)[:, :, t]) <= BF16_REL_L2, (n, S, t)
