"""Out-of-bounds canaries for the tree, sink and cache entry points: every buffer that a call writes sits between bands of sentinel
bytes, the workspaces are as small as the library asks for, and calls on another stream find memory of their own."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import rows
from test_gpu_guard_bands import DEV, Guarded, plx  # noqa: F401
from test_gpu_streams import _noise

pytestmark = pytest.mark.gpu


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _rand(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator(DEV).manual_seed(seed), device=DEV).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,Hq,Hkv,d,Tq,L,S", [(2, 4, 2, 128, 7, 301, 3), (2, 6, 2, 64, 13, 500, 2), (1, 16, 2, 128, 21, 1000, 5),
                                               (3, 4, 4, 64, 70, 90, 1), (1, 2, 2, 128, 5, 200, 40)])
def test_decode(plx, dtype, B, Hq, Hkv, d, Tq, L, S):
    g = Guarded()
    q, r = (_rand((B, Hq, Tq, d), dtype, s) for s in (1, 2))
    k, v = (_rand((B, Hkv, L, d), dtype, s) for s in (3, 4))
    mask = torch.from_numpy(rows.words(rows.random_tree(Tq, np.random.default_rng(Tq)))).to(DEV)
    for call in (lambda **o: plx.parallax_decode_tree(q, r, k, v, 0.1, mask, num_splits=S, **o),
                 lambda **o: plx.parallax_decode(q, r, k, v, 0.1, window=64, sinks=5, num_splits=S, **o)):
        want = call()
        out, ws = g.like(q), g.empty((B * Hq * Tq * S * (2 * d + 4),), torch.float32)
        call(out=out, workspace=ws)
        g.check((dtype, B, Hq, d, Tq, L, S))
        assert torch.equal(out, want)


@pytest.mark.parametrize("dtype,B,Hq,Hkv,T,d,window,sinks", [
    (torch.bfloat16, 1, 4, 2, 333, 128, 70, 5), (torch.bfloat16, 2, 4, 4, 1001, 64, 200, 130), (torch.bfloat16, 1, 2, 1, 65, 128, 3, 1),
    (torch.float32, 1, 4, 2, 333, 64, 70, 5), (torch.float32, 2, 2, 2, 701, 128, 30, 40), (torch.float32, 1, 2, 1, 65, 36, 3, 17)])
def test_prefill_and_backward(plx, dtype, B, Hq, Hkv, T, d, window, sinks):
    g = Guarded()
    q, r, up = (_rand((B, Hq, T, d), dtype, s) for s in (1, 2, 3))
    k, v = (_rand((B, Hkv, T, d), dtype, s) for s in (4, 5))
    want, vbar, stats = plx.parallax_prefill(q, r, k, v, 0.1, window=window, sinks=sinks, save_for_backward=True)
    grads = plx.parallax_prefill_backward(q, r, k, v, want, vbar, stats, up, 0.1, window=window, sinks=sinks)
    out = g.like(q)
    plx.parallax_prefill(q, r, k, v, 0.1, window=window, sinks=sinks, out=out)
    into = [g.like(t) for t in (q, r, k, v)]
    a = plx.prefill_bwd_args(q, r, k, v, want, vbar, stats, up, *into, 0.1, True, stats, window)
    lib = plx.load_library()
    need = lib.parallax_prefill_backward_sinks_workspace_bytes(ctypes.byref(a), sinks)
    assert need > 16 * B * Hq * T and need % 16 == 0
    ws = g.empty((need // 4,), torch.float32)
    a.workspace, a.workspace_bytes = ws.data_ptr(), need
    assert lib.parallax_prefill_backward_sinks(ctypes.byref(a), sinks, plx._stream_ptr(None)) == 0
    g.check((dtype, B, T, d, window, sinks))
    for x, y in zip([out] + into, (want,) + tuple(grads)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("page,heads,d", [(16, 2, 128), (5, 1, 64)])
def test_cache(plx, page, heads, d):
    """Table, counts, free list, lists of a call and pools, each of exactly its size."""
    g = Guarded()
    sequences, width, pages = 5, 7, 23
    first = plx.PageTable.empty(sequences, width, pages, page, device=DEV)
    state = []
    for t in (first.block_table, first.seq_lens, first.page_refs, first.free_pages, first.free_count):
        state.append(g.like(t))
        state[-1].copy_(t)
    t = plx.PageTable(*state, page)
    k, v = (g.empty((pages, heads, page, d), torch.bfloat16) for _ in range(2))
    k.zero_(), v.zero_()
    lib, stream = plx.load_library(), plx._stream_ptr(None)
    seqs, to = _ints([0, 1, 2, -1, 9, 0]), _ints([3 * page + 2, 1, width * page, 4, 4, 4])
    lists = [g.empty((6,), torch.int32) for _ in range(3)] + [g.empty((1,), torch.int32)]
    st = lib.parallax_cache_extend(ctypes.byref(t._args), seqs.data_ptr(), to.data_ptr(), 6, *(x.data_ptr() for x in lists), stream)
    assert st == 0 and lists[3].tolist() == [0]
    assert lists[0].tolist() == lists[1].tolist() == [-1] * 6 and lists[2].tolist() == [0] * 6
    plx.parallax_cache_fork(t, _ints([0, 1, 7]), _ints([3, 4, 2]))
    assert plx.parallax_cache_extend(t, _ints([3, 0]), _ints([3 * page + 3, 3 * page + 3]), k, v).tolist() == [0]
    new = g.empty((sequences,), torch.int32)
    plx.parallax_cache_compact(k, v, t.seq_lens, _ints([3, 1, 9, 0, 4]), _ints([[0, 2], [0, 0], [4, 8], [0, 0], [1, 3]]),
                               _ints([2, 1, 2, 0, 2]), block_table=t.block_table, new_lens=new)
    plx.parallax_cache_free(t, _ints([0, 1, 2, 3, 4, 5, -3]))
    g.check((page, heads, d))
    assert t.free_count.tolist() == [pages] and t.page_refs.tolist() == [0] * pages and sorted(t.free_pages.tolist()) == list(range(pages))
    assert (t.block_table == -1).all() and t.seq_lens.tolist() == [0] * sequences


def test_other_stream_between_busy_memory(plx):
    q, r, up = (_rand((1, 4, 700, 128), torch.bfloat16, s) for s in (1, 2, 3))
    k, v = (_rand((1, 2, 700, 128), torch.bfloat16, s) for s in (4, 5))
    f = {t: _rand((1, 2, 600, 64), torch.float32, i) for i, t in enumerate("qrkvg")}
    mask = torch.from_numpy(rows.words(rows.random_tree(40, np.random.default_rng(1)))).to(DEV)
    qt, rt = (x[:, :, :40].contiguous() for x in (q, r))
    saved = plx.parallax_prefill(q, r, k, v, 0.1, window=90, sinks=6, save_for_backward=True)
    saved32 = plx.parallax_prefill(f["q"], f["r"], f["k"], f["v"], 0.1, window=90, sinks=6, save_for_backward=True)
    calls = dict(
        tree=lambda s: plx.parallax_decode_tree(qt, rt, k, v, 0.1, mask, num_splits=4, stream=s),
        sinks=lambda s: plx.parallax_decode(qt, rt, k, v, 0.1, window=300, sinks=4, num_splits=9, stream=s),
        prefill=lambda s: plx.parallax_prefill(q, r, k, v, 0.1, window=90, sinks=6, stream=s),
        backward=lambda s: plx.parallax_prefill_backward(q, r, k, v, *saved, up, 0.1, window=90, sinks=6, stream=s),
        backward_f32=lambda s: plx.parallax_prefill_backward(f["q"], f["r"], f["k"], f["v"], *saved32, f["g"], 0.1, window=90,
                                                             sinks=6, stream=s),
        compact=lambda s: plx.parallax_cache_compact(k.clone(), v.clone(), _ints([500]), _ints([9]), _ints([[1, 5]]), _ints([2]),
                                                     stream=s))
    side = torch.cuda.Stream()
    for name, call in calls.items():
        want = call(None)
        torch.cuda.synchronize()
        if name == "compact":  # (its arguments are made on the current stream)
            kk, vv, args = k.clone(), v.clone(), [_ints([500]), _ints([9]), _ints([[1, 5]]), _ints([2])]
            call = lambda s: plx.parallax_cache_compact(kk, vv, *args, stream=s)  # noqa: B023
            torch.cuda.synchronize()
        blocks = _noise()
        torch.cuda._sleep(3_000_000)
        for b in blocks:
            b.fill_(float("nan"))
        del blocks, b  # free, with the writes still behind the pause
        got = call(side)
        after = _noise()
        torch.cuda.synchronize()
        for a, b in zip(want if isinstance(want, tuple) else (want,), got if isinstance(got, tuple) else (got,)):
            assert torch.equal(a, b), name
        del after
