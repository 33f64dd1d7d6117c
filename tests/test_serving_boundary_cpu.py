"""Host-side checks of the entry points for drafted trees, sinks and cache pages that need no GPU: struct layouts, refusals before
any launch, split counts."""
import ctypes
import os
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def binding():
    from paper_2605_29157_amd import binding as b

    if not os.path.exists(b.LIB_PATH):
        from paper_2605_29157_amd import build

        build.build_library(verbose=False)
    b.load_library()
    return b


def test_struct_layouts_match_a_c_compiler(binding, tmp_path):
    structs = ["plx_decode_tree_args", "plx_page_table", "plx_cache_pools", "plx_cache_compact_args"]
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "parallax.h"', 'int main(void) {']
    for name in structs:
        lines.append('printf("%s %%zu\\n", sizeof(%s));' % (name, name))
        lines += ['printf("%s.%s %%zu\\n", offsetof(%s, %s));' % (name, f[0], name, f[0]) for f in getattr(binding, name)._fields_]
    lines += ['printf("extend %d\\nnodes %d\\n", PLX_MAX_EXTEND, PLX_MAX_TREE_NODES);', 'return 0;', '}']
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split("\n")
    want = dict(line.split() for line in out if line)
    for name in structs:
        cls = getattr(binding, name)
        assert ctypes.sizeof(cls) == int(want[name]), name
        for f in cls._fields_:
            assert getattr(cls, f[0]).offset == int(want["%s.%s" % (name, f[0])]), (name, f[0])
    assert (want["extend"], want["nodes"]) == ("1024", "256")


def _decode(binding, a=None, **fields):
    a = binding.plx_decode_args() if a is None else a
    a.q = a.r = a.k = a.v = a.o = 0x1000
    a.B, a.Hq, a.Hkv, a.Lmax, a.d, a.Tq = 2, 4, 2, 64, 128, 8
    a.k_stride_b, a.k_stride_h, a.k_stride_l = 2 * 64 * 128, 64 * 128, 128
    a.v_stride_b, a.v_stride_h, a.v_stride_l = 2 * 64 * 128, 64 * 128, 128
    a.scale, a.use_r, a.num_splits, a.dtype = 0.1, 1, 1, binding.PLX_BF16
    for name, value in fields.items():
        setattr(a, name, value)
    return a


def test_decode_sinks_refusals(binding):
    lib = binding.load_library()
    assert lib.parallax_decode_sinks(None, 4, None) == binding.PLX_ERR_NULL
    assert lib.parallax_decode_sinks_call_splits(None, 4) == 0
    for status, sinks, fields in [
            (binding.PLX_ERR_SHAPE, -1, dict(window=8)), (binding.PLX_ERR_SHAPE, 4, dict(window=0)),
            (binding.PLX_ERR_SHAPE, 4, dict(window=-2)), (binding.PLX_ERR_NULL, 4, dict(window=8, k=None)),
            (binding.PLX_ERR_NULL, 4, dict(window=8, o=None)), (binding.PLX_ERR_SHAPE, 4, dict(window=8, Lmax=0)),
            (binding.PLX_ERR_SHAPE, 4, dict(window=8, Tq=-1)), (binding.PLX_ERR_SHAPE, 4, dict(window=8, d=96)),
            (binding.PLX_ERR_ALIGN, 4, dict(window=8, q=0x1004)), (binding.PLX_ERR_SCALE, 4, dict(window=8, scale=-1.0)),
            (binding.PLX_ERR_DTYPE, 4, dict(window=8, dtype=9)), (binding.PLX_ERR_SPLITS, 4, dict(window=8, num_splits=129)),
            (binding.PLX_ERR_WORKSPACE, 4, dict(window=8, num_splits=4)),
            (binding.PLX_ERR_WORKSPACE, 4, dict(window=8, num_splits=4, workspace=0x2000, workspace_bytes=64))]:
        a = _decode(binding, **fields)
        assert lib.parallax_decode_sinks(ctypes.byref(a), sinks, None) == status, (sinks, fields)
        if status != binding.PLX_ERR_WORKSPACE and fields.get("o", 1):
            assert lib.parallax_decode_sinks_call_splits(ctypes.byref(a), sinks) == 0, (sinks, fields)
    a = _decode(binding, window=8)
    a.prep = binding.plx_qr_prep(q_gamma=0x3000, r_gamma=0x3000)  # rows are prepared beforehand here
    assert lib.parallax_decode_sinks(ctypes.byref(a), 4, None) == binding.PLX_ERR_SHAPE


def test_decode_tree_refusals(binding):
    lib = binding.load_library()

    def tree(mask=0x4000, drafts=None, batch=1, sinks=0, **fields):
        t = binding.plx_decode_tree_args()
        _decode(binding, t.decode, **fields)
        t.tree_mask, t.draft_lens, t.mask_batch, t.sinks = mask, drafts, batch, sinks
        return ctypes.byref(t)

    assert lib.parallax_decode_tree(None, None) == binding.PLX_ERR_NULL
    assert lib.parallax_decode_tree_call_splits(None) == 0
    assert lib.parallax_decode_tree_call_splits(tree(drafts=0x5000, batch=2)) == 1  # (a good one)
    for status, t in [
            (binding.PLX_ERR_NULL, tree(mask=None)), (binding.PLX_ERR_ALIGN, tree(mask=0x4004)),
            (binding.PLX_ERR_ALIGN, tree(drafts=0x5002)), (binding.PLX_ERR_SHAPE, tree(batch=0)),
            (binding.PLX_ERR_SHAPE, tree(batch=3)), (binding.PLX_ERR_SHAPE, tree(Tq=257)),
            (binding.PLX_ERR_SHAPE, tree(sinks=3)), (binding.PLX_ERR_SHAPE, tree(sinks=-1, window=9)),
            (binding.PLX_ERR_NULL, tree(r=None)), (binding.PLX_ERR_SHAPE, tree(Hq=5)),
            (binding.PLX_ERR_ALIGN, tree(seq_lens=0x6001)), (binding.PLX_ERR_WORKSPACE, tree(num_splits=3))]:
        assert lib.parallax_decode_tree(t, None) == status, status
    t = binding.plx_decode_tree_args()
    _decode(binding, t.decode)
    t.tree_mask, t.mask_batch, t.decode.prep = 0x4000, 1, binding.plx_qr_prep(q_gamma=0x3000, r_gamma=0x3000)
    assert lib.parallax_decode_tree(ctypes.byref(t), None) == binding.PLX_ERR_SHAPE


def test_splits_of_a_tree_call(binding):
    """On 256 compute units (what the library counts on without a GPU, too)."""
    lib = binding.load_library()

    def splits(B, Hkv, G, Tq, L, d=128, window=0, sinks=0, dtype=None):
        t = binding.plx_decode_tree_args()
        _decode(binding, t.decode, B=B, Hq=Hkv * G, Hkv=Hkv, Lmax=L, Tq=Tq, d=d, num_splits=0, window=window)
        for x in "kv":
            for s, n in zip("bhl", (Hkv * L * d, L * d, d)):
                setattr(t.decode, "%s_stride_%s" % (x, s), n)
        if dtype is not None:
            t.decode.dtype = dtype
        t.tree_mask, t.mask_batch, t.sinks = 0x4000, 1, sinks
        return lib.parallax_decode_tree_call_splits(ctypes.byref(t))

    assert splits(8, 4, 4, 64, 16384) == 4     # 256 workgroups of 128 columns
    assert splits(8, 4, 4, 32, 16384) == 8
    assert splits(16, 8, 2, 26, 6000) == 2     # 256 of 64
    assert splits(64, 8, 2, 26, 6000) == 1     # two rounds as it is
    assert splits(16, 8, 2, 26, 200) == 1      # two tiles: a merge costs more
    # up to 16 columns: as plain rows over as many keys, more where units stay idle
    assert [splits(1, 8, 2, 8, L) for L in (500, 1028, 1500)] == [1, 8, 12]
    assert splits(16, 8, 2, 8, 16384) == binding.parallax_decode_num_splits(16, 16, 8, 16384, 128, 256)
    assert splits(1, 8, 2, 8, 100000, window=512, sinks=4) == splits(1, 8, 2, 8, 523)
    assert splits(1, 8, 2, 26, 100000, window=500, sinks=4) == splits(1, 8, 2, 26, 529)
    for shape in ((1, 1, 16, 256, 1 << 20), (1, 1, 16, 256, 1), (300, 8, 2, 100, 40000), (1, 8, 2, 20, 131072)):
        assert 1 <= splits(*shape) <= binding.PLX_MAX_SPLITS
        assert 1 <= splits(*shape, dtype=binding.PLX_F32) <= binding.PLX_MAX_SPLITS


def _table(binding, **fields):
    t = binding.plx_page_table()
    t.block_table = t.seq_lens = t.page_refs = t.free_pages = t.free_count = 0x1000
    t.sequences, t.pages_per_sequence, t.block_table_stride, t.num_pages, t.page_size = 4, 8, 8, 32, 16
    for name, value in fields.items():
        setattr(t, name, value)
    return t


def test_page_table_refusals(binding):
    lib = binding.load_library()
    calls = [lambda t: lib.parallax_cache_fork(t, 0x2000, 0x2000, 2, None),
             lambda t: lib.parallax_cache_extend(t, 0x2000, 0x2000, 2, 0x2000, 0x2000, 0x2000, 0x2000, None),
             lambda t: lib.parallax_cache_free(t, 0x2000, None, None, 2, None)]
    for call in calls:
        assert call(None) == binding.PLX_ERR_NULL
        for name in ("block_table", "seq_lens", "page_refs", "free_pages", "free_count"):
            assert call(ctypes.byref(_table(binding, **{name: None}))) == binding.PLX_ERR_NULL, name
            assert call(ctypes.byref(_table(binding, **{name: 0x1002}))) == binding.PLX_ERR_ALIGN, name
        for fields in (dict(sequences=0), dict(pages_per_sequence=0), dict(num_pages=0), dict(page_size=0), dict(block_table_stride=7),
                       dict(pages_per_sequence=1 << 20, block_table_stride=1 << 20, page_size=1 << 12)):
            assert call(ctypes.byref(_table(binding, **fields))) == binding.PLX_ERR_SHAPE, fields


def test_list_refusals(binding):
    lib, t = binding.load_library(), ctypes.byref(_table(binding))
    fork, extend, free = lib.parallax_cache_fork, lib.parallax_cache_extend, lib.parallax_cache_free
    assert fork(t, None, None, 0, None) == binding.PLX_OK and free(t, None, None, None, 0, None) == binding.PLX_OK
    for n in (-1, 65536):
        assert fork(t, 0x2000, 0x2000, n, None) == binding.PLX_ERR_SHAPE
        assert free(t, 0x2000, None, None, n, None) == binding.PLX_ERR_SHAPE
    for n in (-1, 1025):
        assert extend(t, 0x2000, 0x2000, n, 0x2000, 0x2000, 0x2000, 0x2000, None) == binding.PLX_ERR_SHAPE
    assert fork(t, None, 0x2000, 1, None) == binding.PLX_ERR_NULL and fork(t, 0x2000, 0x2001, 1, None) == binding.PLX_ERR_ALIGN
    assert free(t, None, None, None, 1, None) == binding.PLX_ERR_NULL
    assert free(t, 0x2000, 0x2002, None, 1, None) == binding.PLX_ERR_ALIGN
    assert free(t, 0x2000, None, 0x2002, 1, None) == binding.PLX_ERR_ALIGN
    for missing in range(6):
        lists = [0x2000] * 6
        lists[missing] = None
        assert extend(t, *lists[:2], 1, *lists[2:], None) == binding.PLX_ERR_NULL
        lists[missing] = 0x2002
        assert extend(t, *lists[:2], 1, *lists[2:], None) == binding.PLX_ERR_ALIGN
    assert extend(t, None, None, 0, None, None, None, None, None) == binding.PLX_ERR_NULL  # (missing is always written)


def _pools(binding, p=None, **fields):
    p = binding.plx_cache_pools() if p is None else p
    p.k = p.v = 0x1000
    p.num_pages, p.heads, p.page_size, p.d, p.dtype = 32, 2, 16, 128, binding.PLX_BF16
    p.k_stride = p.v_stride = (ctypes.c_int64 * 3)(2 * 16 * 128, 16 * 128, 128)
    for name, value in fields.items():
        setattr(p, name, (ctypes.c_int64 * 3)(*value) if "stride" in name else value)
    return p


BAD_POOLS = [("PLX_ERR_NULL", dict(k=None)), ("PLX_ERR_DTYPE", dict(dtype=5)), ("PLX_ERR_SHAPE", dict(num_pages=0)),
             ("PLX_ERR_SHAPE", dict(heads=0)), ("PLX_ERR_SHAPE", dict(page_size=0)), ("PLX_ERR_SHAPE", dict(d=0)),
             ("PLX_ERR_ALIGN", dict(d=100)), ("PLX_ERR_ALIGN", dict(k=0x1008)), ("PLX_ERR_ALIGN", dict(v=0x1008)),
             ("PLX_ERR_ALIGN", dict(k_stride=(4096, 2048, 132))), ("PLX_ERR_SHAPE", dict(k_stride=(4096, 2048, 64))),
             ("PLX_ERR_SHAPE", dict(v_stride=(-4096, 2048, 128))),
             ("PLX_ERR_SHAPE", dict(heads=1 << 16, page_size=1 << 16))]


@pytest.mark.parametrize("status,fields", BAD_POOLS)
def test_copy_and_compact_refuse_pools(binding, status, fields):
    lib = binding.load_library()
    p = _pools(binding, **fields)
    assert lib.parallax_cache_copy(ctypes.byref(p), 0x2000, 0x2000, None, 2, None) == getattr(binding, status)
    a = _compact(binding)
    _pools(binding, a.pools, **fields)
    assert lib.parallax_cache_compact(ctypes.byref(a), None) == getattr(binding, status)


def _compact(binding, **fields):
    a = binding.plx_cache_compact_args()
    _pools(binding, a.pools)
    a.block_table = a.seq_lens = a.draft_lens = a.accepted = a.n_accepted = 0x2000
    a.new_lens, a.B, a.block_table_stride, a.max_draft, a.max_accepted = 0x3000, 4, 8, 26, 10
    for name, value in fields.items():
        setattr(a, name, value)
    return a


def test_copy_and_compact_refusals(binding):
    lib = binding.load_library()
    p = ctypes.byref(_pools(binding))
    copy = lib.parallax_cache_copy
    assert copy(None, 0x2000, 0x2000, None, 1, None) == binding.PLX_ERR_NULL
    assert copy(p, None, None, None, 0, None) == binding.PLX_OK
    assert copy(p, 0x2000, 0x2000, None, -1, None) == binding.PLX_ERR_SHAPE
    assert copy(p, None, 0x2000, None, 1, None) == binding.PLX_ERR_NULL
    assert copy(p, 0x2000, 0x2002, None, 1, None) == binding.PLX_ERR_ALIGN
    assert copy(p, 0x2000, 0x2000, 0x2002, 1, None) == binding.PLX_ERR_ALIGN
    compact = lambda **f: lib.parallax_cache_compact(ctypes.byref(_compact(binding, **f)), None)
    assert lib.parallax_cache_compact(None, None) == binding.PLX_ERR_NULL
    for name in ("seq_lens", "accepted", "n_accepted", "new_lens"):
        assert compact(**{name: None}) == binding.PLX_ERR_NULL, name
    for name in ("seq_lens", "accepted", "n_accepted", "new_lens", "draft_lens", "block_table"):
        assert compact(**{name: 0x2002}) == binding.PLX_ERR_ALIGN, name
    for fields in (dict(B=0), dict(max_draft=0), dict(max_draft=257), dict(max_accepted=0), dict(max_accepted=27),
                   dict(block_table_stride=0), dict(new_lens=0x2000), dict(block_table=None)):  # (contiguous: num_pages = B)
        assert compact(**fields) == binding.PLX_ERR_SHAPE, fields


def _strides(a, names, T, d):
    for name, H in names:
        setattr(a, name + "_stride", (ctypes.c_int64 * 3)(H * T * d, T * d, d))


def test_prefill_and_backward_sinks_refusals(binding):
    lib = binding.load_library()

    def prefill(sinks, **fields):
        a = binding.plx_prefill_args()
        a.q = a.r = a.k = a.v = a.o = 0x1000
        a.B, a.Hq, a.Hkv, a.T, a.d, a.window = 1, 4, 2, 128, 128, 32
        _strides(a, (("q", 4), ("r", 4), ("o", 4), ("k", 2), ("v", 2)), 128, 128)
        a.scale, a.causal, a.use_r, a.dtype = 0.1, 1, 1, binding.PLX_BF16
        for name, value in fields.items():
            setattr(a, name, value)
        return lib.parallax_prefill_sinks(ctypes.byref(a), sinks, None)

    def backward(sinks, query=False, **fields):
        a = binding.plx_prefill_bwd_args()
        for name in ("q", "r", "k", "v", "o", "vbar", "row_stats", "d_o", "dq", "dr", "dk", "dv", "workspace"):
            setattr(a, name, 0x1000)
        a.B, a.Hq, a.Hkv, a.T, a.Tkv, a.d, a.window, a.workspace_bytes = 1, 4, 2, 512, 512, 128, 32, 1 << 30
        _strides(a, [(x, 2 if x in ("k", "v", "dk", "dv") else 4) for x in
                     ("q", "r", "k", "v", "o", "vbar", "d_o", "dq", "dr", "dk", "dv")], 512, 128)
        a.scale, a.causal, a.dtype = 0.1, 1, binding.PLX_BF16
        for name, value in fields.items():
            setattr(a, name, value)
        if query:
            return lib.parallax_prefill_backward_sinks_workspace_bytes(ctypes.byref(a), sinks)
        return lib.parallax_prefill_backward_sinks(ctypes.byref(a), sinks, None)

    assert lib.parallax_prefill_sinks(None, 4, None) == binding.PLX_ERR_NULL
    assert lib.parallax_prefill_backward_sinks(None, 4, None) == binding.PLX_ERR_NULL
    assert lib.parallax_prefill_backward_sinks_workspace_bytes(None, 4) == 0
    lists = dict(sparse_row_ptr=0x1000, sparse_tile_idx=0x1000, sparse_batch=1, sparse_heads=1)
    for sinks, fields, status in ((-1, {}, "PLX_ERR_SHAPE"), (4, dict(window=0), "PLX_ERR_SHAPE"),
                                  (4, dict(window=-3), "PLX_ERR_SHAPE"), (4, dict(causal=0), "PLX_ERR_SHAPE"),
                                  (4, lists, "PLX_ERR_SHAPE"), (4, dict(k=None), "PLX_ERR_NULL"),
                                  (4, dict(d=96), "PLX_ERR_SHAPE"), (4, dict(scale=float("nan")), "PLX_ERR_SCALE")):
        assert prefill(sinks, **fields) == getattr(binding, status), (sinks, fields)
        if fields is lists:
            fields = dict(lists, sparse_col_ptr=0x1000, sparse_col_idx=0x1000)
        assert backward(sinks, **fields) == getattr(binding, status), (sinks, fields)
        assert backward(sinks, query=True, **fields) == 0, (sinks, fields)
    # the sums of the sinks' parts come on top; where the window and the sinks leave nothing out, or without sinks, nothing does
    rows = binding.load_library().parallax_prefill_backward_workspace_bytes(1, 4, 512)
    for dtype in (binding.PLX_BF16, binding.PLX_F32):
        need = backward(4, query=True, dtype=dtype)
        assert need > rows and backward(0, query=True, dtype=dtype) == rows
        assert backward(500, query=True, dtype=dtype) == rows
        assert backward(4, dtype=dtype, workspace_bytes=need - 1) == binding.PLX_ERR_WORKSPACE
        assert backward(4, query=True, dtype=dtype, workspace=None, workspace_bytes=0) == need


def test_sums_of_fp32_parts_stay_small(binding):
    """A 512th of all items to a part at least: however many sinks there are, not many more than 512 parts (but one a block)."""
    lib = binding.load_library()
    for B, Hkv, G, T, window, sinks, d in ((1, 8, 1, 8192, 96, 4, 64), (1, 8, 1, 8192, 16, 4000, 64), (4, 2, 8, 4096, 1, 2000, 256),
                                           (1, 1, 1, 1 << 15, 64, 1 << 14, 128), (2, 3, 2, 40, 3, 20, 36),
                                           (1, 1, 1, 1 << 17, 64, 1 << 16, 128)):
        a = binding.plx_prefill_bwd_args()
        for name in ("q", "r", "k", "v", "o", "vbar", "row_stats", "d_o", "dq", "dr", "dk", "dv"):
            setattr(a, name, 0x1000)
        a.B, a.Hq, a.Hkv, a.T, a.Tkv, a.d, a.window = B, Hkv * G, Hkv, T, T, d, window
        _strides(a, [(x, Hkv if x in ("k", "v", "dk", "dv") else Hkv * G) for x in
                     ("q", "r", "k", "v", "o", "vbar", "d_o", "dq", "dr", "dk", "dv")], T, d)
        a.scale, a.causal, a.dtype = 0.1, 1, binding.PLX_F32
        need = lib.parallax_prefill_backward_sinks_workspace_bytes(ctypes.byref(a), sinks)
        rows = lib.parallax_prefill_backward_workspace_bytes(B, Hkv * G, T)
        if T > 65535:  # (the limit of the fp32 backward)
            assert need == 0
            continue
        blocks = -(-sinks // 16) * B * Hkv
        assert 0 < need - rows <= (512 + 2 * blocks) * 2 * 16 * d * 4, (need, rows)


class _Somewhere:
    """A tensor as far as the check of devices looks at it."""
    def __init__(self, device):
        self.get_device = lambda: device


def test_binding_refuses_other_devices(binding, monkeypatch):
    monkeypatch.setattr(binding, "_here", lambda: 0)
    binding._on_current_device("x", _Somewhere(0), None, _Somewhere(0))
    for tensors in ((_Somewhere(-1),), (_Somewhere(0), _Somewhere(-1)), (_Somewhere(0), _Somewhere(1)), (_Somewhere(1), None, _Somewhere(1))):
        with pytest.raises(ValueError):
            binding._on_current_device("x", *tensors)


def test_binding_refuses_streams_of_other_devices(binding, monkeypatch):
    monkeypatch.setattr(binding, "_here", lambda: 0)
    stream = type("Stream", (), dict(device_index=1, cuda_stream=0x70))()
    with pytest.raises(ValueError):
        binding._launch_stream("x", stream)
    stream.device_index = 0
    assert binding._launch_stream("x", stream) == 0x70


def test_binding_refuses_tensors_that_do_not_fit(binding, monkeypatch):
    monkeypatch.setattr(binding, "_on_current_device", lambda *a: None)
    q, k = torch.zeros(1, 4, 8, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 32, 64, dtype=torch.bfloat16)
    binding._sink_shapes("x", q, (q, None), k, k)
    for args in ((q, (q[:, :2],), k, k), (q, (q,), k, k[:, :, :30]), (q, (q.float(),), k, k), (q, (q,), k.float(), k.float()),
                 (q[0], (), k, k), (q, (q,), k[..., :32], k[..., :32]), (q, (q.transpose(2, 3),), k, k)):
        with pytest.raises((ValueError, TypeError)):
            binding._sink_shapes("x", *args)


def test_binding_refuses_host_tensors(binding):
    q, k = torch.zeros(1, 4, 8, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 32, 64, dtype=torch.bfloat16)
    mask, lens = _chain_of_words(binding, 8), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        binding.parallax_decode_tree(q, q, k, k, 0.1, mask)
    with pytest.raises(ValueError):
        binding.parallax_decode(q, q, k, k, 0.1, window=4, sinks=2)
    with pytest.raises(ValueError):
        binding.parallax_decode(q, q, k, k, 0.1, window=4, sinks=2, prep=binding.plx_qr_prep())
    with pytest.raises(ValueError):
        binding.parallax_decode(q, q, k, k, 0.1, window=4, sinks=2, split_counters=lens)
    with pytest.raises(ValueError):
        binding.parallax_cache_copy(k, k, lens, lens)
    with pytest.raises((TypeError, ValueError)):
        binding.parallax_cache_compact(k, k, lens, lens, torch.zeros(1, 4, dtype=torch.int32), lens)
    with pytest.raises(TypeError):
        binding.PageTable(lens.view(1, 1), lens, lens, lens, lens, 16)


def _chain_of_words(binding, n):
    return binding.tree_mask_words(torch.arange(n) - 1)


def test_tree_mask_words(binding):
    """Bit m % 64 of word m / 64 of node t: m is t or one of its ancestors."""
    for n in (1, 2, 63, 64, 65, 200, 256):
        g = torch.Generator().manual_seed(n)
        parents = torch.stack([torch.tensor([int(torch.randint(-1, t, (1,), generator=g)) for t in range(n)]) for _ in range(2)])
        words = binding.tree_mask_words(parents)
        assert words.dtype == torch.int64 and words.shape == (2, n, -(-n // 64))
        bits = (words.unsqueeze(-1) >> torch.arange(64)) & 1
        see = bits.reshape(2, n, -1).bool()
        assert not see[:, :, n:].any()
        for b in range(2):
            for t in range(n):
                want, m = set(), t
                while m >= 0:
                    want.add(m)
                    m = int(parents[b, m])
                assert set(see[b, t].nonzero().flatten().tolist()) == want, (n, b, t)
    with pytest.raises(ValueError):
        binding.tree_mask_words(torch.tensor([-1, 1, 0]))
