"""Host-side checks of the entry points for 4-bit caches, block bounds, selection and decode over lists that need no GPU: struct
layouts, refusals before any launch, split counts, what the binding refuses."""
import ctypes
import os
import subprocess

import pytest
import torch

from oracle import blocks
from test_serving_boundary_cpu import _decode, binding  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_struct_layouts_match_a_c_compiler(binding, tmp_path):  # noqa: F811
    structs = ["plx_q4_cache", "plx_q4_rows_args", "plx_cache_bounds_args", "plx_select_blocks_args", "plx_decode_blocks_args",
               "plx_decode_q4_args"]
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "parallax.h"', 'int main(void) {']
    for name in structs:
        lines.append('printf("%s %%zu\\n", sizeof(%s));' % (name, name))
        lines += ['printf("%s.%s %%zu\\n", offsetof(%s, %s));' % (name, f[0], name, f[0]) for f in getattr(binding, name)._fields_]
    lines += ['printf("block %d\\n", PLX_BLOCK_KEYS);', 'return 0;', '}']
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
    assert want["block"] == "64"


def test_row_bytes(binding):  # noqa: F811
    lib = binding.load_library()
    assert [lib.parallax_q4_row_bytes(d) for d in (64, 128, 0, 32, 96, 256, -64)] == [80, 144, 0, 0, 0, 0, 0]
    assert all(binding.parallax_q4_row_bytes(d) == blocks.row_bytes(d) for d in (64, 128))


def _q4(binding, c=None, **fields):  # noqa: F811
    c = binding.plx_q4_cache() if c is None else c
    c.rows, c.B, c.Hkv, c.capacity, c.d = 0x1000, 2, 2, 64, 128
    c.stride[:] = (2 * 64 * 144, 64 * 144, 144)
    _set(c, fields)
    return c


def _set(obj, fields):
    for name, value in fields.items():
        if name.startswith("stride") and name[-1] in "012":
            obj.stride[int(name[-1])] = value
        else:
            setattr(obj, name, value)


_BAD_CACHES = [("NULL", dict(rows=None)), ("SHAPE", dict(B=0)), ("SHAPE", dict(Hkv=0)), ("SHAPE", dict(capacity=0)), ("SHAPE", dict(d=96)),
               ("SHAPE", dict(d=256)), ("SHAPE", dict(B=65536)), ("ALIGN", dict(rows=0x1008)), ("SHAPE", dict(stride0=-16)),
               ("ALIGN", dict(stride1=8)), ("SHAPE", dict(stride2=128)), ("ALIGN", dict(stride2=152)), ("ALIGN", dict(block_table=0x2002)),
               ("SHAPE", dict(block_table=0x2000, page_size=0, num_pages=4, block_table_stride=4)),
               ("SHAPE", dict(block_table=0x2000, page_size=16, num_pages=0, block_table_stride=4)),
               ("SHAPE", dict(block_table=0x2000, page_size=16, num_pages=4, block_table_stride=3))]


def test_refusals_of_rows(binding):  # noqa: F811
    lib = binding.load_library()

    def rows(cache=(), **fields):
        a = binding.plx_q4_rows_args()
        _q4(binding, a.cache, **dict(cache))
        a.k, a.v, a.T, a.dtype = 0x3000, 0x4000, 5, binding.PLX_BF16
        a.k_stride[:] = a.v_stride[:] = (2 * 5 * 128, 5 * 128, 128)
        for name, value in fields.items():
            if name[-1] in "012":
                getattr(a, name[:-1])[int(name[-1])] = value
            else:
                setattr(a, name, value)
        return ctypes.byref(a)

    for call in (lib.parallax_cache_write_q4, lib.parallax_cache_read_q4):
        assert call(None, None) == binding.PLX_ERR_NULL
        for status, fields in _BAD_CACHES:
            assert call(rows(fields.items()), None) == getattr(binding, "PLX_ERR_" + status), fields
        for status, fields in [("NULL", dict(k=None)), ("NULL", dict(v=None)), ("DTYPE", dict(dtype=5)), ("SHAPE", dict(T=-1)),
                               ("SHAPE", dict(T=1 << 30)), ("ALIGN", dict(k=0x3008)), ("ALIGN", dict(v=0x4002)),
                               ("ALIGN", dict(start=0x5001)), ("ALIGN", dict(counts=0x5002)), ("SHAPE", dict(k_stride0=-8)),
                               ("ALIGN", dict(v_stride1=4)), ("SHAPE", dict(k_stride2=64)), ("SHAPE", dict(v_stride2=120))]:
            assert call(rows(**fields), None) == getattr(binding, "PLX_ERR_" + status), fields
        assert call(rows(T=0), None) == binding.PLX_OK  # (nothing to do, nothing launched)


def _q4_decode(binding, cache=(), sinks=0, names=None, n=0, **fields):  # noqa: F811
    a = binding.plx_decode_q4_args()
    _decode(binding, a.decode, **dict(dict(Tq=1, k=None, v=None), **fields))
    _q4(binding, a.cache, **dict(cache))
    a.sinks, a.block_list, a.n_list = sinks, names, n
    return a


def test_refusals_of_q4_decode(binding):  # noqa: F811
    lib = binding.load_library()
    assert lib.parallax_decode_q4(None, None) == binding.PLX_ERR_NULL
    assert lib.parallax_decode_q4_call_splits(None) == 0
    for good in (_q4_decode(binding), _q4_decode(binding, Lmax=0, Tq=8), _q4_decode(binding, sinks=3, window=9),
                 _q4_decode(binding, names=0x7000, n=3), _q4_decode(binding, Hq=32, seq_lens=0x6000)):
        assert lib.parallax_decode_q4_call_splits(ctypes.byref(good)) == 1
    bad = [(s, dict(cache=f.items())) for s, f in _BAD_CACHES]
    bad += [("SHAPE", dict(B=3)), ("SHAPE", dict(Hkv=1)), ("SHAPE", dict(d=64)), ("SHAPE", dict(Lmax=65)), ("SHAPE", dict(Lmax=-1)),
            ("NULL", dict(q=None)), ("NULL", dict(r=None)), ("DTYPE", dict(dtype=binding.PLX_F32)),
            ("SHAPE", dict(Tq=9)), ("SHAPE", dict(Hq=34)), ("SHAPE", dict(Hq=5)), ("SHAPE", dict(Tq=-1)), ("SHAPE", dict(window=-1)),
            ("SHAPE", dict(sinks=3)), ("SHAPE", dict(sinks=-1, window=4)), ("SCALE", dict(scale=-1.0)),
            ("ALIGN", dict(q=0x1004)), ("ALIGN", dict(seq_lens=0x6001)), ("SPLITS", dict(num_splits=129)),
            ("ALIGN", dict(names=0x7002, n=3)), ("SHAPE", dict(names=0x7000, n=0)), ("SHAPE", dict(names=0x7000, n=3, window=64)),
            ("SHAPE", dict(names=0x7000, n=(1 << 29) + 1))]
    for status, fields in bad:
        a = _q4_decode(binding, **fields)
        assert lib.parallax_decode_q4(ctypes.byref(a), None) == getattr(binding, "PLX_ERR_" + status), fields
        assert lib.parallax_decode_q4_call_splits(ctypes.byref(a)) == 0, fields
    for status, fields in [("NULL", dict(o=None)), ("WORKSPACE", dict(num_splits=3)),
                           ("WORKSPACE", dict(num_splits=3, workspace=0x2000, workspace_bytes=64)),
                           ("WORKSPACE", dict(num_splits=3, workspace=0x2008, workspace_bytes=1 << 30))]:
        a = _q4_decode(binding, **fields)
        assert lib.parallax_decode_q4(ctypes.byref(a), None) == getattr(binding, "PLX_ERR_" + status), fields
    a = _q4_decode(binding)
    a.decode.prep = binding.plx_qr_prep(q_gamma=0x3000, r_gamma=0x3000)  # rows are prepared beforehand here
    assert lib.parallax_decode_q4(ctypes.byref(a), None) == binding.PLX_ERR_SHAPE


def test_refusals_of_decode_over_lists(binding):  # noqa: F811
    lib = binding.load_library()

    def call(names=0x7000, n=3, **fields):
        a = binding.plx_decode_blocks_args()
        _decode(binding, a.decode, **dict(dict(Tq=1), **fields))
        a.block_list, a.n_list = names, n
        return a

    assert lib.parallax_decode_blocks(None, None) == binding.PLX_ERR_NULL
    assert lib.parallax_decode_blocks_call_splits(None) == 0
    assert lib.parallax_decode_blocks_call_splits(ctypes.byref(call())) == 1
    for status, fields in [("NULL", dict(names=None)), ("ALIGN", dict(names=0x7001)), ("SHAPE", dict(n=0)), ("SHAPE", dict(n=-1)),
                           ("SHAPE", dict(window=4)), ("SHAPE", dict(Tq=9)), ("DTYPE", dict(dtype=binding.PLX_F32)), ("NULL", dict(k=None)),
                           ("SHAPE", dict(Lmax=0)), ("ALIGN", dict(k=0x1004)), ("SHAPE", dict(d=96))]:
        a = call(**fields)
        assert lib.parallax_decode_blocks(ctypes.byref(a), None) == getattr(binding, "PLX_ERR_" + status), fields
        assert lib.parallax_decode_blocks_call_splits(ctypes.byref(a)) == 0, fields
    assert lib.parallax_decode_blocks(ctypes.byref(call(num_splits=2)), None) == binding.PLX_ERR_WORKSPACE
    a = call()
    a.decode.prep = binding.plx_qr_prep(q_gamma=0x3000, r_gamma=0x3000)
    assert lib.parallax_decode_blocks(ctypes.byref(a), None) == binding.PLX_ERR_SHAPE


def test_refusals_of_bounds(binding):  # noqa: F811
    lib = binding.load_library()

    def call(q4=None, **fields):
        a = binding.plx_cache_bounds_args()
        a.k, a.B, a.Hkv, a.capacity, a.d, a.bounds, a.n_blocks = 0x1000, 2, 2, 130, 128, 0x2000, 3
        a.k_stride[:] = (2 * 130 * 128, 130 * 128, 128)
        if q4 is not None:
            a.k, a.q4 = None, ctypes.addressof(q4)
        for name, value in fields.items():
            if name[-1] in "012":
                a.k_stride[int(name[-1])] = value
            else:
                setattr(a, name, value)
        return ctypes.byref(a)

    assert lib.parallax_cache_bounds(None, None) == binding.PLX_ERR_NULL
    for status, fields in [("NULL", dict(k=None)), ("NULL", dict(bounds=None)), ("SHAPE", dict(B=0)), ("SHAPE", dict(Hkv=65536)),
                           ("SHAPE", dict(capacity=0)), ("SHAPE", dict(d=32)), ("ALIGN", dict(k=0x1002)), ("ALIGN", dict(bounds=0x2008)),
                           ("SHAPE", dict(k_stride0=-8)), ("ALIGN", dict(k_stride1=4)), ("SHAPE", dict(k_stride2=64)),
                           ("SHAPE", dict(n_blocks=2)), ("SHAPE", dict(max_new=-1)), ("ALIGN", dict(seq_lens=0x3001)),
                           ("ALIGN", dict(from_lens=0x3002)), ("ALIGN", dict(block_table=0x3002)),
                           ("SHAPE", dict(block_table=0x3000, page_size=16, num_pages=9, block_table_stride=8)),
                           ("SHAPE", dict(block_table=0x3000, page_size=0, num_pages=9, block_table_stride=9))]:
        assert lib.parallax_cache_bounds(call(**fields), None) == getattr(binding, "PLX_ERR_" + status), fields
    for status, fields in _BAD_CACHES:
        cache = _q4(binding, **fields)
        assert lib.parallax_cache_bounds(call(cache), None) == getattr(binding, "PLX_ERR_" + status), fields
    assert lib.parallax_cache_bounds(call(_q4(binding, capacity=200)), None) == binding.PLX_ERR_SHAPE  # (four blocks)


def test_refusals_of_selection(binding):  # noqa: F811
    lib = binding.load_library()

    def call(**fields):
        a = binding.plx_select_blocks_args()
        a.q, a.bounds, a.block_list, a.workspace, a.workspace_bytes = 0x1000, 0x2000, 0x3000, 0x4000, 2 * 2 * 9 * 8
        a.B, a.Hq, a.Hkv, a.Tq, a.d, a.n_blocks, a.keep, a.first, a.recent = 2, 4, 2, 1, 128, 9, 5, 1, 2
        for name, value in fields.items():
            setattr(a, name, value)
        return ctypes.byref(a)

    assert lib.parallax_select_blocks(None, None) == binding.PLX_ERR_NULL
    for status, fields in [("NULL", dict(q=None)), ("NULL", dict(bounds=None)), ("NULL", dict(block_list=None)), ("SHAPE", dict(B=0)),
                           ("SHAPE", dict(Hq=5)), ("SHAPE", dict(Hkv=0)), ("SHAPE", dict(d=256)), ("SHAPE", dict(Tq=-1)), ("SHAPE", dict(Tq=9)),
                           ("SHAPE", dict(Hq=34)), ("SHAPE", dict(Tq=1 << 30)), ("SHAPE", dict(n_blocks=0)), ("SHAPE", dict(n_blocks=1 << 26)),
                           ("SHAPE", dict(keep=0)), ("SHAPE", dict(first=-1)), ("SHAPE", dict(recent=-1)), ("SHAPE", dict(keep=2)),
                           ("SHAPE", dict(first=2 ** 31 - 1, recent=2 ** 31 - 1)), ("ALIGN", dict(q=0x1008)), ("ALIGN", dict(bounds=0x2004)),
                           ("ALIGN", dict(seq_lens=0x5001)), ("ALIGN", dict(block_list=0x3002)), ("WORKSPACE", dict(workspace=None)),
                           ("WORKSPACE", dict(workspace=0x4008)), ("WORKSPACE", dict(workspace_bytes=2 * 2 * 9 * 8 - 1))]:
        assert lib.parallax_select_blocks(call(**fields), None) == getattr(binding, "PLX_ERR_" + status), fields
    assert lib.parallax_select_blocks_workspace_bytes(2, 2, 9) == 288
    assert lib.parallax_select_blocks_workspace_bytes(65535, 65535, 1 << 20) == 65535 * 65535 * (1 << 20) * 8
    assert [lib.parallax_select_blocks_workspace_bytes(*x) for x in ((0, 1, 1), (1, 0, 1), (1, 1, 0))] == [0, 0, 0]


def test_splits_of_q4_calls(binding):  # noqa: F811
    """On 256 compute units (what the library counts on without a GPU, too)."""
    lib = binding.load_library()

    def splits(B, Hkv, L, d=128, n=0, **fields):
        cache = dict(B=B, Hkv=Hkv, capacity=L, d=d)
        row = binding.parallax_q4_row_bytes(d)
        cache.update(stride0=Hkv * L * row, stride1=L * row, stride2=row)
        a = _q4_decode(binding, cache.items(), B=B, Hq=2 * Hkv, Hkv=Hkv, Lmax=L, d=d, num_splits=0, names=0x7000 if n else None, n=n,
                       **fields)
        return lib.parallax_decode_q4_call_splits(ctypes.byref(a))

    assert splits(1, 8, 500) == 1                     # a merge costs more than the shorter loop saves
    assert splits(1, 8, 1500) == 6                    # a tile for every wave
    assert splits(16, 8, 32768) in (2, 4)             # units full, few records
    assert splits(16, 8, 8192) == 2                   # 128 pairs on 256 units
    assert splits(64, 8, 2000) == 1
    assert splits(16, 8, 65536, n=64) == splits(16, 8, 4096)
    assert splits(4, 8, 100000, window=1000, sinks=24) == splits(4, 8, 1024)
    assert 1 <= splits(1, 1, 1 << 30, d=64) <= binding.PLX_MAX_SPLITS


def test_the_binding_refuses_host_tensors(binding):  # noqa: F811
    k = torch.zeros(1, 1, 4, 64, dtype=torch.bfloat16)
    cache = torch.zeros(1, 1, 8, 80, dtype=torch.uint8)
    bounds = torch.zeros(1, 1, 1, 2, 64, dtype=torch.bfloat16)
    q = torch.zeros(1, 1, 64, dtype=torch.bfloat16)
    for call in (lambda: binding.parallax_cache_write_q4(k, k, cache), lambda: binding.parallax_cache_read_q4(cache, 64, 4),
                 lambda: binding.parallax_decode_q4(q, q, cache, 0.1), lambda: binding.parallax_cache_bounds(k, bounds),
                 lambda: binding.parallax_select_blocks(q, bounds, None, 3),
                 lambda: binding.parallax_decode(q, q, k, k, 0.1, block_list=torch.zeros(1, 1, 1, dtype=torch.int32))):
        with pytest.raises(ValueError):
            call()


def test_one_place_for_several_rows_is_not_written(binding):  # noqa: F811
    """A cache that sequences or heads share by a stride of 0 can be read, and is refused by a write."""
    lib = binding.load_library()
    for fields, status in ((dict(stride0=0), binding.PLX_ERR_SHAPE), (dict(stride1=0), binding.PLX_ERR_SHAPE),
                           (dict(stride0=0, B=1), binding.PLX_OK), (dict(stride1=0, Hkv=1), binding.PLX_OK)):
        a = binding.plx_q4_rows_args()
        _q4(binding, a.cache, **fields)
        a.k, a.v, a.T, a.dtype = 0x3000, 0x4000, 0, binding.PLX_BF16
        a.k_stride[:] = a.v_stride[:] = (128, 128, 128)
        assert lib.parallax_cache_write_q4(ctypes.byref(a), None) == status, fields
        assert lib.parallax_cache_read_q4(ctypes.byref(a), None) == binding.PLX_OK, fields


def test_strides_of_rows_and_pages_have_a_limit(binding):  # noqa: F811
    lib = binding.load_library()
    table = dict(block_table=0x2000, page_size=16, num_pages=4, block_table_stride=4)
    for fields, status in ((dict(stride2=1 << 36), binding.PLX_ERR_SHAPE), (dict(stride0=1 << 36, **table), binding.PLX_ERR_SHAPE),
                           (dict(stride2=(1 << 36) - 16), binding.PLX_OK), (dict(stride0=1 << 40), binding.PLX_OK)):
        a = binding.plx_q4_rows_args()
        _q4(binding, a.cache, **fields)
        a.k, a.v, a.T, a.dtype = 0x3000, 0x4000, 0, binding.PLX_BF16
        a.k_stride[:] = a.v_stride[:] = (128, 128, 128)
        assert lib.parallax_cache_write_q4(ctypes.byref(a), None) == status, fields
        assert lib.parallax_cache_read_q4(ctypes.byref(a), None) == status, fields


def test_one_place_for_several_pages_is_not_written(binding):  # noqa: F811
    """Pools whose pages share one place can be read, and are refused by a write, as are sequences of one place without a table."""
    lib = binding.load_library()
    table = dict(block_table=0x2000, page_size=16, block_table_stride=4)
    for fields, status in ((dict(stride0=0, num_pages=4, **table), binding.PLX_ERR_SHAPE), (dict(stride0=0, num_pages=4, B=1, **table), binding.PLX_ERR_SHAPE),
                           (dict(stride1=0, num_pages=4, **table), binding.PLX_ERR_SHAPE), (dict(stride0=0, num_pages=1, **table), binding.PLX_OK),
                           (dict(num_pages=4, **table), binding.PLX_OK)):
        a = binding.plx_q4_rows_args()
        _q4(binding, a.cache, **fields)
        a.k, a.v, a.T, a.dtype = 0x3000, 0x4000, 0, binding.PLX_BF16
        a.k_stride[:] = a.v_stride[:] = (128, 128, 128)
        assert lib.parallax_cache_write_q4(ctypes.byref(a), None) == status, fields
        assert lib.parallax_cache_read_q4(ctypes.byref(a), None) == binding.PLX_OK, fields


def test_one_place_for_several_rows_is_not_read_into(binding):  # noqa: F811
    """Rows that sequences or heads share by a stride of 0 can be written from, and are refused as what a read back writes."""
    lib = binding.load_library()
    for tensor in ("k_stride", "v_stride"):
        for axis, alone in ((0, dict(B=1)), (1, dict(Hkv=1))):
            for fields, status in ((dict(), binding.PLX_ERR_SHAPE), (alone, binding.PLX_OK)):
                a = binding.plx_q4_rows_args()
                _q4(binding, a.cache, **fields)
                a.k, a.v, a.T, a.dtype = 0x3000, 0x4000, 0, binding.PLX_BF16
                a.k_stride[:] = a.v_stride[:] = (256, 128, 128)
                getattr(a, tensor)[axis] = 0
                assert lib.parallax_cache_read_q4(ctypes.byref(a), None) == status, (tensor, axis, fields)
                assert lib.parallax_cache_write_q4(ctypes.byref(a), None) == binding.PLX_OK, (tensor, axis, fields)
