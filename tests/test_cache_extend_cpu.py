"""parallax_cache_extend looks at the pools of every layer before it changes the table (the library's calls recorded, no GPU)."""
from types import SimpleNamespace

import pytest
import torch


@pytest.fixture
def extend(monkeypatch):
    """(call, names of the entry points that it reached): a table of 20 pages of 4 tokens; the checks of devices are left out."""
    from paper_2605_29157_amd import binding

    real, reached = binding.load_library(), []

    def cache_extend(*args):
        reached.append("extend")
        return binding.PLX_OK

    def cache_copy(pools, src, dst, rows, n, stream):
        if n:
            reached.append("copy")
            return binding.PLX_OK
        return real.parallax_cache_copy(pools, src, dst, rows, n, stream)  # (launches nothing)

    monkeypatch.setattr(binding, "load_library", lambda: SimpleNamespace(parallax_cache_extend=cache_extend, parallax_cache_copy=cache_copy,
                                                                           parallax_strerror=real.parallax_strerror))
    monkeypatch.setattr(binding, "_on_current_device", lambda *a: None)
    monkeypatch.setattr(binding, "_table_device", lambda *a: 0)
    monkeypatch.setattr(binding, "_int_list", lambda where, name, t, *a: t.data_ptr())
    monkeypatch.setattr(binding, "_launch_stream", lambda *a: 0)
    monkeypatch.setattr(binding, "_result_maker", lambda stream, make: make)
    ints = torch.zeros(20, dtype=torch.int32)
    pages = SimpleNamespace(_args=binding.plx_page_table(), page_refs=ints, block_table=ints.view(4, 5), page_size=4)
    return lambda *pools: binding.parallax_cache_extend(pages, ints[:2], ints[:2], *pools), reached


def _pool(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype)


BAD = [lambda k: (k, k[:, :1]), lambda k: (k, k.float()), lambda k: (k[:19], k[:19]), lambda k: (k[:, :, :3], k[:, :, :3]),
       lambda k: (k, k[:19]), lambda k: (k.transpose(2, 3), k.transpose(2, 3)), lambda k: (_pool(20, 2, 4, 60), _pool(20, 2, 4, 60)),
       lambda k: (k.half(), k.half()), lambda k: (_pool(20 * 512 + 1)[1:].view(20, 2, 4, 64), k),
       lambda k: (k, _pool(20 * 512 + 1)[1:].view(20, 2, 4, 64)), lambda k: (_pool(20, 2, 4, 68)[..., :64], k), lambda k: (k,)]


@pytest.mark.parametrize("bad", range(len(BAD)))
@pytest.mark.parametrize("good_before", [0, 2])
def test_a_pool_that_does_not_fit(extend, bad, good_before):
    call, reached = extend
    k = _pool(20, 2, 4, 64)
    layers = [k] * (2 * good_before) + list(BAD[bad](k))
    with pytest.raises((ValueError, TypeError, RuntimeError)):
        call(*layers)
    assert reached == []


def test_pools_that_fit(extend):
    call, reached = extend
    k, latent = _pool(20, 2, 4, 64), _pool(20, 4, 576)
    call(k, k, latent, None)
    assert reached == ["extend", "copy", "copy"]
    call()
    assert reached == ["extend", "copy", "copy", "extend"]
