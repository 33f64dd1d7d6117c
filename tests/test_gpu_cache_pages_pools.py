"""Pools that do not fit the table they are extended with are refused before anything changes."""
import numpy as np
import pytest
import torch

from test_gpu_cache_pages import DEV, _ints, _same, _state, plx  # noqa: F401

pytestmark = pytest.mark.gpu


def test_extend_looks_at_all_pools_first(plx):
    """A pool that does not fit, of whichever layer, is refused before the table changes."""
    t, o = _state(plx, 3, 6, 20, 4, np.random.default_rng(3))
    pool = lambda *shape, dtype=torch.bfloat16: torch.randn(*shape, device=DEV).to(dtype)
    k, v = pool(20, 2, 4, 64), pool(20, 2, 4, 64)
    assert plx.parallax_cache_extend(t, _ints([0]), _ints([6]), k, v).tolist() == [0]
    o.extend([0], [6])
    plx.parallax_cache_fork(t, _ints([0]), _ints([1]))
    o.fork([0], [1])
    odd = pool(20 * 2 * 4 * 64 + 1)[1:].view(20, 2, 4, 64)  # 2 bytes off a multiple of 16
    bad = [(k, v[:, :1]), (k, v.float()), (k[:19], v[:19]), (k[:, :, :3], v[:, :, :3]), (k, v[:19]), (k, v[:, :, :3]),
           (odd, v), (k, odd), (k.transpose(2, 3), v.transpose(2, 3)), (pool(20, 2, 4, 60), pool(20, 2, 4, 60)),
           (k.half(), v.half()), (k.cpu(), v), (k, v.cpu()), (pool(20, 2, 4, 64, 1), v), (pool(20, 2, 4, 68)[..., :64], v)]
    rows_before = k.clone(), v.clone()
    for pools in bad:
        for layers in (pools, (k, v, *pools), (*pools, k, v)):
            with pytest.raises((ValueError, TypeError, RuntimeError)):
                plx.parallax_cache_extend(t, _ints([0, 1]), _ints([9, 8]), *layers)
            _same(t, o)
    assert torch.equal(k, rows_before[0]) and torch.equal(v, rows_before[1])
    assert plx.parallax_cache_extend(t, _ints([0, 1]), _ints([9, 8]), k, v).tolist() == [0]
    o.extend([0, 1], [9, 8])
    _same(t, o)
