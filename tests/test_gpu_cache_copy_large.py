"""Pages near the most chunks that a copy takes (2^30 - 1 a pool): heads that all name the same rows, so that little memory is
needed."""
import pytest
import torch

from test_gpu_cache_pages import DEV, _ints, plx  # noqa: F401

pytestmark = pytest.mark.gpu


def test_the_largest_page(plx):
    heads, page, d = 65535, 128, 1024
    chunks = heads * page * d * 2 // 16  # of one pool; a thread's next one, 65535 x 256 further on, is behind 2^31
    assert chunks < 2**30 and 2 * chunks + 65535 * 256 > 2**31
    gen = torch.Generator().manual_seed(1)
    base = [torch.randn(4, 1, page, d, generator=gen).to(torch.bfloat16).to(DEV) for _ in range(2)]
    want = [b.clone() for b in base]
    for w in want:
        w[2] = w[1]
    plx.parallax_cache_copy(*(b.expand(4, heads, page, d) for b in base), _ints([1]), _ints([2]))
    for b, w in zip(base, want):
        assert torch.equal(b, w)
