"""How far decode over 4-bit rows and over lists of blocks is from exact on ordinary inputs: no further than the rounding of its result.

A value m 2^e, 1 <= m < 2, rounded to bf16 is off by up to 2^-8 2^e, evenly: 2^-8 / sqrt(3) = 2.26e-3 in the square mean against a mean m^2 of
about 2 (between 1.9 and 2.4 for sums of many products): 1.65e-3 of the whole, 1.7e-3 with what is left of weights in 11 bits (2^-11, 1/8 of it).
Weights in one bf16 add as much again, 2.3e-3. In between: 2.0e-3.
"""
import numpy as np
import pytest
import torch

from oracle import blocks, masked, rows
from parity import host, rel_l2
from test_gpu_q4 import DEV, _normal, plx  # noqa: F401

pytestmark = pytest.mark.gpu

MOST = 2.0e-3
# off by, of a weight: 11 bits 2^-11; a bf16 and one for what it leaves 2^-16; scores in fp32 (errors of 2^-24 of up to 40 at each of a few steps) 2^-15
EPS_Q4, EPS_LIST = 2.0 ** -11 + 2.0 ** -15, 2.0 ** -14


def _far(got, q, r, k, v, scale, see, eps_p):
    got = host(got).astype(np.float64)
    ref = masked.masked_forward(q, r, k, v, scale, see)
    bound = rows.bf16_bound(q, r, k, v, scale, see, eps_p=eps_p)
    assert (np.abs(got - ref) <= bound).all(), float((np.abs(got - ref) / bound).max())
    return rel_l2(got, ref)


@pytest.mark.parametrize("lists", [False, True])
@pytest.mark.parametrize("d,Hq,Hkv,Tq", [(128, 16, 8, 1), (128, 8, 2, 1), (128, 8, 2, 2), (128, 8, 1, 2), (64, 16, 8, 1), (64, 8, 2, 2), (64, 8, 1, 2)])
def test_no_further_than_the_rounding_of_the_result(plx, d, Hq, Hkv, Tq, lists):  # noqa: F811
    B, L = 2, 1500
    k, v = (_normal((B, Hkv, L, d), s) for s in (1, 2))
    q, r = (_normal((B, Hq, Tq, d), s) for s in (3, 4))
    cache = torch.zeros(B, Hkv, L, blocks.row_bytes(d), dtype=torch.uint8, device=DEV)
    plx.parallax_cache_write_q4(k, v, cache)
    k4, v4 = blocks.unpack(cache.cpu().numpy(), d)
    see = np.broadcast_to(rows.chain(L, Tq, L)[None, None], (B, Hq, Tq, L))
    more = {}
    if lists:
        rng = np.random.default_rng(5)
        names = [[sorted(rng.choice(24, 14, replace=False).tolist()) for _ in range(Hkv)] for _ in range(B)]
        more = dict(block_list=torch.tensor(names, dtype=torch.int32, device=DEV))
        named = np.stack([np.stack([blocks.listed_keys(x, L, L) for x in of]) for of in names])
        see = see & np.repeat(named, Hq // Hkv, axis=1)[:, :, None]
    hq, hr = host(q).astype(np.float64), host(r).astype(np.float64)
    for S in (1, 3):
        got = plx.parallax_decode_q4(q, r, cache, d ** -0.5, num_splits=S, **more)
        assert _far(got, hq, hr, k4, v4, d ** -0.5, see, EPS_Q4) <= MOST, S
        if lists:
            got = plx.parallax_decode(q, r, k, v, d ** -0.5, num_splits=S, **more)
            assert _far(got, hq, hr, host(k).astype(np.float64), host(v).astype(np.float64), d ** -0.5, see, EPS_LIST) <= MOST, S
