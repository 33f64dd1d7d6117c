"""Decode over 4-bit rows where sizes are far apart: keys of little weight with large values or large products rho.k, keys of
large weight with values of zero, values near the ends of bf16's range.

Weights are rounded to the 11 bits of f16 (off by at most 2^-11 of themselves) or cut to 16. Where they are f16 the largest of 64 neighbours
is at least 2^-12 of the row's largest in all tiles that a sum here comes from. It counts 2^13 (P rho.k: 2^7) times that, times a scale of
at least 2^-7, and products are multiples of 2^-24: off by at most 2^-12 of that largest weight times scale. Scores (sums of d products in fp32,
magnitudes up to 120, errors of 2^-24 of that for each of a few steps) and the exponentials add less than 2^-15: 2^-11 + 2^-12 + 2^-15 < 2^-10.
"""
import numpy as np
import pytest
import torch

from oracle import blocks, masked, rows
from parity import host
from test_gpu_q4 import DEV, _normal, plx  # noqa: F401

pytestmark = pytest.mark.gpu

EPS_P = 2.0 ** -10
SHAPES = [(128, 2, 1), (128, 4, 1), (128, 8, 1), (128, 8, 2), (64, 3, 1), (64, 4, 2), (64, 4, 4)]  # d, Hq, Tq


def _compare(plx, q, r, k, v, splits=(1, 2, 5), seen=None):  # noqa: F811
    """k, v [1, 1, L, d] (fp32) as 4-bit rows, against the values that the rows stand for."""
    d, Tq, L = q.shape[-1], q.shape[2], k.shape[2]
    cache = torch.zeros(1, 1, L, blocks.row_bytes(d), dtype=torch.uint8, device=DEV)
    plx.parallax_cache_write_q4(k, v, cache)
    hk, hv = blocks.unpack(cache.cpu().numpy(), d)
    hq, hr = host(q).astype(np.float64), host(r).astype(np.float64)
    see = np.broadcast_to(rows.chain(L, Tq, L)[None, None], (1, q.shape[1], Tq, L))
    ref = masked.masked_forward(hq, hr, hk, hv, d ** -0.5, see)
    bound = rows.bf16_bound(hq, hr, hk, hv, d ** -0.5, see, eps_p=EPS_P)
    for S in splits:
        got = host(plx.parallax_decode_q4(q, r, cache, d ** -0.5, num_splits=S)).astype(np.float64)
        assert np.isfinite(got).all(), S
        assert (np.abs(got - ref) <= bound).all(), (S, float((np.abs(got - ref) / np.maximum(bound, 1e-300)).max()))


def _inputs(d, Hq, Tq, L, seed=1):
    """Rows that all ask the same, so that one key can be far from all of them."""
    k, v = (_normal((1, 1, L, d), seed + i).float() for i in (0, 1))
    q = _normal((1, 1, 1, d), seed + 2).expand(1, Hq, Tq, d).contiguous()
    return q, _normal((1, Hq, Tq, d), seed + 3), k, v


def _against(q, scale, score):
    """A key whose scaled product with q is `score`."""
    x = q[0, 0, 0].float()
    return score / scale * x / (x * x).sum()


@pytest.mark.parametrize("power", [14, 17, 30, 50, 100])
@pytest.mark.parametrize("place", ["first", "64th", "middle", "last"])
@pytest.mark.parametrize("d,Hq,Tq", SHAPES)
def test_a_large_value_of_no_weight(plx, d, Hq, Tq, place, power):  # noqa: F811
    """One key's values are 2^power larger than the others', its score 60 below theirs (a weight of 2^-86)."""
    L = 1500
    at = {"first": 0, "64th": 63, "middle": L // 2, "last": L - Tq}[place]
    q, r, k, v = _inputs(d, Hq, Tq, L)
    k[0, 0, at] = _against(q, d ** -0.5, -60.0)
    v[0, 0, at] *= 2.0 ** power
    _compare(plx, q, r, k, v)


@pytest.mark.parametrize("power", [10, 20, 30])
@pytest.mark.parametrize("d,Hq,Tq", SHAPES)
def test_a_large_value_whose_weight_makes_up_for_it(plx, d, Hq, Tq, power):  # noqa: F811
    """Keys of weights around 2^-power with values 2^power larger: what they add is of the size of all others."""
    L = 900
    q, r, k, v = _inputs(d, Hq, Tq, L)
    for at in (5, 400, 700):
        k[0, 0, at] = _against(q, d ** -0.5, -power * np.log(2.0))
        v[0, 0, at] *= 2.0 ** power
    _compare(plx, q, r, k, v)


@pytest.mark.parametrize("score", [8.0, 14.0, 20.0])
@pytest.mark.parametrize("d,Hq,Tq", SHAPES)
def test_a_heavy_key_without_a_value(plx, d, Hq, Tq, score):  # noqa: F811
    """The first key has nearly all of the weight and values of zero: the result is made of the others."""
    q, r, k, v = _inputs(d, Hq, Tq, 700)
    k[0, 0, 0] = _against(q, d ** -0.5, score)
    v[0, 0, 0] = 0.0
    _compare(plx, q, r, k, v)


@pytest.mark.parametrize("power", [14, 30, 50])
@pytest.mark.parametrize("d,Hq,Tq", SHAPES)
def test_a_large_probe_product_of_no_weight(plx, d, Hq, Tq, power):  # noqa: F811
    """One key's rho.k is 2^power larger than the others', with a weight that leaves nothing of it."""
    q, r, k, v = _inputs(d, Hq, Tq, 700)
    q[..., d // 2:] = 0
    k[0, 0, 3] = _against(q, d ** -0.5, -60.0)
    k[0, 0, 3, d // 2:] = r[0, 0, 0, d // 2:].float() * 2.0 ** power
    _compare(plx, q, r, k, v)


@pytest.mark.parametrize("score", [-120.0, 120.0])
@pytest.mark.parametrize("d,Hq,Tq", SHAPES)
def test_scores_that_jump(plx, d, Hq, Tq, score):  # noqa: F811
    """The first 320 keys' scores are 2^173 times smaller or larger than all that follow: nothing, or all, of the result is theirs."""
    q, r, k, v = _inputs(d, Hq, Tq, 700)
    k[0, 0, :320] = _against(q, d ** -0.5, score) + k[0, 0, :320] / 64
    v[0, 0, :320] *= 4.0
    _compare(plx, q, (r.float() / 16).to(torch.bfloat16), k, v)


@pytest.mark.parametrize("power", [-98, 118, 122, 124])
@pytest.mark.parametrize("d,Hq,Tq", SHAPES)
def test_values_near_the_ends_of_the_range(plx, d, Hq, Tq, power):  # noqa: F811
    q, r, k, v = _inputs(d, Hq, Tq, 130)
    _compare(plx, q, (r.float() / 16).to(torch.bfloat16), k, v * 2.0 ** power)


@pytest.mark.parametrize("large", [3.0, 8.0])
@pytest.mark.parametrize("d,Hq,Tq", SHAPES)
def test_rows_with_few_heavy_keys(plx, d, Hq, Tq, large):  # noqa: F811
    """Scores of a standard deviation of 3 or 8, values whose size changes from block to block and dimension to dimension."""
    L = 2000
    q, r, k, v = _inputs(d, Hq, Tq, L)
    q = (_normal((1, Hq, Tq, d), 9).float() * large).to(torch.bfloat16)
    v = v * torch.exp2((torch.arange(L, device=DEV) // 64 % 13 - 6).float())[:, None] * torch.exp2((torch.arange(d, device=DEV) // 16 % 5 - 2).float())
    _compare(plx, q, r, k, v)


@pytest.mark.parametrize("codes", ["any", "zeros"])
@pytest.mark.parametrize("at", [70, 450, 510])
@pytest.mark.parametrize("d,Hq,Tq", SHAPES)
def test_scale_255_is_nan_to_a_decode_too(plx, d, Hq, Tq, at, codes):  # noqa: F811
    """Rows from elsewhere with scale byte 255 and codes that are not 0: NaN in the 16 dimensions of V for the rows that see them, whatever the
    codes, as reading them back gives; all else as it was."""
    L, group = 512, 1
    q, r = _normal((1, Hq, Tq, d), 1), _normal((1, Hq, Tq, d), 2)
    cache = torch.zeros(1, 1, L, blocks.row_bytes(d), dtype=torch.uint8, device=DEV)
    plx.parallax_cache_write_q4(_normal((1, 1, L, d), 3), _normal((1, 1, L, d), 4), cache)
    want = host(plx.parallax_decode_q4(q, r, cache, d ** -0.5, num_splits=1))
    if codes == "zeros":
        cache[0, 0, at, d // 2 + 8 * group: d // 2 + 8 * group + 8] = 0
    cache[0, 0, at, d + d // 16 + group] = 255
    v = host(plx.parallax_cache_read_q4(cache, d, L)[1])
    assert np.isnan(v[0, 0, at, 16 * group: 16 * group + 16]).all() and np.isnan(v).sum() == 16
    names = torch.arange(8, dtype=torch.int32, device=DEV).reshape(1, 1, 8)
    for more in (dict(num_splits=1), dict(num_splits=3), dict(block_list=names)):
        got = host(plx.parallax_decode_q4(q, r, cache, d ** -0.5, **more))
        nan = np.zeros(got.shape, dtype=bool)
        for t in range(Tq):
            nan[:, :, t, 16 * group: 16 * group + 16] = at <= L - Tq + t
        assert np.array_equal(np.isnan(got), nan), more
        assert np.isfinite(got[~nan]).all() and np.linalg.norm((got - want)[~nan]) <= 1e-2 * np.linalg.norm(want[~nan])
