"""Pins of the oracle for 4-bit rows, block bounds and selection."""
import math

import numpy as np
import pytest

from oracle import blocks


def test_codes_of_halfway_values():
    e = 127 + 3  # scale 8
    for x, want in ((0.25, 0.0), (0.75, 1.0), (1.25, 1.0), (1.75, 2.0), (2.5, 2.0), (3.5, 4.0), (5.0, 4.0), (5.01, 6.0), (6.99, 6.0)):
        for sign in (1, -1):
            c = blocks.code(sign * 8 * x, e)
            assert blocks.LEVELS[c & 7] == want and (c >> 3) == (sign < 0)


def test_scales():
    for top, e in ((3.5, 127), (6.99, 127), (7.0, 128), (3.49, 126), (0.0, 4), (2.0 ** -130, 4), (1e30, 127 + 97),
                   (3.3895313892515355e38, 252), (float("inf"), 255), (float("nan"), 255)):
        assert blocks.group_scale(np.array([0.0, -top] + [0.0] * 14)) == e, top


@pytest.mark.parametrize("d", [64, 128])
def test_rows_come_back(d):
    rng = np.random.default_rng(d)
    k, v = rng.standard_normal((2, d))
    row = blocks.pack_row(k, v)
    assert row.shape == ({64: 80, 128: 144}[d],) and not row[d + d // 8:].any()
    for x, y in zip((k, v), blocks.unpack(row, d)):
        # half a step of the code: 0.25, 0.5 or 1 of a scale that is at most 2 / 7 of the largest magnitude
        top = np.repeat(np.abs(x).reshape(-1, 16).max(1), 16)
        assert (np.abs(x - y) <= top / 3.5 * np.where(np.abs(x) < top / 7 * 2, 0.5, 1.0)).all()
        assert np.array_equal(blocks.unpack(blocks.pack_row(y, y), d)[0], y)  # (a row of codes is one already)


def test_no_key_scores_above_its_block():
    rng = np.random.default_rng(0)
    k, q = rng.standard_normal((200, 64)), rng.standard_normal((3, 64))
    low, high = blocks.bounds(k, 200)
    assert low.shape == (4, 64)
    best = np.maximum(q[:, None] * low, q[:, None] * high).sum(-1)
    for j in range(4):
        assert ((q @ k[64 * j: 64 * j + 64].T).max(1) <= best[:, j] + 1e-12).all()


def test_selection():
    low = np.zeros((6, 64))
    high = np.zeros((6, 64))
    high[:, 0] = [1, 5, 2, 5, 5, 1]
    q = np.zeros((1, 64))
    q[0, 0] = 2.0
    assert blocks.select(q, low, high, 4, 1, 1) == [0, 1, 3, 5]
    assert blocks.select(q, low, high, 3, 0, 0) == [1, 3, 4]
    assert blocks.select(q, low, high, 9, 1, 1) == [0, 1, 2, 3, 4, 5]
    high[4, 3] = np.nan
    assert blocks.select(q, low, high, 1, 0, 0) == [4]


def test_listed_keys():
    see = blocks.listed_keys([0, 0, 2, -1, 7], 140, 200)
    assert see.sum() == 64 + 12 and see[:64].all() and see[128:140].all()


def test_sums_of_products_within_2_to_the_30_are_exact_in_any_order():
    """128 products of two bf16 (integers below 2^16 times powers of two): with the largest 2^30 times the smallest that is not 0, sums of 64
    bits have no rounding; at 2^37 they have."""
    def orders(x):
        yield x
        yield x[::-1]
        rng = np.random.default_rng(1)
        for _ in range(20):
            yield rng.permutation(x)

    def sums(x):
        for y in orders(x):
            total = 0.0
            for v in y.tolist():
                total += v
            yield total
            yield float(y.reshape(16, 8).sum(1).reshape(2, 8).sum(0).sum())

    for small in (255 * 255, 129 * 129, 193 * 255, 2 ** 14):  # (significands of 8 bits each)
        for sign in (1.0, -1.0):
            high = float(255 * 255)
            e = math.floor(math.log2(2.0 ** 30 * small / high))
            x = np.full(128, high * 2.0 ** e)
            assert 2.0 ** 29 < x[0] / small <= 2.0 ** 30
            x[::3] = sign * small
            x[1::5] *= -1.0
            assert set(sums(x)) == {math.fsum(x)}, (small, sign)
            x[:] = high * 2.0 ** e
            x[77] = small  # the sum is as large as it gets
            assert set(sums(x)) == {math.fsum(x)}
    x = np.array([255.0 * 255 * 2.0 ** 35] * 64 + [129.0 * 129 * 2.0 ** -1] * 64)
    assert len(set(sums(x))) > 1
