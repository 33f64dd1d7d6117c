"""Pins of the oracle for 4-bit rows, block bounds and selection."""
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
