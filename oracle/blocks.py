"""Caches held in 4 bits, and blocks of keys that a score picks -- CPU ORACLE in numpy (test infrastructure, not product):
plain loops over the definitions.

A 4-bit row: d / 2 bytes of K codes, d / 2 of V codes (dimension 2 i in the low half of byte i), d / 16 scale bytes of K and of V,
zeros up to a multiple of 16. A code is a sign over one of LEVELS; scale byte e: 2^(e - 127) for 16 dimensions, 255: NaN. The
scale written brings the largest magnitude into [3.5, 7), e within 4 .. 252; of two codes equally near the even one.
"""
from __future__ import annotations

import math

import numpy as np

LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def row_bytes(d):
    return -(-(d + d // 8) // 16) * 16


def group_scale(x):
    """The scale byte of 16 numbers."""
    if not np.all(np.isfinite(x)):
        return 255
    top = max(abs(float(v)) for v in x)
    e = 4
    while e < 252 and math.ldexp(top, 127 - e) >= 7.0:
        e += 1
    return e


def code(x, e):
    """The code of x under scale byte e."""
    a = abs(math.ldexp(float(x), 127 - e))
    best = min(range(8), key=lambda i: (abs(a - LEVELS[i]), i % 2))
    return best + (8 if math.copysign(1.0, float(x)) < 0 else 0)


def pack_row(k, v):
    """k, v [d] -> uint8 [row_bytes(d)]"""
    d = len(k)
    out = np.zeros(row_bytes(d), dtype=np.uint8)
    for i, x in enumerate((k, v)):
        for g in range(d // 16):
            part = x[16 * g: 16 * g + 16]
            e = group_scale(part)
            out[d + i * (d // 16) + g] = e
            if e == 255:
                continue
            for n in range(16):
                out[i * (d // 2) + 8 * g + n // 2] |= code(part[n], e) << (4 * (n % 2))
    return out


def unpack(rows, d):
    """uint8 [.., row_bytes(d)] -> K, V [.., d] in double precision"""
    rows = np.asarray(rows, dtype=np.uint8)
    signed = np.array(list(LEVELS) + [-x for x in LEVELS])
    both = []
    for i in (0, 1):
        codes = rows[..., i * (d // 2): (i + 1) * (d // 2)]
        x = np.stack([signed[codes & 15], signed[codes >> 4]], -1).reshape(*rows.shape[:-1], d)
        e = rows[..., d + i * (d // 16): d + (i + 1) * (d // 16)].astype(np.float64)
        s = np.where(e == 255, np.nan, np.exp2(e - 127.0))
        both.append(x * np.repeat(s, 16, axis=-1))
    return both


def bounds(k, length, block=64):
    """Keys [cap, d] of a sequence of `length` -> (smallest, largest) [ceil(length / block), d]"""
    low, high = [], []
    for j in range(0, length, block):
        part = k[j: min(j + block, length)]
        low.append(part.min(axis=0))
        high.append(part.max(axis=0))
    return np.array(low), np.array(high)


def select(q, low, high, keep, first, recent):
    """q [columns, d], bounds [n, d] -> the sorted numbers of the blocks kept"""
    n = len(low)
    score = []
    for j in range(n):
        if not (np.all(np.isfinite(low[j])) and np.all(np.isfinite(high[j]))):
            score.append(math.inf)
            continue
        sums = [math.fsum(max(float(a) * float(l), float(a) * float(h)) for a, l, h in zip(x, low[j], high[j])) for x in q]
        score.append(math.inf if any(math.isnan(s) for s in sums) else max(sums))
    forced = set(range(min(first, n))) | set(range(max(n - recent, 0), n))
    order = sorted(range(n), key=lambda j: (j not in forced, -score[j], j))
    return sorted(order[:keep])


def listed_keys(names, length, cap, block=64):
    """The keys that a list of a sequence of `length` tokens names: bool [cap]"""
    see = np.zeros(cap, dtype=bool)
    for i, n in enumerate(names):
        if 0 <= n <= (length - 1) // block and (i == 0 or n > names[i - 1]):
            see[block * n: min(block * n + block, length)] = True
    return see
