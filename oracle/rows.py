"""Which cached keys the rows of a decode call see -- CPU ORACLE in numpy (test infrastructure, not product): plain
loops over the definitions, for oracle/masked.py to sum over.

`chain`: the rows are the last Tq positions of a sequence of L cached tokens; a row at position pos sees the keys
j <= pos with j > pos - window or j < sinks (window 0: all).
`tree`: the last n = min(drafted, Tq, L) cached tokens are drafted nodes behind base = L - n committed ones. Node t < n
is at position base + (number of its bits) - 1 (no bits: base) and sees the committed keys and the drafted key base + m of
every node m whose bit it has, all of them with window > 0 only where their position is > its own - window, or < sinks (a
committed key's position is its place in the cache). Node t >= n sees nothing.
"""
from __future__ import annotations

import numpy as np


def chain(L, Tq, cap, window=0, sinks=0):
    see = np.zeros((Tq, cap), dtype=bool)
    for t in range(Tq):
        pos = L - Tq + t
        for j in range(max(pos + 1, 0)):
            see[t, j] = window == 0 or j > pos - window or j < sinks
    return see


def tree(L, Tq, cap, bits, drafted=None, window=0, sinks=0):
    n = min(Tq if drafted is None else max(drafted, 0), Tq, L)
    base = L - n
    see = np.zeros((Tq, cap), dtype=bool)
    pos = [base + max(int(sum(bits[t][:n])) - 1, 0) for t in range(n)]
    for t in range(n):
        for j in range(base):
            see[t, j] = window == 0 or j > pos[t] - window or j < sinks
        for m in range(n):
            see[t, base + m] = bits[t][m] and (window == 0 or pos[m] > pos[t] - window or pos[m] < sinks)
    return see


def words(bits):
    """bits [.., Tq, Tq] -> int64 words [.., Tq, ceil(Tq / 64)]"""
    bits = np.asarray(bits, dtype=bool)
    Tq = bits.shape[-1]
    out = np.zeros(bits.shape[:-1] + (-(-Tq // 64),), dtype=np.uint64)
    for m in range(Tq):
        out[..., m // 64] |= bits[..., m].astype(np.uint64) << np.uint64(m % 64)
    return out.view(np.int64)


def random_tree(Tq, rng, reach=6):
    """Ancestor bits [Tq, Tq] of a random tree (several roots, parents up to `reach` nodes back)."""
    bits = np.zeros((Tq, Tq), dtype=bool)
    for t in range(Tq):
        parent = int(rng.integers(max(-1, t - reach - 1), t)) if t else -1
        if parent >= 0:
            bits[t] = bits[parent]
        bits[t, t] = True
    return bits


def bf16_bound(q, r, k, v, scale, mask, eps=2.0 ** -8, eps_p=None):
    """Element-wise bound on a bf16 kernel's error that rounds P1 = p, P2 = p u and the output to bf16 (half a step is 2^-8 of
    a value) and keeps everything else in fp32: O1 and d1 hold the same rounded P1, O2 and d2 the same rounded P2, so
    with o = O1 / d1 (1 + d2 / d1) - O2 / d1
        |err| <= 2^-8 (|o| + 2 |1 + ubar| sum p |v| + sum p |u| |v| + 3 (sum p |u|) sum p |v|) + second order
    (each quotient by d1 moves by at most 2^-8 of itself); 1.02 covers the second order and the fp32 sums.
    eps_p: what P1 and P2 are off by, relative to them, where a kernel holds them in other bits than the output."""
    eps_p = eps if eps_p is None else eps_p
    q, r, k, v = (np.asarray(x, dtype=np.float64) for x in (q, r, k, v))
    B, Hq, Tq, d = q.shape
    G = Hq // k.shape[1]
    mask = np.broadcast_to(np.asarray(mask, dtype=bool), (B, Hq, Tq, k.shape[2]))
    bound = np.zeros_like(q)
    for b in range(B):
        for h in range(Hq):
            K, V, M = k[b, h // G], v[b, h // G], mask[b, h]
            V = np.where(M.any(axis=0)[:, None], V, 0.0)
            K = np.where(M.any(axis=0)[:, None], K, 0.0)
            A = np.where(M, scale * (q[b, h] @ K.T), -np.inf)
            amax = A.max(axis=1, keepdims=True)
            W = np.where(M, np.exp(A - np.where(np.isfinite(amax), amax, 0.0)), 0.0)
            P = W / np.maximum(W.sum(axis=1, keepdims=True), 1e-300)
            U = r[b, h] @ K.T
            ubar, ua = (P * U).sum(axis=1, keepdims=True), (P * np.abs(U)).sum(axis=1, keepdims=True)
            o = (P * (1 + ubar - U)) @ V
            pv = P @ np.abs(V)
            bound[b, h] = 1.02 * (eps * np.abs(o) + eps_p * (2 * np.abs(1 + ubar) * pv + (P * np.abs(U)) @ np.abs(V) + 3 * ua * pv))
    return bound


def bf16_backward_bound(q, r, k, v, d_o, scale, mask, eps=2.0 ** -8):
    """Element-wise bounds on the error of bf16 gradients (dq, dr, dk, dv) of the closed forms of App. D where the forward's
    o and vbar come in bf16 (o off by at most bf16_bound, vbar by 2^-8 (|vbar| + 2 sum p |v|): rounded P1 in both sums, then
    rounded itself), the weights g1, g2 and w = p (1 + ubar - u) are rounded to bf16 as matrix operands and the results
    once more, and all else is fp32. With eps = 2^-8, a = dO.v, delta = a - beta:
        tau = dO.o moves by dt <= sum |dO| |do|,   beta = dO.vbar by db <= sum |dO| |dvbar|
        g1 = p (a - tau + (ubar - u) delta) by p (dt + |ubar - u| db) + eps |g1|,   g2 = -p delta by p db + eps |g2|
        dq = scale sum g1 k,  dr = sum g2 k,  dk = scale sum g1 q + sum g2 r,  dv = sum w dO:  the sums of these moves, + eps
    fp32 steps: scores are sums of d products, so p is off by d 2^-24 sum |q k| scale of itself, u by d 2^-24 sum |r k|,
    and a - tau + .. is a difference of terms whose sizes are added up (64 2^-24 covers exp2 and the sums of each).
    fp32 throughout: eps = 64 2^-24 (a sum over keys or rows adds a few dozen terms one after the other: blocks of 16
    dealt to four waves)."""
    q, r, k, v, d_o = (np.asarray(x, dtype=np.float64) for x in (q, r, k, v, d_o))
    B, Hq, Tq, d = q.shape
    G, tiny = Hq // k.shape[1], 2.0 ** -24
    mask = np.broadcast_to(np.asarray(mask, dtype=bool), (B, Hq, Tq, k.shape[2]))
    off_o = bf16_bound(q, r, k, v, scale, mask, eps)
    out = [np.zeros_like(q), np.zeros_like(q), np.zeros_like(k), np.zeros_like(k)]
    exact = [np.zeros_like(k), np.zeros_like(k)]  # dk, dv, for their own rounding
    for b in range(B):
        for h in range(Hq):
            hk = h // G
            K, V, M, Q, R, D = k[b, hk], v[b, hk], mask[b, h], q[b, h], r[b, h], d_o[b, h]
            A = np.where(M, scale * (Q @ K.T), -np.inf)
            amax = A.max(axis=1, keepdims=True)
            W = np.where(M, np.exp(A - np.where(np.isfinite(amax), amax, 0.0)), 0.0)
            P = W / np.maximum(W.sum(axis=1, keepdims=True), 1e-300)
            U, a = R @ K.T, D @ V.T
            ubar = (P * U).sum(axis=1, keepdims=True)
            c = 1 + ubar - U
            o, vbar = (P * c) @ V, P @ V
            tau, beta = (D * o).sum(axis=1, keepdims=True), (D * vbar).sum(axis=1, keepdims=True)
            dt = (np.abs(D) * off_o[b, h]).sum(axis=1, keepdims=True)
            db = (np.abs(D) * eps * (np.abs(vbar) + 2 * (P @ np.abs(V)))).sum(axis=1, keepdims=True)
            delta = a - beta
            g1, g2, w = P * (a - tau + (ubar - U) * delta), -P * delta, P * c
            size_a = np.abs(D) @ np.abs(V).T + (np.abs(D) * (P @ np.abs(V))).sum(axis=1, keepdims=True)
            size_u = np.abs(R) @ np.abs(K).T + (P * (np.abs(R) @ np.abs(K).T)).sum(axis=1, keepdims=True)
            size_1 = size_a + np.abs(tau) + size_u * size_a
            soft = tiny * (64 + d * scale * (np.abs(Q) @ np.abs(K).T) * 2)  # relative, of p
            e1 = P * (dt + np.abs(ubar - U) * db) + eps * np.abs(g1) + soft * np.abs(g1) + 64 * tiny * P * size_1
            e2 = P * db + eps * np.abs(g2) + soft * np.abs(g2) + 64 * tiny * P * size_a
            ew = eps * np.abs(w) + soft * np.abs(w) + 64 * tiny * P * size_u
            out[0][b, h] = scale * (e1 @ np.abs(K)) + eps * np.abs(scale * (g1 @ K))
            out[1][b, h] = e2 @ np.abs(K) + eps * np.abs(g2 @ K)
            out[2][b, hk] += scale * (e1.T @ np.abs(Q)) + e2.T @ np.abs(R)
            out[3][b, hk] += ew.T @ np.abs(D)
            exact[0][b, hk] += scale * (g1.T @ Q) + g2.T @ R
            exact[1][b, hk] += w.T @ D
    out[2] += eps * np.abs(exact[0])
    out[3] += eps * np.abs(exact[1])
    return [1.02 * x for x in out]
