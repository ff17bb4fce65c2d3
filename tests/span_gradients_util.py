"""Capped span attention whose scores lie on one side, and bounds that follow the cap's factor.

Relative to itself, u = 2^-24: with x the score over the cap, the factor 1 - tanh^2 x changes by 2 |dx|, as its
logarithm's slope is at most 2.  dx is the score's error over the cap and 4 u |x| (the product with the
scale, the cap in powers of two, its inverse and the product with that).  exp(2 |x|) takes its argument's two
roundings, 4 u |x|, and one unit in its last place, 2 u; the sum 1 u, the reciprocal 2 u, the last product 1 u:
4 |x| u + 6 u.  A capped score is off by its own error times the factor (twice that, for the factor's
change), by 8 u of itself, 4 u of the cap and 2 u of itself where it is used."""

import numpy as np

from oracle import ops

U = 2.0 ** -24


def one_sided_case(seed, dh, low, high, Tq=150, Tk=170, H=2, Hkv=1, cap=1.5):
    """Each query's scores within some percent of one value between low and high times the cap.  Most see
    a few states only: over many, gradients of the same factor cancel each other."""
    g = np.random.default_rng(seed)
    a = {"B": 1, "Tq": Tq, "Tk": Tk, "H": H, "Hkv": Hkv, "dh": dh, "cap": 1, "bias": 0}
    level = g.uniform(low, high, (Tq, H, 1)) * cap / np.sqrt(dh)
    q = (level * (1 + 0.1 * g.standard_normal((Tq, H, dh)))).reshape(Tq, -1).astype(np.float32)
    kv = g.standard_normal((Tk, 2, Hkv, dh))
    kv[:, 0] = 1 + 0.5 * kv[:, 0]
    dy = g.standard_normal(q.shape, np.float32)
    span = np.tile(np.array([0, Tk, 0], np.int32), (Tq, 1))
    few = np.arange(Tq) % 8 != 0
    span[few, 0] = g.integers(0, Tk - 7, few.sum())
    span[few, 1] = span[few, 0] + g.integers(2, 8, few.sum())
    return a, q, kv.reshape(Tk, -1).astype(np.float32), span, np.array([cap], np.float32), dy


def one_sided_bounds(q, kv, span, mod, dy, a):
    """Bounds of dq and dkv."""
    f = np.float64
    Q, K, V, G = ops._cross_parts(q.astype(f), kv.astype(f), a)
    D = dy.astype(f).reshape(a["B"], a["Tq"], a["H"], a["dh"]).transpose(0, 2, 1, 3)
    eq, ek, ev = np.zeros_like(Q), np.zeros_like(K), np.zeros_like(V)
    scale, es, cap = 1 / np.sqrt(a["dh"]), (a["dh"] / 2 + 16) * U, float(mod[0])
    sums, rows = (6 * a["Tk"] / 16 + 32) * U, (6 * a["Tq"] * G / 16 + 32) * U
    sp = span.reshape(a["B"], a["Tq"], 3)
    for b in range(a["B"]):
        for h in range(a["H"]):
            j = h // G
            k, v, qq, d = K[b, j], V[b, j], Q[b, h], D[b, h]
            S, turn = ops._span_scores(qq, k, sp[b], h, a, mod)
            seen = S > -np.inf
            P, lse = ops._span_probs(S)
            mag = np.where(seen, np.abs(S), 0.0)
            raw, x = es * scale * np.abs(qq) @ np.abs(k).T, np.abs(qq @ k.T) * scale / cap
            e_turn = 2 * (raw / cap + 4 * U * x) + 4 * U * x + 6 * U           # relative
            eS = np.where(seen, 2 * (raw + 4 * U * x * cap) * turn + 10 * U * mag + 4 * U * cap, 0.0)
            some = np.where(seen.any(1), lse, 0.0)[:, None]
            reach = np.where(seen, np.abs(np.where(seen, S, 0.0) - some), 0.0) + 8
            eP = eS + eS.max(-1, keepdims=True) + 2 * U * reach + sums
            eP = eP + 4 * U * (np.abs(some) + mag.max(-1, keepdims=True))
            y, dP = P @ v, d @ v.T
            ey = (P * (eP + sums)) @ np.abs(v)
            delta = (d * y).sum(-1, keepdims=True)
            e_dP = es * np.abs(d) @ np.abs(v).T
            e_delta = (np.abs(d) * (ey + (a["dh"] / 16 + 16) * U * np.abs(y))).sum(-1, keepdims=True)
            dS = P * np.abs(dP - delta) * scale * turn
            e_dS = dS * (eP + e_turn + 4 * U) + P * scale * turn * (e_dP + e_delta)
            eq[b, h] = (e_dS + sums * dS) @ np.abs(k)
            ek[b, j] += (e_dS + rows * dS).T @ np.abs(qq)
            ev[b, j] += (P * (eP + rows)).T @ np.abs(d)
    return (eq.transpose(0, 2, 1, 3).reshape(q.shape),
            np.stack([ek, ev]).transpose(1, 3, 0, 2, 4).reshape(kv.shape))
