"""Inputs, calls and error bounds of the rotation, the per-head norms and the cross attention,
shared by the host and the GPU tests.

The bounds follow the operations' roundings, u = 2^-24 relative each (half a step of fp32):

* a rotated value c x0 - s x1: c and s are each off by at most 4 u of the magnitude m (the reduced
  angle's rounding and the series' last sums, then the product with m), each product and the sum
  round once more: 8 u m (|x0| + |x1|).
* a root mean square over dh values: at most dh / 16 + 10 additions behind one another and one
  rounding per square, half of it through the root, then root, quotient and two products.
* a score: its products are exact in three pieces each, and every matrix instruction (6 per 16
  columns, a few columns' padding) or addition rounds once: (dh / 2 + 16) u sum |q| |k|.
* a probability exp(S - lse): twice the scores' error, 2 u per unit of the exponent, and 8 more;
  sums over n states: 6 n / 16 instructions and 32 u for the joins.
* a gradient's error is that of its factors, carried through absolute sums.
"""

import numpy as np

from oracle import ops
from paper_2010_14109_amd import netdef, ooc

U = 2.0 ** -24
R, W = ooc.R, ooc.W



def positions(g, rows, far):
    if far:
        return g.integers(-(1 << 20), 1 << 31, rows, dtype=np.int64).astype(np.int32)
    return (np.arange(rows) % 7).astype(np.int32)


def table(rot, stretched):
    return np.array(netdef.rotary_table(rot, scale=16.0, trained=4096) if stretched
                    else netdef.rotary_table(rot))


# ---------------------------------------------------------------- rotation
def rope_case(seed, rows, heads, dh, rot, layout, rest, far):
    g = np.random.default_rng(seed)
    a = {"heads": heads, "dh": dh, "rot": rot, "layout": layout}
    x = g.standard_normal((rows, heads * dh + rest), np.float32)
    return a, x, positions(g, rows, far), table(rot, far)


def rope_attrs(x, a):
    return list(x.shape) + [a["heads"], a["dh"], a["rot"], a["layout"]]


def pair_sums(h, a):
    """|x0| + |x1| at both places of each pair of h [rows, heads, dh]; |x| elsewhere."""
    out = np.abs(h)
    if a["rot"]:
        i0, i1 = ops._pairs(a["rot"], a["layout"])
        both = out[..., i0] + out[..., i1]
        out = out.copy()
        out[..., i0] = out[..., i1] = both
    return out


def rope_bound(x, a, m):
    n = a["heads"] * a["dh"]
    out = np.zeros(x.shape)
    h = x[:, :n].astype(np.float64).reshape(len(x), a["heads"], a["dh"])
    b = 8 * U * m * pair_sums(h, a)
    b[..., a["rot"]:] = 0          # copied
    out[:, :n] = b.reshape(len(x), n)
    return out


# ---------------------------------------------------------------- per-head norm
def qknorm_case(seed, rows, h1, h2, dh, rot, layout, rest, far):
    g = np.random.default_rng(seed)
    a = {"h1": h1, "h2": h2, "dh": dh, "rot": rot, "layout": layout}
    x = g.standard_normal((rows, (h1 + h2) * dh + rest), np.float32)
    x *= 10.0 ** g.uniform(-3, 3, (rows, 1)).astype(np.float32)     # the eps counts in some rows
    gain = (1 + 0.3 * g.standard_normal((2 if h2 else 1, dh))).astype(np.float32)
    dy = g.standard_normal(x.shape, np.float32)
    where = [positions(g, rows, far), table(rot, far)] if rot else []
    return a, x, gain, where, dy


def qknorm_attrs(x, a):
    return list(x.shape) + [a["h1"], a["h2"], a["dh"], a["rot"], a["layout"]]


def _norm_parts(x, gain, a):
    heads = a["h1"] + a["h2"]
    h = x[:, :heads * a["dh"]].astype(np.float64).reshape(len(x), heads, a["dh"])
    r = 1 / np.sqrt((h * h).mean(-1, keepdims=True) + 1e-5)
    return h, r, ops._head_gain(gain.astype(np.float64), a)


def qknorm_bound(x, gain, where, a):
    h, r, g = _norm_parts(x, gain, a)
    m = where[1][-1] if where else 1.0
    c = (a["dh"] / 16 + 10) / 2 + 4 + 8
    out = np.zeros(x.shape)
    out[:, :h[0].size] = (c * U * m * pair_sums(g * h * r, a)).reshape(len(x), -1)
    return out


def qknorm_back_bound(x, gain, where, dy, a, slices):
    """Bounds of dx and dgain."""
    h, r, g = _norm_parts(x, gain, a)
    heads = a["h1"] + a["h2"]
    m = where[1][-1] if where else 1.0
    z = m * pair_sums(dy[:, :h[0].size].astype(np.float64).reshape(h.shape), a)
    u = np.abs(h) * r
    c = 32 + a["dh"] / 4
    dx = np.zeros(x.shape)
    w = np.abs(g) * z
    dx[:, :h[0].size] = (c * U * r * (w + u * (w * u).mean(-1, keepdims=True))).reshape(len(x), -1)
    # a lane's additions: the rows of a slice times the heads; the waves of a slice; the slices
    chain = c + -(-len(x) // slices) * heads + 16 + slices
    per = (z * u).sum(0)
    parts = [per[:a["h1"]].sum(0)] + ([per[a["h1"]:].sum(0)] if a["h2"] else [])
    return dx, chain * U * np.stack(parts)


# ---------------------------------------------------------------- cross attention
def cross_case(seed, B, Tq, Tk, H, Hkv, dh, klen=None, spread=1.0):
    g = np.random.default_rng(seed)
    a = {"B": B, "Tq": Tq, "Tk": Tk, "H": H, "Hkv": Hkv, "dh": dh}
    q = (spread * g.standard_normal((B * Tq, H * dh))).astype(np.float32)
    kv = g.standard_normal((B * Tk, 2 * Hkv * dh), np.float32)
    dy = g.standard_normal((B * Tq, H * dh), np.float32)
    if klen is None:
        klen = g.integers(0, Tk + 1, B)
    klen = np.broadcast_to(np.asarray(klen, np.int32), (B,)).copy()
    return a, q, kv, klen, dy


def cross_shape(a):
    return [a[k] for k in ("B", "Tq", "Tk", "H", "Hkv", "dh")]


def cross_bounds(q, kv, klen, dy, a):
    """Bounds of y, lse, dq, dkv."""
    f = np.float64
    Q, K, V, G = ops._cross_parts(q.astype(f), kv.astype(f), a)
    D = dy.astype(f).reshape(a["B"], a["Tq"], a["H"], a["dh"]).transpose(0, 2, 1, 3)
    ey, else_ = np.zeros_like(Q), np.zeros(Q.shape[:3])
    eq, ek, ev = np.zeros_like(Q), np.zeros_like(K), np.zeros_like(V)
    scale, es = 1 / np.sqrt(a["dh"]), (a["dh"] / 2 + 16) * U
    for b in range(a["B"]):
        n = int(klen[b])
        for h in range(a["H"] if n else 0):
            j = h // G
            k, v, qq, d = K[b, j, :n], V[b, j, :n], Q[b, h], D[b, h]
            P, lse = ops._cross_probs(qq, K[b, j], n)
            S = qq @ k.T * scale
            dS_err = es * scale * np.abs(qq) @ np.abs(k).T
            sums = (6 * n / 16 + 32) * U
            reach = np.abs(S - lse[:, None]) + 8
            eP = dS_err + dS_err.max(-1, keepdims=True) + 2 * U * reach + sums     # relative
            else_[b, h] = dS_err.max(-1) + sums + 4 * U * (np.abs(lse) + np.abs(S).max(-1))
            ey[b, h] = (P * (eP + sums)) @ np.abs(v)
            dP = d @ v.T
            y = P @ v
            delta = (d * y).sum(-1, keepdims=True)
            e_dP = es * np.abs(d) @ np.abs(v).T
            e_delta = (np.abs(d) * (ey[b, h] + (a["dh"] / 16 + 16) * U * np.abs(y))).sum(-1, keepdims=True)
            e_dS = P * scale * ((np.abs(dP - delta)) * (eP + 4 * U) + e_dP + e_delta)
            dS = P * np.abs(dP - delta) * scale
            rows = (6 * a["Tq"] * G / 16 + 32) * U
            eq[b, h] = (e_dS + sums * dS) @ np.abs(k)
            ek[b, j, :n] += (e_dS + rows * dS).T @ np.abs(qq)
            ev[b, j, :n] += (P * (eP + rows)).T @ np.abs(d)
    def back(t):
        return t.transpose(0, 2, 1, 3).reshape(q.shape)
    return back(ey), else_, back(eq), np.stack([ek, ev]).transpose(1, 3, 0, 2, 4).reshape(kv.shape)


def within(name, got, ref, bound):
    """Every value within its bound; equal where the reference is not finite."""
    got, ref = np.asarray(got, np.float64).reshape(ref.shape), np.asarray(ref, np.float64)
    finite = np.isfinite(ref)
    assert np.array_equal(got[~finite], ref[~finite], equal_nan=True), name
    assert np.isfinite(got[finite]).all(), name
    err = np.abs(got[finite] - ref[finite])
    b = np.broadcast_to(bound, ref.shape)[finite] + 1e-37     # the smallest values are not kept
    worst = int(np.argmax(err - b)) if err.size else 0
    assert not err.size or (err <= b).all(), (name, float(err[worst]), float(b[worst]))
    return float((err / b).max(initial=0.0))
