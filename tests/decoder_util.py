"""Inputs, calls and error bounds of dropout, block joins and gated recurrences, shared by the host and
the GPU tests.

The bounds count roundings, u = 2^-24 relative each (half a step of fp32):

* a dropped value: the factor is rounded, and the product.
* 1 / rms of a row: at most 32 additions of squares behind one another (16 in a lane, 6 across a wave,
  8 waves, the squares' own), half of it through the root; sum, division, root and quotient: R = 20.
* a join's values: each product or sum once, carried through absolute sums.
* a gate: the exponential 2, sum, quotient, product: 7.  A step multiplies what came before once (1),
  and the runs' joins add less than 3 a step, whatever their order: 12 for each step behind a term.
"""

import numpy as np

from oracle import ops
from paper_2010_14109_amd import ooc

U = 2.0 ** -24
R_ERR = 20
FIELDS = ("rows", "d", "groups", "drop", "salt")


# ---------------------------------------------------------------- joins
def join_case(seed, rows, d, groups, p=0.0, wide=False):
    g = np.random.default_rng(seed)

    def normal(*shape):
        return g.standard_normal(shape, np.float32)
    a = {"rows": rows, "d": d, "groups": groups, "drop": int(p * 2 ** 32), "salt": 5 + (1 << 35)}
    x, f = normal(rows, d), normal(rows, d)
    if wide:      # the 1e-5 counts in some rows
        f *= 10.0 ** g.uniform(-4, 3, (rows, 1)).astype(np.float32)
    v = {"x": x, "f": f, "post": 1 + 0.3 * normal(d), "gate": 0.5 * normal(groups, d),
         "pre": 1 + 0.3 * normal(d), "scale": np.array([0.9], np.float32),
         "seed": g.integers(0, 1 << 32, 2, dtype=np.uint32), "dh": normal(rows, d),
         "dn": normal(rows, d)}
    return a, v


def join_attrs(a):
    return [a[k] for k in FIELDS]


def join_oracle(a, v):
    f = {k: t.astype(np.float64) for k, t in v.items() if k != "seed"}
    return ops.join_fwd(f["x"], f["f"], f["post"], f["gate"], f["pre"], f["scale"], a, v["seed"])


def join_back_oracle(a, v, h, stream=True):
    f = {k: t.astype(np.float64) for k, t in v.items() if k != "seed"}
    return ops.join_bwd(f["f"], h.astype(np.float64), f["post"], f["gate"], f["pre"], f["scale"],
                        f["dh"] if stream else None, f["dn"], a, v["seed"])


def _abs(a, v):
    f = {k: np.abs(t.astype(np.float64)) for k, t in v.items() if k != "seed"}
    f["r"] = 1 / np.sqrt((f["f"] ** 2).mean(-1, keepdims=True) + 1e-5)
    f["m"] = ops.dropout_factor(f["f"].shape, v["seed"], a)
    f["g"] = np.repeat(f["gate"], a["rows"] // a["groups"], 0)
    return f


def join_bounds(a, v):
    """Bounds of h, n, stats."""
    f = _abs(a, v)
    H, N, st = join_oracle(a, v)
    eh = (R_ERR + 6) * U * (f["g"] * f["post"] * f["f"] * f["r"] * f["m"] + f["scale"] * f["x"])
    s = st[:, 1:]
    es = s * s * (np.abs(H) * eh).mean(-1, keepdims=True) + R_ERR * U      # relative
    return eh, f["pre"] * s * eh + np.abs(N) * (es + 3 * U), st * np.concatenate([es * 0 + R_ERR * U, es], 1)


def join_back_bounds(a, v, h, slices, stream=True):
    """Bounds of dx, df, dpost, dgate, dpre, h being the device's."""
    f = _abs(a, v)
    h = h.astype(np.float64)
    dx, df, dpost, dgate, dpre = join_back_oracle(a, v, h, stream)
    s = 1 / np.sqrt((h * h).mean(-1, keepdims=True) + 1e-5)
    vv, t, m = f["f"] * f["r"], np.abs(h) * s, f["pre"] * f["dn"]
    mt = (m * t).mean(-1, keepdims=True)
    dh = np.abs(dx / f["scale"])
    eg = (R_ERR * 2 + 40) * U * ((f["dh"] if stream else 0.0) + s * (m + t * mt))
    per = a["rows"] // a["groups"]
    chain = (-(-per // slices) + 4 + a["groups"] * slices / 16 + 18 + R_ERR + 6) * U
    w = f["post"] * vv * f["m"]

    def by_gate(z):
        return z.reshape(a["groups"], per, -1).sum(1)
    edu = f["g"] * f["m"] * (eg + 4 * U * dh)
    du = f["g"] * f["m"] * dh
    edv, dv = f["post"] * (edu + U * du), f["post"] * du
    p, ep = (dv * vv).mean(-1, keepdims=True), (vv * edv).mean(-1, keepdims=True)
    ep = ep + (R_ERR + 34) * U * p
    edf = f["r"] * (edv + vv * ep + (2 * R_ERR + 6) * U * (dv + vv * p))
    return (f["scale"] * (eg + U * dh), edf, (vv * edu + chain * du * vv).sum(0),
            by_gate(w * eg + chain * dh * w), chain * (f["dn"] * t).sum(0))


# ---------------------------------------------------------------- recurrences
def scan_case(seed, B, T, C, carry=False, fresh=False, shift=2.0):
    g = np.random.default_rng(seed)
    a = {"B": B, "T": T, "C": C, "carry": int(carry), "fresh": int(fresh)}
    fx = g.standard_normal((B * T, 2 * C), np.float32)
    fx[:, :C] = 2 * fx[:, :C] + np.float32(shift)
    h0 = g.standard_normal((B, C), np.float32) if carry else None
    fr = (g.random(B * T) < 0.02).astype(np.int32) * 7 if fresh else None
    return a, fx, h0, fr, g.standard_normal((B * T, C), np.float32)


def scan_shape(a):
    return [a["B"], a["T"], a["C"]]


def scan_attrs(a, slices):
    return scan_shape(a) + [a["carry"], a["fresh"], slices]


def _f64(x):
    return None if x is None else x.astype(np.float64)


def scan_oracle(a, fx, h0, fr):
    return ops.scan_fwd(_f64(fx), a, _f64(h0), fr)


def scan_bound(a, fx, h0, fr):
    x, gate, rest, live = ops._gates(_f64(fx), fr, a)
    m = np.zeros(x[:, 0].shape) if h0 is None else np.abs(_f64(h0))
    e, out = np.zeros_like(m), np.zeros(x.shape)
    for t in range(a["T"]):
        w, b = gate[:, t] * live[:, t], rest[:, t] * np.abs(x[:, t])
        e, m = w * (e + 12 * U * m) + 12 * U * b, w * m + b
        out[:, t] = e + 3 * U * m
    return out.reshape(-1, a["C"])


def scan_back_bounds(a, fx, h0, fr, h, dh):
    """Bounds of dfx and dh0, h being the device's."""
    x, gate, rest, live = ops._gates(_f64(fx), fr, a)
    d, hh = np.abs(_f64(dh)).reshape(x.shape), _f64(h).reshape(x.shape)
    first = np.zeros(x[:, :1].shape) if h0 is None else _f64(h0)[:, None]
    diff = np.abs(np.concatenate([first, hh[:, :-1]], 1) * live - x)
    m, e = np.zeros(x[:, 0].shape), np.zeros(x[:, 0].shape)
    eg, mg = np.zeros(x.shape), np.zeros(x.shape)
    for t in range(a["T"] - 1, -1, -1):
        mg[:, t], eg[:, t] = d[:, t] + m, e + 3 * U * (m + d[:, t])
        w = gate[:, t] * live[:, t]
        e, m = w * (e + 12 * U * (m + d[:, t])), w * (m + d[:, t])
    k = gate * rest
    both = np.stack([k * diff * (eg + 20 * U * mg), rest * (eg + 9 * U * mg)], 2)
    return both.reshape(fx.shape), e + 3 * U * m


def scan_part(a, slices):
    return [(slices * a["B"], 2 * a["C"])] if slices > 1 else []


def scan_ins(fx, h0, fr):
    return [t for t in (fx, h0, fr) if t is not None]


R, W = ooc.R, ooc.W


# ---------------------------------------------------------------- span attention
# A score's error is that of attention_util, and: under the cap 8 u of itself and 4 u of the cap (its
# tangent is off by 2^-21 of itself, the cap's quotient and product round); the bias rounds the distance's
# product and the sum, 2 u of each.  The cap's factor 1 - tanh^2 is off by 8 u, and by the score's error
# over the cap, as its slope is less than 1.
def spans(kind, g, B, Tq, Tk):
    i = np.broadcast_to(np.arange(Tq), (B, Tq)) + (Tk - Tq)
    lo, hi, at = np.zeros((B, Tq), int), i + 1, i
    if kind == "window":
        lo = hi - max(1, Tk // 5)
    elif kind == "docs":
        cuts = np.sort(g.integers(0, Tk, (B, 3)), 1)
        lo = np.where(i[:, :, None] >= cuts[:, None], cuts[:, None], 0).max(-1)
        hi = np.where(i < Tk - Tk // 7, hi, lo)
    elif kind == "prefix":
        hi = np.maximum(hi, g.integers(0, Tk + 1, (B, 1)))
    elif kind == "any":            # spans of any order and length, a quarter of them empty
        lo = g.integers(0, Tk + 1, (B, Tq))
        hi = np.where(g.random((B, Tq)) < 0.25, lo - g.integers(0, 3, (B, Tq)),
                      g.integers(0, Tk + 1, (B, Tq)))
        at = g.integers(-5, Tk + 5, (B, Tq))
    elif kind == "all":
        lo, hi = np.zeros((B, Tq), int), np.full((B, Tq), Tk)
    elif kind == "none":
        hi = lo
    return np.stack([np.maximum(lo, 0), hi, at], -1).reshape(B * Tq, 3).astype(np.int32)


def span_case(seed, B, Tq, Tk, H, Hkv, dh, kind, cap=0.0, bias=False, spread=1.0):
    g = np.random.default_rng(seed)
    a = {"B": B, "Tq": Tq, "Tk": Tk, "H": H, "Hkv": Hkv, "dh": dh, "cap": int(cap > 0), "bias": int(bias)}
    q = (spread * g.standard_normal((B * Tq, H * dh))).astype(np.float32)
    kv, dy = (g.standard_normal(s, np.float32) for s in ((B * Tk, 2 * Hkv * dh), q.shape))
    mod = ([cap] if cap else []) + (list(2.0 ** -g.uniform(0, 8, H)) if bias else [])
    return a, q, kv, spans(kind, g, B, Tq, Tk), np.array(mod, np.float32), dy


def span_attrs(a):
    return [a[k] for k in ("B", "Tq", "Tk", "H", "Hkv", "dh", "cap", "bias")]


def span_bounds(q, kv, span, mod, dy, a):
    """Bounds of y, lse, dq, dkv."""
    f = np.float64
    Q, K, V, G = ops._cross_parts(q.astype(f), kv.astype(f), a)
    D = dy.astype(f).reshape(a["B"], a["Tq"], a["H"], a["dh"]).transpose(0, 2, 1, 3)
    ey, el = np.zeros_like(Q), np.zeros(Q.shape[:3])
    eq, ek, ev = np.zeros_like(Q), np.zeros_like(K), np.zeros_like(V)
    scale, es = 1 / np.sqrt(a["dh"]), (a["dh"] / 2 + 16) * U
    sp = span.reshape(a["B"], a["Tq"], 3)
    cap = float(mod[0]) if a["cap"] else np.inf
    sums = (6 * a["Tk"] / 16 + 32) * U
    rows = (6 * a["Tq"] * G / 16 + 32) * U
    for b in range(a["B"]):
        for h in range(a["H"]):
            j = h // G
            k, v, qq, d = K[b, j], V[b, j], Q[b, h], D[b, h]
            S, turn = ops._span_scores(qq, k, sp[b], h, a, mod)
            seen = S > -np.inf
            P, lse = ops._span_probs(S)
            mag = np.where(seen, np.abs(S), 0.0)
            raw = es * scale * np.abs(qq) @ np.abs(k).T
            e_turn = raw / cap + 8 * U if a["cap"] else 0.0
            if a["bias"]:
                far = np.abs(np.arange(a["Tk"]) - sp[b][:, 2:]) * float(mod[a["cap"] + h])
            else:
                far = 0.0
            eS = raw + ((8 * U * (mag + far) + 4 * U * cap) if a["cap"] else 0.0) + 2 * U * (far + mag)
            eS = np.where(seen, eS, 0.0)
            some = np.where(seen.any(1), lse, 0.0)
            reach = np.where(seen, np.abs(np.where(seen, S, 0.0) - some[:, None]), 0.0) + 8
            eP = eS + eS.max(-1, keepdims=True) + 2 * U * reach + sums     # relative
            eP = eP + 4 * U * (np.abs(some) + mag.max(-1))[:, None]
            el[b, h] = eS.max(-1) + sums + 4 * U * (np.abs(some) + mag.max(-1))
            ey[b, h] = (P * (eP + sums)) @ np.abs(v)
            dP = d @ v.T
            y = P @ v
            delta = (d * y).sum(-1, keepdims=True)
            e_dP = es * np.abs(d) @ np.abs(v).T
            e_delta = (np.abs(d) * (ey[b, h] + (a["dh"] / 16 + 16) * U * np.abs(y))).sum(-1, keepdims=True)
            dS = P * np.abs(dP - delta) * scale
            e_dS = dS * turn * (eP + 4 * U) + P * scale * turn * (e_dP + e_delta) + dS * e_turn
            dS = dS * turn
            eq[b, h] = (e_dS + sums * dS) @ np.abs(k)
            ek[b, j] += (e_dS + rows * dS).T @ np.abs(qq)
            ev[b, j] += (P * (eP + rows)).T @ np.abs(d)
    return (ey.transpose(0, 2, 1, 3).reshape(q.shape), el, eq.transpose(0, 2, 1, 3).reshape(q.shape),
            np.stack([ek, ev]).transpose(1, 3, 0, 2, 4).reshape(kv.shape))
