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
