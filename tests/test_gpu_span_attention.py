"""Span attention on the device against the 64-bit oracle.  Error bounds: decoder_util."""

import numpy as np
import pytest

import attention_util as au
import decoder_util as du
import hip_util as hu
from oracle import ops
from paper_2010_14109_amd import ooc
from test_gpu_attention_ops import cross_bwd, cross_fwd, outputs

pytestmark = pytest.mark.gpu
R, W = ooc.R, ooc.W


def span_fwd(a, q, kv, span, mod, slices=None, stream=None):
    if slices is None:
        slices = ooc.attention_slices("span_attention_fwd", au.cross_shape(a))[0][0]
    lse = (a["B"], a["H"], a["Tq"])
    part = [(slices, q.size + int(np.prod(lse)))] if slices > 1 else []
    return outputs("span_attention_fwd", [q, kv, span] + ([mod] if mod.size else []),
                   [q.shape, lse] + part, du.span_attrs(a) + [slices], stream)[:2]


def span_bwd(a, q, kv, span, mod, y, lse, dy, slices=None, stream=None):
    if slices is None:
        slices = ooc.attention_slices("span_attention_bwd", au.cross_shape(a))[0]
    sq, sk = slices
    n = max(sq * q.size if sq > 1 else 0, sk * kv.size if sk > 1 else 0)
    return outputs("span_attention_bwd", [q, kv, span] + ([mod] if mod.size else []) + [y, lse, dy],
                   [q.shape, kv.shape, lse.shape, (a["B"], -(-a["Tq"] // 32), 2)] + ([(n,)] if n else []),
                   du.span_attrs(a) + list(slices), stream)[:3]


def check_span(a, q, kv, span, mod, dy, slices=(None, None)):
    f = np.float64
    y, lse = span_fwd(a, q, kv, span, mod, slices[0])
    wy, wl = ops.span_attention_fwd(q.astype(f), kv.astype(f), span, a, mod)
    by, bl, bq, bk = du.span_bounds(q, kv, span, mod, dy, a)
    au.within("y", y, wy, by)
    au.within("lse", lse, wl, bl)
    dq, dkv, delta = span_bwd(a, q, kv, span, mod, y, lse, dy, slices[1])
    wq, wk, _ = ops.span_attention_bwd(q.astype(f), kv.astype(f), span, dy.astype(f), a, mod)
    au.within("dq", dq, wq, bq)
    au.within("dkv", dkv, wk, bk)
    d = (dy.astype(f) * y).reshape(a["B"], a["Tq"], a["H"], -1)
    au.within("delta", delta, d.sum(-1).transpose(0, 2, 1),
              (a["dh"] / 16 + 16) * au.U * np.abs(d).sum(-1).transpose(0, 2, 1))
    return y, lse, dq, dkv


SPAN = [
    # B Tq Tk H Hkv dh kind cap bias
    (1, 1, 1, 1, 1, 1, "causal", 0, False), (2, 1, 1, 2, 1, 4, "none", 5, True), (2, 5, 5, 4, 2, 16, "causal", 0, True),
    (2, 33, 33, 2, 2, 64, "causal", 0, False), (1, 128, 128, 2, 1, 64, "docs", 0, False),
    (2, 129, 129, 4, 4, 32, "any", 3, True), (1, 257, 257, 2, 2, 64, "window", 5, False),
    (2, 300, 300, 4, 1, 128, "causal", 0, False), (1, 190, 190, 3, 3, 85, "prefix", 0, True),
    (2, 3, 130, 6, 2, 40, "causal", 2, True), (1, 70, 70, 1, 1, 256, "any", 0, True), (1, 150, 150, 2, 1, 200, "docs", 4, True),
    (2, 90, 90, 2, 2, 96, "any", 3, False), (1, 1, 3000, 8, 2, 64, "window", 5, True), (4, 1, 513, 4, 4, 128, "any", 3, True),
    (1, 600, 600, 2, 1, 80, "window", 0, True), (1, 1000, 1000, 1, 1, 64, "docs", 0, True),
    (3, 97, 97, 5, 5, 17, "all", 0, False), (2, 333, 333, 2, 2, 48, "prefix", 9, False), (1, 31, 2049, 2, 2, 33, "any", 0, True),
    (2, 8, 8, 16, 2, 8, "any", 1, True), (1, 260, 260, 4, 2, 129, "causal", 0, True), (2, 64, 64, 2, 2, 160, "prefix", 5, True),
    (6, 2, 40, 3, 1, 72, "any", 0, False), (1, 700, 700, 16, 2, 64, "any", 0, False), (2, 150, 150, 3, 3, 192, "window", 0, False),
    (16, 512, 512, 32, 32, 32, "docs", 0, False), (1, 40, 90, 4, 1, 128, "any", 3, True), (1, 4, 700, 4, 1, 96, "any", 3, True),
    (3, 7, 7, 12, 4, 64, "none", 0, False), (1, 2100, 2100, 1, 1, 32, "window", 0, False),
]


@pytest.mark.parametrize("case", SPAN, ids=str)
def test_span_attention(case):
    big = case[0] * case[3] > 100
    a, q, kv, span, mod, dy = du.span_case(71, *case)
    if not big:
        check_span(a, q, kv, span, mod, dy)
        return
    # many heads: the wide kernels; a few heads of it against the oracle
    y, lse = span_fwd(a, q, kv, span, mod)
    dq, dkv, _ = span_bwd(a, q, kv, span, mod, y, lse, dy)
    B, T, H, dh = a["B"], a["Tq"], a["H"], a["dh"]
    one = dict(a, B=1, H=1, Hkv=1)
    f = np.float64
    for b, h in ((0, 0), (7, 31), (15, 13)):
        rows, c = slice(b * T, (b + 1) * T), slice(h * dh, (h + 1) * dh)
        cv = slice((H + h) * dh, (H + h + 1) * dh)
        q1, d1 = q[rows, c], dy[rows, c]
        kv1 = np.concatenate([kv[rows, c], kv[rows, cv]], 1)
        s1 = span[rows]
        wy, wl = ops.span_attention_fwd(q1.astype(f), kv1.astype(f), s1, one, mod)
        wq, wk, _ = ops.span_attention_bwd(q1.astype(f), kv1.astype(f), s1, d1.astype(f), one, mod)
        by, bl, bq, bk = du.span_bounds(q1, kv1, s1, mod, d1, one)
        au.within("y", y[rows, c], wy, by)
        au.within("lse", lse[b:b + 1, h:h + 1], wl, bl)
        au.within("dq", dq[rows, c], wq, bq)
        au.within("dkv", np.concatenate([dkv[rows, c], dkv[rows, cv]], 1), wk, bk)


@pytest.mark.parametrize("slices", [(2, (3, 1)), (5, (1, 4)), (64, (64, 64))], ids=str)
def test_span_attention_slices(slices):
    for dh, cap in ((64, 0), (96, 4.0)):
        check_span(*du.span_case(72, 2, 70, 140, 4, 2, dh, "any", cap, True), slices=slices)


@pytest.mark.parametrize("spread,cap", [(0.0, 3.0), (8.0, 20.0), (60.0, 1.0), (60.0, 0.0)])
def test_span_attention_flat_and_peaked_rows(spread, cap):
    """All scores equal, far apart, and far above the cap."""
    check_span(*du.span_case(73, 2, 150, 150, 2, 1, 64, "causal", cap, False, spread=spread))


@pytest.mark.parametrize("dh", [32, 64, 96, 200])
def test_the_first_states_are_a_span(dh):
    """Spans of the first klen states give what cross attention gives."""
    a, q, kv, klen, dy = au.cross_case(74, 3, 140, 200, 4, 2, dh, [200, 77, 0])
    s = np.stack([np.zeros(420, int), np.repeat(klen, 140), np.zeros(420, int)], 1).astype(np.int32)
    a = dict(a, cap=0, bias=0)
    none = np.zeros(0, np.float32)
    by, bl, bq, bk = au.cross_bounds(q, kv, klen, dy, a)
    y, lse = span_fwd(a, q, kv, s, none)
    cy, cl = cross_fwd(a, q, kv, klen)
    au.within("y", y, cy, 2 * by)
    au.within("lse", lse, cl, 2 * bl)
    dq, dkv, _ = span_bwd(a, q, kv, s, none, y, lse, dy)
    cq, ck, _ = cross_bwd(a, q, kv, klen, cy, cl, dy)
    au.within("dq", dq, cq, 2 * bq)
    au.within("dkv", dkv, ck, 2 * bk)


@pytest.mark.parametrize("Tq,dh", [(90, 64), (90, 32), (90, 128), (90, 256), (3, 64), (3, 128)])
def test_what_is_not_finite_stays_with_those_who_see_it(Tq, dh):
    """Documents share tiles: states, queries and gradients with NaN or infinities make NaN what they
    reach and nothing else."""
    g = np.random.default_rng(75)
    a, q, kv, span, mod, dy = du.span_case(75, 2, Tq, 90, 2, 1, dh, "any", 4.0, True)
    f, odd = np.float64, np.array([np.nan, np.inf, -np.inf], np.float32)
    bad = kv.copy()
    rows = np.r_[5, 40, 41, 90 + 77]
    for k, r in enumerate(rows):
        bad[r, g.integers(0, 2 * dh)] = odd[k % 3]
    zero = np.where(np.isfinite(bad), bad, 0).astype(np.float32)
    j = np.concatenate([np.repeat(np.arange(2), Tq)[:, None] * 90 + np.arange(90)] , 0)
    seen = (np.arange(90) >= span[:, :1]) & (np.arange(90) < span[:, 1:2])
    hit = (seen & np.isin(j, rows)).any(1)
    assert hit.any() and not hit.all()
    y, lse = span_fwd(a, q, bad, span, mod)
    wy, wl = ops.span_attention_fwd(q.astype(f), zero.astype(f), span, a, mod)
    by, bl, bq, bk = du.span_bounds(q, zero, span, mod, dy, a)
    hl = hit.reshape(2, 1, Tq).repeat(2, 1)
    assert np.isnan(y[hit]).all() and np.isnan(lse[hl]).all()
    au.within("y", y[~hit], wy[~hit], by[~hit])
    au.within("lse", lse[~hl], wl[~hl], bl[~hl])
    # gradients with the rows that hit taken out of the loss (their dY is 0 and lse NaN)
    dq, dkv, _ = span_bwd(a, q, bad, span, mod, y, lse, dy)
    assert np.isnan(dq[hit]).all()
    wq, wk, _ = ops.span_attention_bwd(q.astype(f), zero.astype(f), span, dy.astype(f), a, mod)
    au.within("dq", dq[~hit], wq[~hit], bq[~hit])
    reached = np.zeros((2, 90), bool)
    np.logical_or.at(reached, np.repeat(np.arange(2), Tq)[hit], seen[hit])
    reached = reached.reshape(-1)
    assert np.isnan(dkv[reached]).any(1).all()
    au.within("dkv", dkv[~reached], wk[~reached], bk[~reached])
    # a query's own
    y, lse = span_fwd(a, q, kv, span, mod)
    bad_q, bad_d = q.copy(), dy.copy()
    r1, r2 = np.flatnonzero(seen.any(1))[[0, -1]]
    bad_q[r1, 0], bad_d[r2, -1] = np.nan, np.inf
    empty = np.flatnonzero(~seen.any(1))
    if empty.size:
        bad_d[empty[0]] = np.nan
    y2, l2 = span_fwd(a, bad_q, kv, span, mod)
    assert np.isnan(y2[r1, :dh]).all()
    ok = np.arange(len(q)) != r1
    assert np.isfinite(y2[ok]).all()
    dq, dkv, _ = span_bwd(a, bad_q, kv, span, mod, y2, l2, bad_d)
    touched = np.zeros((2, 90), bool)
    for r in (r1, r2):
        touched[r // Tq] |= seen[r]
    touched = touched.reshape(-1)
    assert np.isnan(dkv[touched]).any(1).all() and np.isfinite(dkv[~touched]).all()
    keep = ~np.isin(np.arange(len(q)), [r1, r2])
    assert np.isfinite(dq[keep]).all() and (not empty.size or not dq[empty].any())


def test_spans_outside_the_states():
    """Such queries get NaN and nothing else changes; empty spans may lie anywhere."""
    for Tq, dh in ((70, 64), (70, 96), (2, 64)):
        a, q, kv, span, mod, dy = du.span_case(76, 2, Tq, 70, 2, 2, dh, "all", 0, True)
        span[0], span[Tq] = (-1, 5, 0), (69, 71, 0)
        span[1], span[Tq + 1] = (1 << 30, -(1 << 30), 0), (500, 500, 0)
        clean = span.copy()
        clean[[0, Tq]] = 0
        y, lse = span_fwd(a, q, kv, span, mod)
        cy, cl = span_fwd(a, q, kv, clean, mod)
        out = np.zeros(2 * Tq, bool)
        out[[0, Tq]] = True
        assert np.isnan(y[out]).all() and np.array_equal(y[~out], cy[~out])
        assert not y[1].any() and np.isneginf(lse[0, :, 1]).all() and np.isnan(lse[:, :, 0]).all()
        dq, dkv, _ = span_bwd(a, q, kv, span, mod, y, lse, dy)
        _, ck, _ = span_bwd(a, q, kv, clean, mod, cy, cl, dy)
        assert np.isnan(dq[out]).all() and np.array_equal(dkv, ck)


def test_span_attention_repeats_and_replays():
    """The same bits each time, and from a graph whose spans change between its replays."""
    a, q, kv, span, mod, dy = du.span_case(77, 2, 300, 300, 4, 2, 64, "docs", 5.0, True)
    first = check_span(a, q, kv, span, mod, dy)
    y, lse = span_fwd(a, q, kv, span, mod)
    again = [y, lse] + span_bwd(a, q, kv, span, mod, y, lse, dy)[:2]
    assert all(np.array_equal(x, z) for x, z in zip(first, again))
    s = hu.Stream()
    (sf,), pf = ooc.attention_slices("span_attention_fwd", au.cross_shape(a))
    sb, pb = ooc.attention_slices("span_attention_bwd", au.cross_shape(a))
    ins = [hu.Array(t) for t in (q, kv, span, mod)]
    d = hu.Array(dy)
    out = [hu.empty(q.shape), hu.empty(lse.shape)]
    back = [hu.empty(q.shape), hu.empty(kv.shape), hu.empty(lse.shape), hu.empty((2, 10, 2))]
    parts = [[hu.empty((n // 4,))] if n else [] for n in (pf, pb)]

    def calls():
        hu.call("span_attention_fwd", ins + out + parts[0], [R] * 4 + [W] * (2 + len(parts[0])),
                du.span_attrs(a) + [sf], s)
        hu.call("span_attention_bwd", ins + out + [d] + back + parts[1],
                [R] * 7 + [W] * (4 + len(parts[1])), du.span_attrs(a) + sb, s)
    replay = s.record(calls)
    g = np.random.default_rng(78)
    for kind in ("any", "causal", "docs"):
        new = du.spans(kind, g, 2, 300, 300)
        hu.check(hu.hip().hipMemcpy(hu.ctypes.c_void_p(ins[2].ptr), new.ctypes.data_as(hu.ctypes.c_void_p),
                                    hu.ctypes.c_size_t(new.nbytes), 1), "hipMemcpy")
        replay()
        hu.synchronize()
        y, lse = span_fwd(a, q, kv, new, mod)
        dq, dkv, _ = span_bwd(a, q, kv, new, mod, y, lse, dy)
        for got, want in zip(out + back[:2], (y, lse, dq, dkv)):
            assert np.array_equal(got.get(), want)
