"""Dropout, block joins and gated recurrences on the device against the 64-bit oracle.  Error bounds:
decoder_util."""

import threading

import numpy as np
import pytest

import attention_util as au
import decoder_util as du
import hip_util as hu
from oracle import ops
from paper_2010_14109_amd import ooc
from test_gpu_attention_ops import outputs

pytestmark = pytest.mark.gpu
R, W = ooc.R, ooc.W


# ---------------------------------------------------------------- dropout
@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 1023, 4096, 78851, 4 * 16384 * 256 + 5 * 1024 + 3])
@pytest.mark.parametrize("p", [0.1, 0.5])
def test_dropout(n, p):
    g = np.random.default_rng(n)
    a = {"drop": int(p * 2 ** 32), "salt": 3 + (5 << 32)}
    x, seed = g.standard_normal(n, np.float32), g.integers(0, 1 << 32, 2, dtype=np.uint32)
    attrs = [n, a["drop"], a["salt"]]
    (y,) = outputs("dropout", [x, seed], [(n,)], attrs)
    want = ops.dropout(x.astype(np.float64), seed, a)
    assert np.array_equal(y == 0, want == 0)
    au.within("y", y, want, 2 * du.U * np.abs(want))
    if n < 5000:
        (dx,) = outputs("dropout", [np.ones(n, np.float32), seed], [(n,)], attrs)
        assert np.array_equal(dx > 0, want != 0)
        (other,) = outputs("dropout", [x, seed], [(n,)], attrs[:2] + [a["salt"] + 1])
        if n > 1000:
            assert not np.array_equal(other, y)


def test_dropout_edges():
    """Nothing dropped: the bits; all but 1 in 2^32 dropped; NaN and infinities dropped are 0."""
    x = np.array([np.nan, np.inf, -np.inf, 1e-42, -0.0, 1.5] * 50, np.float32)
    seed = np.array([1, 2], np.uint32)
    (y,) = outputs("dropout", [x, seed], [x.shape], [x.size, 0, 9])
    assert y.tobytes() == x.tobytes()
    (y,) = outputs("dropout", [x, seed], [x.shape], [x.size, (1 << 32) - 1, 9])
    assert not y.any()
    (y,) = outputs("dropout", [x, seed], [x.shape], [x.size, 1 << 31, 9])
    keep = ops.dropout_factor(x.shape, seed, {"drop": 1 << 31, "salt": 9}) > 0
    assert not y[~keep].any() and y[keep].tobytes() == (2 * x[keep]).tobytes()


# ---------------------------------------------------------------- joins
JOIN = [
    # rows d groups p wide
    (1, 1, 1, 0.0, False), (3, 5, 3, 0.5, False), (8, 1024, 1, 0.0, False), (6, 255, 2, 0.1, True),
    (70, 256, 7, 0.1, False), (33, 257, 1, 0.1, True), (36, 512, 4, 0.0, True), (20, 1023, 2, 0.3, False),
    (259, 1024, 1, 0.1, False), (24, 1025, 24, 0.1, False), (15, 2048, 3, 0.1, True), (10, 2050, 1, 0.0, False),
    (9, 4095, 3, 0.2, False), (5, 5001, 5, 0.1, False), (4, 8192, 1, 0.1, False), (2100, 64, 300, 0.1, False),
    (1000, 7, 1, 0.1, True),
]


def join_fwd(a, v, stream=None):
    seed = [v["seed"]] if a["drop"] else []
    x = v["x"].shape
    return outputs("join_fwd", [v[k] for k in ("x", "f", "post", "gate", "pre", "scale")] + seed,
                   [x, x, (a["rows"], 2)], du.join_attrs(a), stream)


def join_bwd(a, v, h, stats, slices=None, stream=True):
    if slices is None:
        slices = ooc.join_slices(a["rows"], a["d"], a["groups"])[0]
    seed = [v["seed"]] if a["drop"] else []
    ins = [v["f"], h, stats] + [v[k] for k in ("post", "gate", "pre", "scale")] + seed
    ins += ([v["dh"]] if stream else []) + [v["dn"]]
    outs = [h.shape, h.shape, (a["d"],), v["gate"].shape, (a["d"],), (a["groups"] * slices, 3, a["d"])]
    return outputs("join_bwd", ins, outs, du.join_attrs(a) + [int(stream), slices])[:5]


@pytest.mark.parametrize("case", JOIN, ids=str)
def test_join(case):
    a, v = du.join_case(41, *case)
    h, n, st = join_fwd(a, v)
    for name, got, want, bound in zip(("h", "n", "stats"), (h, n, st), du.join_oracle(a, v),
                                      du.join_bounds(a, v)):
        au.within(name, got, want, bound)
    per = a["rows"] // a["groups"]
    for slices, stream in ((None, True), (1, False), (min(per, 7), True)):
        got = join_bwd(a, v, h, st, slices, stream)
        used = slices or ooc.join_slices(a["rows"], a["d"], a["groups"])[0]
        want = du.join_back_oracle(a, v, h, stream)
        bounds = du.join_back_bounds(a, v, h, used, stream)
        for name, x, y, b in zip(("dx", "df", "dpost", "dgate", "dpre"), got, want, bounds):
            au.within(name, x, y, b)


def test_join_of_zero_rows_and_closed_gates():
    a, v = du.join_case(42, 12, 40, 3, 0.0)
    v["f"][2], v["x"][5], v["f"][5], v["gate"][1] = 0, 0, 0, 0
    h, n, st = join_fwd(a, v)
    for got, want, bound in zip((h, n, st), du.join_oracle(a, v), du.join_bounds(a, v)):
        au.within("forward", got, want, bound)
    assert not h[5].any() and not n[5].any()
    got = join_bwd(a, v, h, st)
    for x, y, b in zip(got, du.join_back_oracle(a, v, h), du.join_back_bounds(a, v, h, 1)):
        au.within("backward", x, y, b)
    assert not got[1][4:8].any() and got[3][1].any()      # a closed gate passes no gradient but has one


# ---------------------------------------------------------------- recurrences
SCAN = [
    # B T C carry fresh
    (1, 1, 1, False, False), (3, 1, 70, True, False), (2, 1, 64, True, True), (1, 2, 5, True, True),
    (2, 16, 64, False, False), (3, 17, 65, True, False), (2, 127, 63, False, True), (2, 128, 130, True, True),
    (1, 129, 3, False, False), (1, 1000, 200, True, True), (5, 300, 33, True, False), (1, 4099, 64, True, True),
    (300, 9, 64, False, True), (1, 20011, 5, False, True), (258, 1030, 2, True, False),
]


def scan_fwd(a, fx, h0, fr, slices=None, stream=None):
    if slices is None:
        slices = ooc.scan_slices("scan_fwd", du.scan_shape(a))[0]
    return outputs("scan_fwd", du.scan_ins(fx, h0, fr), [(a["B"] * a["T"], a["C"])] + du.scan_part(a, slices),
                   du.scan_attrs(a, slices), stream)[0]


def scan_bwd(a, fx, h0, fr, h, dh, slices=None):
    if slices is None:
        slices = ooc.scan_slices("scan_bwd", du.scan_shape(a))[0]
    outs = [fx.shape] + ([h0.shape] if a["carry"] else []) + du.scan_part(a, slices)
    return outputs("scan_bwd", du.scan_ins(fx, h0, fr) + [h, dh], outs, du.scan_attrs(a, slices))[:1 + a["carry"]]


def check_scan(a, fx, h0, fr, dh, slices=(None, None)):
    h = scan_fwd(a, fx, h0, fr, slices[0])
    au.within("h", h, du.scan_oracle(a, fx, h0, fr), du.scan_bound(a, fx, h0, fr))
    got = scan_bwd(a, fx, h0, fr, h, dh, slices[1])
    want = ops.scan_bwd(fx.astype(np.float64), h.astype(np.float64), dh.astype(np.float64), a,
                        None if h0 is None else h0.astype(np.float64), fr)
    for name, x, y, b in zip(("dfx", "dh0"), got, want, du.scan_back_bounds(a, fx, h0, fr, h, dh)):
        au.within(name, x, y, b)
    return [h] + got


@pytest.mark.parametrize("case", SCAN, ids=str)
def test_scan(case):
    check_scan(*du.scan_case(51, *case))


@pytest.mark.parametrize("slices", [2, 3, 7, 64])
def test_scan_slices(slices):
    """Any count that is accepted, with slices that are empty at the end."""
    check_scan(*du.scan_case(52, 2, 100, 67, True, True), slices=(slices, slices))


@pytest.mark.parametrize("shift", [-60.0, 30.0])
def test_scan_gates_shut_and_open(shift):
    """Gates so near 0 or 1 that only 1 - a keeps the other's bits."""
    check_scan(*du.scan_case(53, 2, 300, 40, True, False, shift))


def test_scan_cut_off_by_a_fresh_row():
    """An infinity or a NaN does not pass a row that starts afresh, in either direction, nor a gate
    of zero; sequences do not reach one another."""
    for slices in (1, 5):
        a, fx, h0, fr, dh = du.scan_case(54, 2, 200, 66, True, True)
        fr[:] = 0
        fr[[60, 130]] = 1
        clean = scan_fwd(a, fx, h0, fr, slices)
        back = scan_bwd(a, fx, h0, fr, clean, dh, slices)
        bad_x, bad_d = fx.copy(), dh.copy()
        bad_x[70, 66:] = np.nan
        h = scan_fwd(a, bad_x, h0, fr, slices)
        assert np.isnan(h[70:130]).all()
        ok = np.r_[0:70, 130:400]
        assert np.array_equal(h[ok], clean[ok])
        bad_d[100] = np.inf
        got = scan_bwd(a, fx, h0, fr, clean, bad_d, slices)
        ok = np.r_[0:60, 101:400]
        assert np.array_equal(got[0][ok], back[0][ok]) and np.array_equal(got[1], back[1])
        assert not np.isfinite(got[0][60:101]).all()
        bad_x = fx.copy()
        bad_x[10, 66:], bad_x[20, :66] = np.nan, -np.inf
        h = scan_fwd(a, bad_x, h0, fr, slices)
        assert np.isnan(h[10:20]).all() and np.array_equal(h[20, :], bad_x[20, 66:])
        assert np.isfinite(h[20:200]).all()


def test_scan_goes_on_from_a_state():
    """Row by row, each from the last state, is the whole."""
    a, fx, h0, fr, _ = du.scan_case(55, 3, 6, 70, True, True)
    fr[[2, 9]] = 1
    whole = scan_fwd(a, fx, h0, fr).reshape(3, 6, 70)
    state, one = h0, dict(a, T=1)
    for t in range(6):
        rows = np.arange(3) * 6 + t
        state = scan_fwd(one, fx[rows], state, fr[rows])
        assert np.allclose(state, whole[:, t], rtol=64 * du.U, atol=64 * du.U)


# ---------------------------------------------------------------- graphs, streams, threads
def test_graphs_follow_their_inputs():
    """A captured join, scan and dropout, replayed with another seed and other values between eager
    work: each replay is the eager result of what the memory then holds."""
    a, v = du.join_case(61, 40, 130, 4, 0.2)
    sa, fx, h0, fr, dh = du.scan_case(61, 2, 150, 66, True, True)
    s = hu.Stream()
    jin = [hu.Array(v[k]) for k in ("x", "f", "post", "gate", "pre", "scale", "seed")]
    jout = [hu.empty((40, 130)), hu.empty((40, 130)), hu.empty((40, 2))]
    sin = [hu.Array(t) for t in (fx, h0, fr)]
    h, part = hu.empty((300, 66)), hu.empty((4, 2 * 66 * 2))
    d = hu.Array(dh)
    sback = [hu.empty(fx.shape), hu.empty(h0.shape)]
    x, y = hu.Array(v["x"]), hu.empty((40, 130))

    def calls():
        hu.call("join_fwd", jin + jout, [R] * 7 + [W] * 3, du.join_attrs(a), s)
        hu.call("scan_fwd", sin + [h, part], [R] * 3 + [W] * 2, du.scan_attrs(sa, 4), s)
        hu.call("scan_bwd", sin + [h, d] + sback + [part], [R] * 5 + [W] * 3, du.scan_attrs(sa, 4), s)
        hu.call("dropout", [x, jin[6], y], [R, R, W], [40 * 130, a["drop"], 4], s)
    replay = s.record(calls)
    g = np.random.default_rng(62)
    for _ in range(3):
        v["seed"] = g.integers(0, 1 << 32, 2, dtype=np.uint32)
        fx = (fx + g.standard_normal(fx.shape, np.float32)).astype(np.float32)
        for arr, new in ((jin[6], v["seed"]), (sin[0], fx)):
            hu.check(hu.hip().hipMemcpy(hu.ctypes.c_void_p(arr.ptr), new.ctypes.data_as(hu.ctypes.c_void_p),
                                        hu.ctypes.c_size_t(new.nbytes), 1), "hipMemcpy")
        replay()
        hu.synchronize()
        eager = join_fwd(a, v)
        for got, want in zip(jout, eager):
            assert np.array_equal(got.get(), want)
        want = scan_fwd(sa, fx, h0, fr, 4)
        assert np.array_equal(h.get(), want)
        for got, b in zip(sback, scan_bwd(sa, fx, h0, fr, want, dh, 4)):
            assert np.array_equal(got.get(), b)
        (drop,) = outputs("dropout", [v["x"], v["seed"]], [(40, 130)], [40 * 130, a["drop"], 4])
        assert np.array_equal(y.get(), drop)


def test_two_threads_and_streams():
    cases = [du.scan_case(63 + i, 2, 400 + i, 100, True, True) for i in range(2)]
    want = [scan_fwd(a, fx, h0, fr) for a, fx, h0, fr, _ in cases]
    bad = []

    def work(i):
        s = hu.Stream()
        a, fx, h0, fr, _ = cases[i]
        for _ in range(10):
            if not np.array_equal(scan_fwd(a, fx, h0, fr, stream=s), want[i]):
                bad.append(i)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad
