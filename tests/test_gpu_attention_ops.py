"""Rotation, per-head norms and cross attention on the device against the 64-bit oracle, alone and
inside training steps.  Error bounds: attention_util."""

import threading

import numpy as np
import pytest

import attention_util as au
import hip_util as hu
from oracle import ops
from oracle import schedule as S
from oracle.interp import run as oracle_run
from oracle.lower import lower
from paper_2010_14109_amd import netdef, ooc, synth
from test_attention_ops_host import small_seq2seq

pytestmark = pytest.mark.gpu
R, W, RW = ooc.R, ooc.W, ooc.RW


def outputs(op, ins, out_shapes, attrs, stream=None):
    """Runs the operation on fresh memory and returns its outputs; the inputs must be unchanged."""
    arrays = [hu.Array(a) for a in ins] + [hu.empty(s) for s in out_shapes]
    hu.call(op, arrays, [R] * len(ins) + [W] * len(out_shapes), attrs, stream)
    hu.synchronize()
    for a, d in zip(ins, arrays):
        assert d.get().tobytes() == np.ascontiguousarray(a).tobytes(), "an input was written"
    return [d.get() for d in arrays[len(ins):]]


# ---------------------------------------------------------------- rotation
ROPE = [
    # rows heads dh rot layout rest far
    (1, 1, 2, 2, 0, 0, False), (1, 1, 2, 2, 1, 0, True), (1, 20, 64, 64, 1, 256, True),
    (3, 2, 10, 6, 0, 5, True), (3, 2, 10, 6, 1, 5, True), (17, 5, 85, 34, 0, 85, True),
    (17, 5, 85, 84, 1, 1, True), (257, 3, 40, 40, 1, 0, False), (64, 4, 128, 32, 0, 512, False),
    (1031, 6, 48, 16, 1, 96, True), (2053, 2, 96, 96, 0, 3, False), (5, 1, 1500, 1024, 1, 7, True),
    (9, 3, 64, 12, 1, 64, True), (9, 3, 64, 8, 0, 0, True), (4099, 2, 17, 2, 1, 0, True),
    (8200, 3, 32, 32, 1, 32, True), (13, 33, 80, 80, 1, 80, False), (70, 7, 6, 4, 0, 2, True),
]


@pytest.mark.parametrize("case", ROPE, ids=str)
def test_rope(case):
    a, x, pos, table = au.rope_case(11, *case)
    attrs = au.rope_attrs(x, a)
    for op, back in (("rope_fwd", False), ("rope_bwd", True)):
        (y,) = outputs(op, [x, pos, table], [x.shape], attrs)
        ref = ops.rope(x.astype(np.float64), pos, table, a, back=back)
        au.within(op, y, ref, au.rope_bound(x, a, table[-1]))
        n = a["heads"] * a["dh"]
        assert np.array_equal(y[:, n:], x[:, n:])     # copied bit for bit


def test_rope_copies_anything():
    """Columns that are not rotated keep their bits: NaN, infinities, subnormals."""
    a, x, pos, table = au.rope_case(12, 33, 3, 20, 8, 1, 6, False)
    odd = np.array([np.nan, np.inf, -np.inf, 1e-42, -0.0], np.float32)
    h = x[:, :60].reshape(33, 3, 20)
    h[..., 8:] = np.resize(odd, h[..., 8:].shape)
    x[:, :60] = h.reshape(33, 60)
    x[:, 60:] = np.resize(odd, (33, 6))
    (y,) = outputs("rope_fwd", [x, pos, table], [x.shape], au.rope_attrs(x, a))
    keep = np.ones(x.shape, bool)
    keep[:, :60] = np.broadcast_to(np.arange(20) >= 8, (33, 3, 20)).reshape(33, 60)
    assert y[keep].tobytes() == x[keep].tobytes() and np.isfinite(y[~keep]).all()


def test_rope_angles_of_far_positions():
    """The turned unit vectors at the largest positions, where a 32-bit angle would be off by
    hundreds."""
    pos = np.array([0, 1, -1, 1 << 20, (1 << 31) - 1, -(1 << 31), 1234567890], np.int32)
    for f in (1.0, 0.1, 1e-9, 6.283185307179586, 1e3):
        t = np.array([f, 1.0])
        x = np.tile(np.array([1, 0], np.float32), (len(pos), 1))
        (y,) = outputs("rope_fwd", [x, pos, t], [x.shape], [len(pos), 2, 1, 2, 2, 0])
        a = pos.astype(np.float64) * f
        assert np.abs(y - np.stack([np.cos(a), np.sin(a)], 1)).max() <= 8 * au.U, f


# ---------------------------------------------------------------- per-head norms
QKNORM = [
    # rows h1 h2 dh rot layout rest far
    (1, 1, 0, 1, 0, 0, 0, False), (1, 16, 4, 64, 64, 1, 256, True), (77, 16, 4, 64, 64, 1, 256, False),
    (3, 2, 1, 10, 6, 0, 5, True), (3, 2, 1, 10, 6, 1, 5, True), (35, 12, 0, 85, 0, 1, 0, False),
    (35, 3, 3, 85, 84, 1, 17, True), (130, 4, 2, 128, 32, 0, 256, False), (9, 2, 2, 256, 256, 1, 0, True),
    (10, 1, 1, 1024, 1024, 1, 3, True), (10, 1, 2, 1000, 500, 0, 0, True), (2100, 2, 2, 40, 40, 1, 8, True),
    (517, 5, 1, 48, 12, 1, 0, False), (17000, 1, 1, 32, 32, 0, 4, True), (64, 3, 3, 80, 80, 1, 240, False),
    (41, 2, 5, 33, 32, 0, 0, True), (5, 4, 0, 3, 2, 1, 1, False), (12, 2, 2, 300, 40, 1, 12, True),
    (20, 3, 2, 85, 34, 0, 3, True), (20, 3, 2, 85, 34, 1, 3, True), (33, 2, 1, 18, 14, 1, 7, False),
    (9, 1, 1, 7, 2, 1, 2, False), (9, 2, 0, 7, 6, 0, 0, True), (12, 2, 1, 6, 6, 1, 0, False),
    (50, 2, 2, 301, 0, 1, 3, False), (40, 2, 1, 30, 16, 1, 0, True), (64, 8, 2, 96, 32, 0, 192, False),
    (21, 3, 1, 62, 62, 1, 2, True), (13, 1, 1, 1023, 1022, 1, 1, True), (700, 2, 2, 130, 66, 1, 130, False),
    (30, 2, 2, 64, 36, 1, 64, False), (30, 2, 2, 64, 22, 0, 64, True),
]


@pytest.mark.parametrize("case", QKNORM, ids=str)
def test_qknorm(case):
    a, x, gain, where, dy = au.qknorm_case(21, *case)
    attrs, f = au.qknorm_attrs(x, a), np.float64
    (y,) = outputs("qknorm_fwd", [x, gain] + where, [x.shape], attrs)
    n = (a["h1"] + a["h2"]) * a["dh"]
    au.within("y", y, ops.qknorm_fwd(x.astype(f), gain.astype(f), *where, a=a),
              au.qknorm_bound(x, gain, where, a))
    assert np.array_equal(y[:, n:], x[:, n:])
    want = ops.qknorm_bwd(x.astype(f), gain.astype(f), dy.astype(f), *where, a=a)
    for slices in sorted({ooc.qknorm_slices(len(x)), 1 if len(x) < 3000 else 700, min(len(x), 7)}):
        dx, dgain, _ = outputs("qknorm_bwd", [x, gain] + where + [dy],
                               [x.shape, gain.shape, (slices,) + gain.shape], attrs + [slices])
        bx, bg = au.qknorm_back_bound(x, gain, where, dy, a, slices)
        au.within("dx", dx, want[0], bx)
        au.within("dgain", dgain, want[1], bg)
        assert np.array_equal(dx[:, n:], dy[:, n:])


def test_qknorm_zero_rows_and_gains():
    """Heads of zeros divide by sqrt(1e-5); a zero gain stops the gradient but not its own."""
    a, x, gain, where, dy = au.qknorm_case(22, 11, 2, 1, 16, 8, 1, 0, False)
    x[3], x[7, :16], gain[0] = 0, 0, 0
    f = np.float64
    (y,) = outputs("qknorm_fwd", [x, gain] + where, [x.shape], au.qknorm_attrs(x, a))
    au.within("y", y, ops.qknorm_fwd(x.astype(f), gain.astype(f), *where, a=a),
              au.qknorm_bound(x, gain, where, a))
    assert not y[3].any()
    dx, dgain, _ = outputs("qknorm_bwd", [x, gain] + where + [dy],
                           [x.shape, gain.shape, (2,) + gain.shape], au.qknorm_attrs(x, a) + [2])
    want = ops.qknorm_bwd(x.astype(f), gain.astype(f), dy.astype(f), *where, a=a)
    bx, bg = au.qknorm_back_bound(x, gain, where, dy, a, 2)
    au.within("dx", dx, want[0], bx)
    au.within("dgain", dgain, want[1], bg)
    assert not dx[:, :32].any() and dgain[0].any()


# ---------------------------------------------------------------- cross attention
CROSS = [
    # B Tq Tk H Hkv dh klen
    (1, 1, 1, 1, 1, 1, 1), (2, 1, 1, 2, 1, 4, [1, 0]), (3, 5, 7, 4, 2, 16, [7, 0, 3]),
    (2, 33, 65, 2, 2, 64, [65, 64]), (1, 128, 128, 2, 1, 64, 128), (2, 129, 31, 4, 4, 32, [31, 1]),
    (1, 257, 200, 2, 2, 64, 199), (2, 40, 300, 4, 1, 128, [300, 17]), (1, 70, 77, 3, 3, 85, 70),
    (2, 3, 130, 6, 2, 40, [130, 33]), (1, 50, 60, 1, 1, 256, 60), (1, 20, 100, 2, 1, 200, 97),
    (2, 17, 90, 2, 2, 96, [0, 90]), (1, 1, 3000, 8, 2, 64, 2999), (4, 1, 513, 4, 4, 128, None),
    (1, 600, 5, 2, 1, 80, 5), (1, 1000, 64, 1, 1, 64, 64), (3, 65, 97, 5, 5, 17, [97, 32, 64]),
    (2, 200, 333, 2, 2, 48, None), (1, 31, 2049, 2, 2, 33, 2049), (2, 8, 8, 16, 2, 8, [8, 4]),
    (1, 300, 260, 4, 2, 129, 260), (1, 64, 64, 2, 2, 160, 33), (6, 2, 40, 3, 1, 72, None),
    (1, 1, 70000, 1, 1, 16, 70000), (1, 5000, 3, 1, 1, 24, 2), (2, 100, 150, 3, 3, 192, [150, 90]),
]


def cross_fwd(a, q, kv, klen, slices=None, stream=None):
    shape = au.cross_shape(a)
    if slices is None:
        slices = ooc.attention_slices("cross_attention_fwd", shape)[0][0]
    lse = (a["B"], a["H"], a["Tq"])
    part = [(slices, q.size + int(np.prod(lse)))] if slices > 1 else []
    return outputs("cross_attention_fwd", [q, kv, klen], [q.shape, lse] + part, shape + [slices],
                   stream)[:2]


def cross_bwd(a, q, kv, klen, y, lse, dy, slices=None, stream=None):
    shape = au.cross_shape(a)
    if slices is None:
        slices = ooc.attention_slices("cross_attention_bwd", shape)[0]
    sq, sk = slices
    n = max(sq * q.size if sq > 1 else 0, sk * kv.size if sk > 1 else 0)
    return outputs("cross_attention_bwd", [q, kv, klen, y, lse, dy],
                   [q.shape, kv.shape, lse.shape] + ([(n,)] if n else []), shape + list(slices),
                   stream)[:3]


def check_cross(a, q, kv, klen, dy, slices=(None, None), clean=None):
    """One forward and backward within their bounds; ``clean``: kv for the oracle."""
    f = np.float64
    ref_kv = (kv if clean is None else clean).astype(f)
    y, lse = cross_fwd(a, q, kv, klen, slices[0])
    wy, wl = ops.cross_attention_fwd(q.astype(f), ref_kv, klen, a)
    by, bl, bq, bk = au.cross_bounds(q, ref_kv, klen, dy, a)
    au.within("y", y, wy, by)
    au.within("lse", lse, wl, bl)
    dq, dkv, delta = cross_bwd(a, q, kv, klen, y, lse, dy, slices[1])
    wq, wk, _ = ops.cross_attention_bwd(q.astype(f), ref_kv, klen, dy.astype(f), a)
    au.within("dq", dq, wq, bq)
    au.within("dkv", dkv, wk, bk)
    # delta is the row sum of dY Y of the outputs given
    d = (dy.astype(f) * y).reshape(a["B"], a["Tq"], a["H"], -1)
    au.within("delta", delta, d.sum(-1).transpose(0, 2, 1),
              (a["dh"] / 16 + 16) * au.U * np.abs(d).sum(-1).transpose(0, 2, 1))
    return y, lse, dq, dkv


@pytest.mark.parametrize("case", CROSS, ids=str)
def test_cross_attention(case):
    check_cross(*au.cross_case(31, *case))


@pytest.mark.parametrize("spread", [0.0, 8.0, 60.0])
def test_cross_attention_flat_and_peaked_rows(spread):
    """All scores equal, and scores so far apart that one state takes everything."""
    check_cross(*au.cross_case(32, 2, 70, 150, 2, 1, 64, [150, 61], spread=spread))


@pytest.mark.parametrize("slices", [(2, (3, 1)), (5, (1, 4)), (7, (2, 2)), (64, (64, 64)), (1, (1, 1))], ids=str)
def test_cross_attention_any_slices(slices):
    """Counts that leave slices short and sequences that end before a slice begins."""
    check_cross(*au.cross_case(33, 3, 100, 203, 4, 2, 40, [203, 0, 9]), slices=slices)


def test_cross_attention_ignores_what_lies_behind_the_length():
    """NaN, infinities and the largest values at and past klen change nothing, bit for bit."""
    a, q, kv, klen, dy = au.cross_case(34, 3, 37, 100, 4, 2, 24, [100, 33, 0])
    zeroed, junk = kv.copy(), kv.copy()
    g = np.random.default_rng(1)
    for b, n in enumerate(klen):
        rows = slice(b * 100 + n, (b + 1) * 100)
        zeroed[rows] = 0
        junk[rows] = g.choice(np.array([np.nan, np.inf, -np.inf, 3e38], np.float32), junk[rows].shape)
    got = [check_cross(a, q, k, klen, dy, clean=zeroed) for k in (zeroed, junk)]
    for u, v in zip(*got):
        assert u.tobytes() == v.tobytes()
    assert not got[1][3][133:200].any() and not got[1][3][200:].any() and not got[1][0][74:].any()


def test_cross_attention_bad_lengths_give_nan():
    a, q, kv, klen, dy = au.cross_case(35, 4, 40, 50, 2, 2, 64, [50, -1, 51, 7])
    y, lse = cross_fwd(a, q, kv, klen)
    dq, dkv, _ = cross_bwd(a, q, kv, klen, y, lse, dy)
    for t, n in ((y, 40), (dq, 40), (dkv, 50)):
        t = t.reshape(4, n, -1)
        assert np.isnan(t[1:3]).all() and np.isfinite(t[[0, 3]]).all()
    assert np.isnan(lse[1:3]).all() and np.isfinite(lse[[0, 3]]).all()


def test_cross_attention_nan_stays_in_its_sequence_and_head():
    a, q, kv, klen, dy = au.cross_case(36, 2, 40, 50, 2, 2, 32, [50, 30])
    q[3, 40] = np.nan                      # sequence 0, row 3, head 1
    kv[55, 5] = np.nan                     # sequence 1, key head 0
    y, lse = cross_fwd(a, q, kv, klen)
    y = y.reshape(2, 40, 2, 32)
    bad = np.isnan(y).any(-1)
    want = np.zeros((2, 40, 2), bool)
    want[0, 3, 1] = True
    want[1, :, 0] = True
    assert np.array_equal(bad, want) and np.array_equal(np.isnan(lse), want.transpose(0, 2, 1))


def test_cross_attention_infinite_value_stays_in_its_column():
    """A value of infinity: its head column is not finite, the other columns are what they are."""
    a, q, kv, klen, dy = au.cross_case(39, 1, 70, 100, 2, 2, 32, [100])
    clean = kv.copy()
    kv[41, 64 + 7], clean[41, 64 + 7] = np.inf, 0      # key head 0, column 7
    y, _ = cross_fwd(a, q, kv, klen)
    f = np.float64
    want, _ = ops.cross_attention_fwd(q.astype(f), clean.astype(f), klen, a)
    bound = au.cross_bounds(q, clean, klen, dy, a)[0]
    bad = np.zeros(64, bool)
    bad[7] = True
    assert not np.isfinite(y[:, bad]).any()
    au.within("y", y[:, ~bad], want[:, ~bad], bound[:, ~bad])


def test_cross_attention_scales():
    """Values of any size, and sequences whose states differ in size by 2^20 along the keys: the
    sums are accurate relative to what they sum."""
    for i, (sq, sk, sv, sg) in enumerate(((1e-20, 1e20, 1e-15, 1e15), (1e10, 1e-10, 1e25, 1e-25),
                                          (1e-30, 1.0, 1e-30, 1e-3), (1.0, 1.0, 1e30, 1e-30))):
        a, q, kv, klen, dy = au.cross_case(70 + i, 2, 40, 150, 2, 1, 40, [150, 33])
        n = kv.shape[1] // 2
        kv[:, :n] *= np.float32(sk)
        kv[:, n:] *= np.float32(sv)
        check_cross(a, q * np.float32(sq), kv, klen, dy * np.float32(sg))
    a, q, kv, klen, dy = au.cross_case(75, 1, 40, 256, 2, 1, 64, [256])
    kv[:128, 64:] *= np.float32(2.0 ** 20)             # values; and a softmax that looks at the others
    kv[:128, :64], kv[128:, :64] = 0, kv[128:, :64]
    kv[128:, 0] = 60 * np.sign(kv[128:, 0])
    q[:, ::64] = 20
    check_cross(a, q, kv, klen, dy)


@pytest.mark.parametrize("dh", [24, 64, 96, 256])
def test_cross_attention_zero_gradients_of_large_states(dh):
    """Tiles whose score gradients are all zero (no gradient arrives, or the probabilities vanish)
    against states, queries and gradients far above 1."""
    for i, (sq, sk, sv, sg) in enumerate(((2.0 ** -40, 2.0 ** 40, 1.0, 1.0), (2.0 ** 40, 2.0 ** -40, 1.0, 1.0),
                                          (1.0, 1.0, 2.0 ** -30, 2.0 ** 50), (1.0, 1.0, 2.0 ** 60, 2.0 ** -60))):
        a, q, kv, klen, dy = au.cross_case(80 + i, 2, 200, 150, 2, 1, dh, [150, 90])
        n = kv.shape[1] // 2
        dy[:100] = 0                   # the first rows of sequence 0
        dy[200:] = 0                   # all of sequence 1
        kv[:64, :n] *= np.float32(0.01)
        kv[64:150, 0], q[:, ::dh] = 700 * dh ** 0.5, 1   # scores that leave the first tiles nothing
        kv[:, :n] *= np.float32(sk)
        kv[:, n:] *= np.float32(sv)
        check_cross(a, q * np.float32(sq), kv, klen, dy * np.float32(sg))


def test_cross_attention_gradient_of_the_forward_by_differences():
    """The device's gradients against differences of the device's own forward, at a step where
    truncation and rounding of the sum stay below a percent."""
    a, q, kv, klen, dy = au.cross_case(37, 2, 9, 20, 4, 2, 16, [20, 11])
    y, lse = cross_fwd(a, q, kv, klen)
    dq, dkv, _ = cross_bwd(a, q, kv, klen, y, lse, dy)
    g, e = np.random.default_rng(3), 2e-3
    for which, grad in ((0, dq), (1, dkv)):
        v = g.standard_normal(grad.shape).astype(np.float32)
        vals = []
        for s in (1, -1):
            args = [q, kv]
            args[which] = (args[which] + np.float32(s * e) * v).astype(np.float32)
            vals.append((cross_fwd(a, *args, klen)[0].astype(np.float64) * dy).sum())
        want = (grad.astype(np.float64) * v).sum()
        assert abs((vals[0] - vals[1]) / (2 * e) - want) <= 0.01 * np.abs(grad * v).sum() / 10


def test_results_do_not_depend_on_the_run():
    a, q, kv, klen, dy = au.cross_case(38, 3, 130, 300, 4, 2, 64, [300, 100, 0])
    first = check_cross(a, q, kv, klen, dy)
    for _ in range(3):
        y, lse = cross_fwd(a, q, kv, klen)
        dq, dkv, _ = cross_bwd(a, q, kv, klen, y, lse, dy)
        for u, v in zip(first, (y, lse, dq, dkv)):
            assert u.tobytes() == v.tobytes()


# ---------------------------------------------------------------- calls of ooc_run_fn
def test_streams_and_graphs():
    """Rotation, norm and attention in one graph, replayed on other inputs with work between the
    replays; two streams at once."""
    rows, a, n = 96, None, 24
    ra, x, pos, table = au.rope_case(41, rows, 4, 32, 32, 1, 128, False)
    qa = {"h1": 4, "h2": 0, "dh": 32, "rot": 0, "layout": 1}
    gain = np.linspace(0.5, 2, 32, dtype=np.float32).reshape(1, 32)
    a, q, kv, klen, dy = au.cross_case(42, 2, rows // 2, 90, 8, 2, 32, [90, n])
    shape = au.cross_shape(a)
    streams, sets = [hu.Stream(), hu.Stream()], []
    for s in streams:
        d = {k: hu.Array(v) for k, v in dict(x=x, pos=pos, table=table, gain=gain, kv=kv, klen=klen,
                                             dy=dy).items()}
        for k in ("rot", "nrm"):
            d[k] = hu.empty(x.shape)
        for k, like in (("y", q), ("dq", q), ("dkv", kv)):
            d[k] = hu.empty(like.shape)
        for k in ("lse", "delta"):
            d[k] = hu.empty((2, 8, rows // 2))
        fs, fp = ooc.attention_slices("cross_attention_fwd", shape)
        bs, bp = ooc.attention_slices("cross_attention_bwd", shape)
        d["fp"], d["bp"] = hu.empty(max(1, fp // 4)), hu.empty(max(1, bp // 4))
        sets.append(d)

        def calls(d=d, s=s):
            hu.call("rope_fwd", [d["x"], d["pos"], d["table"], d["rot"]], [R, R, R, W],
                    au.rope_attrs(x, ra), s)
            hu.call("qknorm_fwd", [d["rot"], d["gain"], d["nrm"]], [R, R, W],
                    list(x.shape) + [4, 0, 32, 0, 1], s)
            extra = [d["fp"]] if fp else []
            hu.call("cross_attention_fwd", [d["nrm"], d["kv"], d["klen"], d["y"], d["lse"]] + extra,
                    [R, R, R, W, W] + [W] * len(extra), shape + fs, s)
            extra = [d["bp"]] if bp else []
            hu.call("cross_attention_bwd", [d["nrm"], d["kv"], d["klen"], d["y"], d["lse"], d["dy"],
                                            d["dq"], d["dkv"], d["delta"]] + extra,
                    [R] * 6 + [W] * (3 + len(extra)), shape + bs, s)
        d["calls"] = calls
    f = np.float64
    g = np.random.default_rng(43)

    def results(d):
        return [d[k].get() for k in ("rot", "nrm", "y", "lse", "dq", "dkv", "delta")]
    x2 = g.standard_normal(x.shape, np.float32)
    sets[0]["calls"]()
    hu.synchronize()
    eager = results(sets[0])
    r = ops.rope(x.astype(f), pos, table, ra)
    r = ops.qknorm_fwd(r, gain.astype(f), a=qa)
    wy, wl = ops.cross_attention_fwd(r, kv.astype(f), klen, a)
    # the inputs of the attention are themselves rounded: ten times the bound of exact inputs
    by = au.cross_bounds(r.astype(np.float32), kv, klen, dy, a)[0]
    au.within("y of the chain", eager[2], wy, 10 * by)
    replays = [s.record(d["calls"], mode) for s, d, mode in zip(streams, sets, (0, 2))]
    import ctypes
    for step in range(4):
        src = x if step % 2 == 0 else x2
        for d in sets:
            hu.check(hu.hip().hipMemcpy(ctypes.c_void_p(d["x"].ptr), src.ctypes.data_as(ctypes.c_void_p),
                                        ctypes.c_size_t(src.nbytes), 1), "hipMemcpy")
        for r_ in replays:            # both at once
            r_()
        hu.synchronize()
        got = [results(d) for d in sets]
        if step % 2 == 0:
            for u, v in zip(eager, got[0]):
                assert u.tobytes() == v.tobytes()
        for u, v in zip(*got):
            assert u.tobytes() == v.tobytes()
        sets[0]["calls"]()            # the program's own eager work between the replays
        hu.synchronize()
        for u, v in zip(got[0], results(sets[0])):
            assert u.tobytes() == v.tobytes()


def test_two_threads_at_once():
    """Two threads, each on its own stream and memory: the results of one alone."""
    cases = [au.cross_case(44, 2, 70, 130, 4, 2, 64, [130, 50]), au.cross_case(45, 3, 1, 900, 8, 2, 40)]
    alone = [cross_fwd(a, q, kv, klen) for a, q, kv, klen, _ in cases]
    streams, got, errors = [hu.Stream(), hu.Stream()], [[], []], []

    def work(i):
        try:
            a, q, kv, klen, _ = cases[i]
            shape = au.cross_shape(a)
            slices, nbytes = ooc.attention_slices("cross_attention_fwd", shape)
            for _ in range(20):
                d = [hu.Array(v) for v in (q, kv, klen)]
                out = [hu.empty(q.shape), hu.empty(alone[i][1].shape)]
                part = [hu.empty(nbytes // 4)] if nbytes else []
                hu.call("cross_attention_fwd", d + out + part, [R] * 3 + [W] * (2 + len(part)),
                        shape + slices, streams[i])
                hu.synchronize()
                got[i].append([o.get() for o in out])
        except BaseException as e:  # noqa: BLE001 - reported by the test
            errors.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    for i in range(2):
        for pair in got[i]:
            for u, v in zip(pair, alone[i]):
                assert u.tobytes() == v.tobytes()


def test_one_tensor_read_twice():
    """The states' own rows as queries, in the same memory."""
    a, _, kv, klen, dy = au.cross_case(46, 2, 45, 45, 4, 2, 32, [45, 20])
    q = hu.Array(kv)
    y, lse, k = hu.empty(kv.shape), hu.empty((2, 4, 45)), hu.Array(klen)
    shape = au.cross_shape(a)
    slices, nbytes = ooc.attention_slices("cross_attention_fwd", shape)
    part = [hu.empty(nbytes // 4)] if nbytes else []
    hu.call("cross_attention_fwd", [q, q, k, y, lse] + part, [R] * 3 + [W] * (2 + len(part)),
            shape + slices)
    hu.synchronize()
    want = cross_fwd(a, kv, kv, klen)
    assert y.get().tobytes() == want[0].tobytes() and lse.get().tobytes() == want[1].tobytes()


def test_run_fn_refuses_bad_memory():
    """Host memory, memory that is too short, a device that is not there."""
    x = hu.Array(np.zeros(64, np.float32))
    host = np.zeros(96, np.float32)
    at = (host.ctypes.data + 15) // 16 * 16
    for ptrs, what in (([x.ptr, at], "not device memory"), ([at, x.ptr], "not device memory")):
        with pytest.raises(ooc.OocError) as e:
            ooc.run_fn("relu_fwd", [(p, 256) for p in ptrs], [R, W], [64])
        assert e.value.status == ooc.E_INVALID and what in e.value.message
    y = hu.Array(np.zeros(64, np.float32))
    n = (hu.GUARD + 256 + hu.GUARD) // 4 * 8
    with pytest.raises(ooc.OocError) as e:
        ooc.run_fn("relu_fwd", [(x.ptr, 4 * n), (y.ptr, 4 * n)], [R, W], [n])
    assert e.value.status == ooc.E_INVALID and ("longer" in e.value.message or "overlaps" in e.value.message)
    with pytest.raises(ooc.OocError) as e:
        ooc.run_fn("relu_fwd", [(x.ptr, 256), (y.ptr, 256)], [R, W], [64], device=77)
    assert e.value.status == ooc.E_DEVICE
    # and the library works on after every refusal
    ooc.run_fn("relu_fwd", [(x.ptr, 256), (y.ptr, 256)], [R, W], [64])
    hu.synchronize()
    assert not y.get().any()


def test_run_fn_runs_what_a_step_runs():
    """Operations that were there before, alone: the bits of the same function in a context."""
    g = np.random.default_rng(51)
    cases = [
        ("linear_fwd", [(33, 20), (14, 20), (14,)], [(33, 14)], [33, 20, 14]),
        ("layernorm_fwd", [(40, 48), (48,), (48,)], [(40, 48), (2 * 40 + 2 * 2 * 48,)], [40, 48, 2]),
        ("gelu_bwd", [(500,), (500,)], [(500,)], [500]),
        ("attention_fwd", [(2 * 24, 3 * 32)], [(2, 4, 24, 24), (48, 32)], [2, 24, 4, 8, 1]),
    ]
    for op, ins, outs, attrs in cases:
        data = [g.standard_normal(s, np.float32) for s in ins]
        access = [R] * len(ins) + [W] * len(outs)
        alone = outputs(op, data, outs, attrs)
        ctx = ooc.Context(0)
        ids = [ctx.add_var(a.nbytes, ooc.INPUT) for a in data]
        ids += [ctx.add_var(4 * int(np.prod(s)), ooc.OUTPUT) for s in outs]
        ctx.add_fn(op, ids, access, attrs)
        ctx.build_schedule()
        ctx.prepare()
        for i, a in zip(ids, data):
            ctx.host_view(i, shape=a.shape)[...] = a
        ctx.upload()
        ctx.step(0.1)
        ctx.download()
        for i, s, got in list(zip(ids[len(ins):], outs, alone))[:2 if op == "attention_fwd" else 1]:
            assert np.array(ctx.host_view(i, shape=s)).tobytes() == got.tobytes(), op
        ctx.close()


# ---------------------------------------------------------------- offsets past 32 bits
def test_offsets_past_32_bits():
    """A cross attention over 2.3e9 cached values and a rotation of as many: the last sequence and
    the last rows are right."""
    import ctypes
    hip = hu.hip()

    def raw(nbytes):
        p = ctypes.c_void_p()
        hu.check(hip.hipMalloc(ctypes.byref(p), ctypes.c_size_t(nbytes)), "hipMalloc")
        # torch-free fill: the library's own op writes zeros (relu of -1 would need input), so memset
        hu.check(hip.hipMemset(p, 0, ctypes.c_size_t(nbytes)), "hipMemset")
        return p.value

    def put(at, a):
        hu.check(hip.hipMemcpy(ctypes.c_void_p(at), a.ctypes.data_as(ctypes.c_void_p),
                               ctypes.c_size_t(a.nbytes), 1), "hipMemcpy")

    def take(at, shape):
        a = np.empty(shape, np.float32)
        hu.check(hip.hipMemcpy(a.ctypes.data_as(ctypes.c_void_p), ctypes.c_void_p(at),
                               ctypes.c_size_t(a.nbytes), 2), "hipMemcpy")
        return a
    B, Tq, Tk, H, Hkv, dh = 2, 3, 1_150_001, 16, 8, 64      # 2 x 1150001 x 1024 values
    a, q, _, klen, dy = au.cross_case(61, B, Tq, 1, H, Hkv, dh, 1)
    tail = 40
    klen = np.array([tail, Tk], np.int32)
    g = np.random.default_rng(62)
    last = g.standard_normal((tail, 2 * Hkv * dh), np.float32)
    last[:, :Hkv * dh] *= 30                                # the last states win
    row = 2 * Hkv * dh * 4
    kv = raw(B * Tk * row)
    put(kv + (B * Tk - tail) * row, last)
    put(kv, last)
    shape = [B, Tq, Tk, H, Hkv, dh]
    d = {k: hu.Array(v) for k, v in dict(q=q, klen=klen, dy=dy).items()}
    y, lse, delta = hu.empty(q.shape), hu.empty((B, H, Tq)), hu.empty((B, H, Tq))
    fs, fp = ooc.attention_slices("cross_attention_fwd", shape)
    part = [hu.empty(fp // 4)] if fp else []

    def pairs(*arrays):
        return [(v, B * Tk * row) if isinstance(v, int) else (v.ptr, v.nbytes) for v in arrays]
    ooc.run_fn("cross_attention_fwd", pairs(d["q"], kv, d["klen"], y, lse, *part),
               [R, R, R, W, W] + [W] * len(part), shape + fs)
    hu.synchronize()
    small = dict(a, Tk=2 * tail)
    f = np.float64
    # Tk - tail states of zero key and value, then the last ones
    Y, L = y.get(), lse.get()
    k_last = last.reshape(tail, 2, Hkv, dh)
    for b in range(B):
        zeros = 0 if b == 0 else Tk - tail
        for h in range(H):
            qq = q.reshape(B, Tq, H, dh)[b, :, h].astype(f)
            Sx = qq @ k_last[:, 0, h // 2].T.astype(f) / 8
            top = np.maximum(Sx.max(-1), 0)
            e = np.exp(Sx - top[:, None])
            tot = e.sum(-1) + zeros * np.exp(-top)
            want = (e / tot[:, None]) @ k_last[:, 1, h // 2].astype(f)
            assert np.allclose(L[b, h], top + np.log(tot), rtol=1e-5, atol=1e-5)
            assert np.allclose(Y.reshape(B, Tq, H, dh)[b, :, h], want, rtol=1e-3, atol=1e-4)
    dkv = raw(B * Tk * row)
    dq = hu.empty(q.shape)
    bs, bp = ooc.attention_slices("cross_attention_bwd", shape)
    part = []
    if bp:
        part = [raw(bp)]
    ooc.run_fn("cross_attention_bwd",
               pairs(d["q"], kv, d["klen"], y, lse, d["dy"], dq, dkv, delta) +
               [(p, bp) for p in part],
               [R] * 6 + [W] * (3 + len(part)), shape + bs)
    hu.synchronize()
    assert np.isfinite(dq.get()).all()
    got = take(dkv + (B * Tk - tail) * row, (tail, 2, Hkv, dh))
    for hk in range(Hkv):
        want_v, want_k = np.zeros((tail, dh)), np.zeros((tail, dh))
        for h in (2 * hk, 2 * hk + 1):
            qq = q.reshape(B, Tq, H, dh)[1, :, h].astype(f)
            dd = dy.reshape(B, Tq, H, dh)[1, :, h].astype(f)
            P = np.exp(qq @ k_last[:, 0, hk].T.astype(f) / 8 - L[1, h][:, None])
            dl = (dd * Y.reshape(B, Tq, H, dh)[1, :, h]).sum(-1, keepdims=True)
            want_v += P.T @ dd
            want_k += (P * (dd @ k_last[:, 1, hk].T.astype(f) - dl) / 8).T @ qq
        assert np.allclose(got[:, 1, hk], want_v, rtol=1e-3, atol=1e-4)
        assert np.allclose(got[:, 0, hk], want_k, rtol=1e-3, atol=1e-4)
    # a rotation of the same memory, the attention's dkv as its output
    rows, cols = B * Tk, 2 * Hkv * dh
    pos = hu.Array(np.arange(rows, dtype=np.int32))
    table = hu.Array(au.table(64, False))
    ooc.run_fn("rope_fwd", [(kv, rows * row), (pos.ptr, pos.nbytes), (table.ptr, table.nbytes),
                            (dkv, rows * row)], [R, R, R, W], [rows, cols, Hkv, dh, 64, 1])
    hu.synchronize()
    got = take(dkv + (rows - tail) * row, (tail, cols))
    ra = {"heads": Hkv, "dh": dh, "rot": 64, "layout": 1}
    want = ops.rope(last.astype(f), np.arange(rows - tail, rows), au.table(64, False), ra)
    au.within("last rows", got, want, au.rope_bound(last, ra, 1.0))
    for p in [kv, dkv] + part:
        hu.check(hip.hipFree(ctypes.c_void_p(p)), "hipFree")


# ---------------------------------------------------------------- whole training steps
def run_step(spec, x, labels, params, extra, budget=ooc.UNLIMITED, policy="C", steps=1):
    net = netdef.Net(spec, keep_grads=True)
    ctx = ooc.Context(0)
    try:
        net.register(ctx)
        ctx.set_chunk(4096)
        ctx.set_budget(budget)
        ctx.set_policy(policy)
        ctx.build_schedule()
        ctx.prepare()
        for name, v in dict(extra, x=x, labels=labels, **params).items():
            if name in net.ids:
                net.view(ctx, name)[...] = v
        for name in net.names:
            if name.startswith("m:"):
                net.view(ctx, name)[...] = 0
        ctx.upload()
        loss = [ctx.step(spec["optimizer"]["lr"], spec["optimizer"]["momentum"])
                for _ in range(steps)][-1]
        ctx.download()
        return loss, {n: np.array(net.view(ctx, n)) for n in net.names
                      if net.meta[n][2] in (ooc.PARAM, ooc.STATE, ooc.OUTPUT)}
    finally:
        ctx.close()


def seq2seq_data(spec):
    layers = {L["op"]: L for L in spec["layers"]}
    tables = {"table": netdef.rotary_table(layers["qknorm"]["dh"] // 2 * 2),
              "src_table": netdef.rotary_table(layers["rope"]["rot"], scale=4.0, trained=8)}
    x, labels = synth.make_inputs(spec, 0)
    return x, labels, synth.make_params(spec, 1), synth.make_extra_inputs(spec, tables)


def rounding_floors(spec, ref, extra):
    """What rounding alone leaves in gradients that are zero in exact arithmetic.  With one state
    to attend to, P = 1 and dP - delta is the difference of two sums of equal value, so dq and dk
    are zero up to the bounds of ``cross_bounds`` (a few u sum |dy| |v| each), and so is everything
    they alone feed: the gains of both norms, the query projection, and gamma and beta of the norm
    before it.  Returns {gradient: bound}, the bounds carried through |.| of the exact factors: of
    the projection's rows dx, the norm receives dx W, so |d beta| <= sum |dx| |W|, and |d gamma| at
    most sqrt(d) times that, as no normalised value of d columns with a mean square of at most 1
    passes sqrt(d)."""
    out = {}
    for L in spec["layers"]:
        if L["op"] != "cross_attention":
            continue
        b = L["name"].rsplit(".", 1)[0]
        q, kv = (ref[f"{b}.{n}"] for n in ("qn", "kn"))
        B, H, Hkv = spec["input"][0], L["heads"], L["kv_heads"]
        a = {"B": B, "Tq": len(q) // B, "Tk": len(kv) // B, "H": H, "Hkv": Hkv, "dh": q.shape[1] // H}
        _, _, bq, bk = au.cross_bounds(q, kv, extra["src_len"], ref[f"d:{b}.cross@{b}.cproj"], a)
        for name, bound, src, heads in (("qn", bq, "q", H), ("kn", bk[:, :bk.shape[1] // 2], "kv", Hkv)):
            x = ref[f"{b}.{src}"][:, :heads * a["dh"]].reshape(-1, heads, a["dh"])
            r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-5)
            w = bound.reshape(x.shape)
            out[f"d:{b}.{name}.gain"] = (w * np.abs(x) * r).sum((0, 1))
            if name == "qn":
                w = w * np.abs(ref[f"{b}.qn.gain"][0])
                u = np.abs(x) * r
                dx = (r * (w + u * (w * u).mean(-1, keepdims=True))).reshape(len(x), -1)
                out[f"d:{b}.q.W"] = dx.T @ np.abs(ref[f"{b}.ln2"])
                out[f"d:{b}.q.b"] = dx.sum(0)
                out[f"d:{b}.ln2.beta"] = dx.sum(0) @ np.abs(ref[f"{b}.q.W"]).reshape(dx.shape[1], -1)
                out[f"d:{b}.ln2.gamma"] = out[f"d:{b}.ln2.beta"] * dx.shape[1] ** 0.5
    return out


@pytest.mark.parametrize("kw", [{}, dict(d=64, heads=2, kv_heads=1, seq=33, src_seq=70, vocab=50),
                                dict(batch=1, seq=1, src_seq=1)], ids=str)
def test_seq2seq_step(kw):
    """Loss, every gradient and update of a step against the oracle; out of core, the same bits."""
    spec = small_seq2seq(**kw)
    x, labels, params, extra = seq2seq_data(spec)
    loss, outs = run_step(spec, x, labels, params, extra)
    reg = lower(spec, keep_grads=True, slices=netdef.Net(spec, True).slices)
    ref = oracle_run(reg, x, labels, {k: v.astype(np.float64) for k, v in params.items()}, inputs=extra)
    assert abs(loss - ref["loss"][-1]) <= 1e-5 * abs(ref["loss"][-1])
    floors = rounding_floors(spec, ref, extra)
    lr = spec["optimizer"]["lr"]
    for name, v in outs.items():
        want = ref[name].reshape(v.shape)
        # the whole-step tolerance of the other networks; a momentum buffer holds its gradient
        floor = floors.get(name.replace("m:", "d:"), np.multiply(floors.get("d:" + name, 0.0), lr))
        norm = np.linalg.norm(want)
        assert np.linalg.norm(v - want) <= 1e-4 * norm + np.linalg.norm(floor) + 1e-9, name
    net = netdef.Net(spec, keep_grads=True)
    b, k, f = net.var_bytes, net.var_kinds, net.fn_vars
    for frac, policy in ((0.5, "C"), (0.0, "C"), (0.4, "L")):
        budget = max(S.budget_for(frac, S.incore_peak(b, k, f, 4096), 4096) if frac else 0,
                     S.working_set_max(b, f, 4096))
        got = run_step(spec, x, labels, params, extra, budget, policy, steps=2)
        want2 = run_step(spec, x, labels, params, extra, steps=2)
        assert got[0] == want2[0]
        for name in got[1]:
            assert got[1][name].tobytes() == want2[1][name].tobytes(), (name, frac, policy)
