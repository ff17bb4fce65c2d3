"""Span attention, dropout, joins and recurrences on tensors of more than 2^32 bytes and values: what lies
at the far end comes out as from a short call.  Error bounds: decoder_util."""

import ctypes

import numpy as np
import pytest

import attention_util as au
import decoder_util as du
import hip_util as hu
from oracle import ops
from paper_2010_14109_amd import ooc

pytestmark = pytest.mark.gpu
R, W = ooc.R, ooc.W


class Far:
    """Device memory of any size, zeros, of which rows are written and read."""

    def __init__(self, rows, width):
        self.rows, self.width, self.nbytes = rows, width, 4 * rows * width
        p = ctypes.c_void_p()
        hu.check(hu.hip().hipMalloc(ctypes.byref(p), ctypes.c_size_t(self.nbytes)), "hipMalloc")
        self.ptr = p.value
        hu.check(hu.hip().hipMemset(p, 0, ctypes.c_size_t(self.nbytes)), "hipMemset")

    def __del__(self):
        if getattr(self, "ptr", None):
            hu.hip().hipFree(ctypes.c_void_p(self.ptr))

    def _at(self, row, n):
        assert 0 <= row and row + n <= self.rows
        return ctypes.c_void_p(self.ptr + 4 * row * self.width), ctypes.c_size_t(4 * n * self.width)

    def put(self, row, a):
        a = np.ascontiguousarray(a, np.float32).reshape(-1, self.width)
        p, n = self._at(row, len(a))
        hu.check(hu.hip().hipMemcpy(p, a.ctypes.data_as(ctypes.c_void_p), n, 1), "hipMemcpy to the device")

    def get(self, row, n):
        a = np.empty((n, self.width), np.float32)
        p, size = self._at(row, n)
        hu.check(hu.hip().hipMemcpy(a.ctypes.data_as(ctypes.c_void_p), p, size, 2), "hipMemcpy to the host")
        return a


def run(op, ins, outs, attrs):
    hu.call(op, ins + outs, [R] * len(ins) + [W] * len(outs), attrs)
    hu.synchronize()


@pytest.mark.parametrize("Tq,dh,cap", [(1, 128, 0.0), (300, 128, 4.0), (300, 64, 0.0), (5, 256, 0.0)])
def test_span_attention_behind_a_long_cache(Tq, dh, cap):
    near, Hkv = 700, 512 // dh
    Tk = (1 << 22) + 5                                    # rows of 1024 values: 17 GB
    a, q, kv, span, mod, dy = du.span_case(81, 1, Tq, near, Hkv, Hkv, dh, "window", cap, True)
    f, off = np.float64, Tk - near
    y, lse = ops.span_attention_fwd(q.astype(f), kv.astype(f), span, a, mod)
    by, bl, bq, bk = du.span_bounds(q, kv, span, mod, dy, a)
    far = Far(Tk, 1024)
    far.put(off, kv)
    ins = [hu.Array(q), far, hu.Array(np.where(span[:, :1] < span[:, 1:2], span + off, span).astype(np.int32)),
           hu.Array(mod)]
    dy_, y_, l_ = hu.Array(dy), hu.empty(q.shape), hu.empty(lse.shape)
    shape = du.span_attrs(dict(a, Tk=Tk))
    run("span_attention_fwd", ins, [y_, l_, hu.empty((7, q.size + lse.size))], shape + [7])
    au.within("y", y_.get(), y, by)
    au.within("lse", l_.get(), lse, bl)
    dq, dkv = hu.empty(q.shape), Far(Tk, 1024)
    dkv.put(0, np.full((3, 1024), np.nan))
    run("span_attention_bwd", ins + [y_, l_, dy_],
        [dq, dkv, hu.empty(lse.shape), hu.empty((1, -(-Tq // 32), 2), np.int32)], shape + [1, 1])
    wq, wk, _ = ops.span_attention_bwd(q.astype(f), kv.astype(f), span, dy.astype(f), a, mod)
    au.within("dq", dq.get(), wq, bq)
    au.within("dkv", dkv.get(off, near), wk, bk)
    for row in (0, 1 << 20, (1 << 21) - 8, off - 300):     # where 32-bit offsets would end up, and before
        assert not dkv.get(row, 300).any()


def test_scan_of_a_long_sequence():
    B, T, C, n = 2, 1 << 20, 1100, 600                    # FX: 4.6 G values
    a, fx, _, _, dh = du.scan_case(82, 1, n, C)
    FX, H = Far(B * T, 2 * C), Far(B * T, C)
    FX.put(B * T - n, fx)
    slices, part = ooc.scan_slices("scan_fwd", [B, T, C])
    run("scan_fwd", [FX], [H] + [hu.empty(part // 4)] * (slices > 1), [B, T, C, 0, 0, slices])
    h = H.get(B * T - n, n)
    au.within("h", h, du.scan_oracle(a, fx, None, None), du.scan_bound(a, fx, None, None))
    assert not H.get(B * T - 2 * n, n).any() and not H.get(T - n, n).any()
    dH, dFX = Far(B * T, C), Far(B * T, 2 * C)
    dH.put(B * T - n, dh)
    slices, part = ooc.scan_slices("scan_bwd", [B, T, C])
    run("scan_bwd", [FX, H, dH], [dFX] + [hu.empty(part // 4)] * (slices > 1), [B, T, C, 0, 0, slices])
    want = ops.scan_bwd(fx.astype(np.float64), h.astype(np.float64), dh.astype(np.float64), a)[0]
    au.within("dfx", dFX.get(B * T - n, n), want, du.scan_back_bounds(a, fx, None, None, h, dh)[0])
    assert not dFX.get(T - n, n).any()


def test_join_of_many_rows():
    rows, d, n = 540001, 8000, 7                          # 4.3 G values
    a, v = du.join_case(83, n, d, 1)
    X, F, H, N = (Far(rows, d) for _ in range(4))
    X.put(rows - n, v["x"])
    F.put(rows - n, v["f"])
    one = {k: hu.Array(v[k]) for k in ("post", "gate", "pre", "scale")}
    post, gate, pre, scale = one.values()
    stats = hu.empty((rows, 2))
    attrs = [rows, d, 1, 0, 0]
    run("join_fwd", [X, F, post, gate, pre, scale], [H, N, stats], attrs)
    h = H.get(rows - n, n)
    for got, want, bound in zip((h, N.get(rows - n, n), stats.get()[-n:]), du.join_oracle(a, v), du.join_bounds(a, v)):
        au.within("forward", got, want, bound)
    assert not N.get(rows - 2 * n, n).any()
    dN, dF, dX = X, N, Far(rows, d)                       # memory that is free again
    dN.put(rows - n, v["dn"])
    slices, part = ooc.join_slices(rows, d, 1)
    sums = [hu.empty(s) for s in ((d,), (1, d), (d,))]
    run("join_bwd", [F, H, stats, post, gate, pre, scale, dN], [dX, dF] + sums + [hu.empty(part // 4)],
        attrs + [0, slices])
    got = [dX.get(rows - n, n), dF.get(rows - n, n)] + [s.get() for s in sums]
    # (zeros add no rounding; the slices' sums are as many as the longer call has)
    want, bound = du.join_back_oracle(a, v, h, False), du.join_back_bounds(a, v, h, 1, False)
    for x, y, b in zip(got, want, bound):
        au.within("backward", x, y, b)
    assert not dF.get(rows - 2 * n, n).any()


def test_dropout_of_many_values():
    n, tail = (1 << 32) + 6, 42
    x, y = Far(n, 1), Far(n, 1)
    ones = np.ones(tail, np.float32)
    x.put(n - tail, ones)
    seed = np.array([5, 9], np.uint32)
    run("dropout", [x, hu.Array(seed)], [y], [n, 1 << 30, 3])
    words = ops.philox(np.arange(n // 4 - 10, n // 4 + 1), 3, seed).reshape(-1)[:tail]
    assert (n - tail) % 4 == 0 and np.array_equal(y.get(n - tail, tail)[:, 0] > 0, words >= 1 << 30)
    assert not y.get(0, 4096).any()
