"""The gated recurrence's kernel of 64 columns a workgroup (more than 1024 rows, or more than 2^21 values), with
columns past the first 64, states handed in, rows that start afresh, and slices.  Bounds: decoder_util."""

import threading

import numpy as np
import pytest

import decoder_util as du
import hip_util as hu
from paper_2010_14109_amd import ooc
from test_gpu_decoder_ops import check_scan, scan_bwd, scan_fwd

pytestmark = pytest.mark.gpu
R, W = ooc.R, ooc.W


@pytest.mark.parametrize("case", [
    # B T C carry fresh
    (1, 2100, 130, True, True), (2, 1500, 1365, True, True), (1, 1500, 128, True, True), (3, 1025, 65, True, False),
    (2, 1100, 191, False, True), (26, 128, 700, True, True), (12, 300, 700, True, True), (300, 120, 96, True, True),
], ids=str)
def test_scan(case):
    check_scan(*du.scan_case(56, *case))


@pytest.mark.parametrize("slices", [1, 2, 3, 7, 64])
def test_scan_slices(slices):
    """Any count that is accepted, with slices that are empty at the end."""
    for B, T, C in ((2, 1100, 130), (3, 700, 1100)):
        check_scan(*du.scan_case(57, B, T, C, True, True), slices=(slices, slices))


@pytest.mark.parametrize("shift", [-60.0, 30.0])
def test_scan_gates_shut_and_open(shift):
    check_scan(*du.scan_case(58, 2, 1300, 70, True, False, shift))


def sliced_case(seed):
    a, fx, h0, fr, dh = du.scan_case(seed, 1, 2100 + seed, 130, True, True)
    counts = [ooc.scan_slices(op, du.scan_shape(a))[0] for op in ("scan_fwd", "scan_bwd")]
    assert min(counts) > 1
    return a, fx, h0, fr, dh


def test_a_graph_follows_its_inputs():
    """Both directions recorded with their slices and replayed on other values: the eager results."""
    a, fx, h0, fr, dh = sliced_case(1)
    (sf, pf), (sb, pb) = (ooc.scan_slices(op, du.scan_shape(a)) for op in ("scan_fwd", "scan_bwd"))
    s = hu.Stream()
    ins, d = [hu.Array(t) for t in (fx, h0, fr)], hu.Array(dh)
    h, back = hu.empty(dh.shape), [hu.empty(fx.shape), hu.empty(h0.shape)]
    parts = [hu.empty((n // 4,)) for n in (pf, pb)]

    def calls():
        hu.call("scan_fwd", ins + [h, parts[0]], [R] * 3 + [W] * 2, du.scan_attrs(a, sf), s)
        hu.call("scan_bwd", ins + [h, d] + back + [parts[1]], [R] * 5 + [W] * 3, du.scan_attrs(a, sb), s)
    replay = s.record(calls)
    g = np.random.default_rng(59)
    for _ in range(3):
        fx = (fx + g.standard_normal(fx.shape, np.float32)).astype(np.float32)
        hu.check(hu.hip().hipMemcpy(hu.ctypes.c_void_p(ins[0].ptr), fx.ctypes.data_as(hu.ctypes.c_void_p),
                                    hu.ctypes.c_size_t(fx.nbytes), 1), "hipMemcpy")
        replay()
        hu.synchronize()
        want = scan_fwd(a, fx, h0, fr)
        for got, w in zip([h] + back, [want] + scan_bwd(a, fx, h0, fr, want, dh)):
            assert np.array_equal(got.get(), w)


def test_two_threads_and_streams():
    cases = [sliced_case(i) for i in range(2)]
    want = []
    for a, fx, h0, fr, dh in cases:
        h = scan_fwd(a, fx, h0, fr)
        want.append([h] + scan_bwd(a, fx, h0, fr, h, dh))
    bad = []

    def work(i):
        s = hu.Stream()
        a, fx, h0, fr, dh = cases[i]
        for _ in range(5):
            got = [scan_fwd(a, fx, h0, fr, stream=s)] + scan_bwd(a, fx, h0, fr, want[i][0], dh)
            bad.extend(i for x, y in zip(got, want[i]) if not np.array_equal(x, y))
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad
