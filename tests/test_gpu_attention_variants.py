"""Cross attention and per-head norms in the kernels that test_gpu_attention_ops leaves out, above all the
forward of large batches (256 columns a workgroup)."""

import numpy as np
import pytest

import attention_util as au
import variants_util as vu
from oracle import ops
from test_gpu_attention_ops import check_cross, cross_bwd, cross_fwd
from test_gpu_qknorm_ranges import check as check_qknorm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", vu.CROSS, ids=str)
def test_cross_attention(case):
    a, q, kv, klen, dy = au.cross_case(131, *case)
    if case[-1] is None:
        klen[:3] = a["Tk"], 0, 1
    check_cross(a, q, kv, klen, dy)


@pytest.mark.parametrize("case", vu.QKNORM, ids=str)
def test_qknorm(case):
    check_qknorm(*au.qknorm_case(132, *case))


@pytest.mark.parametrize("dh", [32, 64, 85, 128])
def test_large_batch_with_junk_and_bad_lengths(dh):
    """What lies behind the lengths changes no bit, bad lengths give NaN and only there, a NaN among the
    states stays in its sequence and head, an infinite value in its column."""
    a, q, kv, klen, dy = au.cross_case(133, 32, 129, 70, 16, 16, dh)
    klen[:6] = 70, 0, 1, 33, -1, 71
    states = kv.reshape(32, 70, 2, 16, dh)
    y, lse = cross_fwd(a, q, kv, klen)
    dq, dkv, _ = cross_bwd(a, q, kv, klen, y, lse, dy)
    good = np.ones(32, bool)
    good[4:6] = False
    for t, n in ((y, 129), (dq, 129), (dkv, 70)):
        t = t.reshape(32, n, -1)
        assert np.isnan(t[~good]).all() and np.isfinite(t[good]).all()
    assert np.isnan(lse[~good]).all() and np.isfinite(lse[good][klen[good] > 0]).all()
    assert (lse[1] == -np.inf).all() and not y.reshape(32, 129, -1)[1].any()
    g = np.random.default_rng(134)
    for b in np.flatnonzero(good):
        states[b, klen[b]:] = g.choice(np.array([np.nan, np.inf, -np.inf, 3e38], np.float32),
                                       states[b, klen[b]:].shape)
    y1, lse1 = cross_fwd(a, q, kv, klen)
    dq1, dkv1, _ = cross_bwd(a, q, kv, klen, y, lse, dy)
    for u, v in ((y, y1), (lse, lse1), (dq, dq1), (dkv, dkv1)):
        assert u.tobytes() == v.tobytes()
    states[3, 32, 0, 5, 2] = np.nan          # the last state of sequence 3, key head 5
    states[0, 69, 1, 7, 3] = np.inf          # value column 3 of sequence 0, head 7
    y2, lse2 = cross_fwd(a, q, kv, klen)
    bad = np.zeros((32, 129, 16, dh), bool)
    bad[3, :, 5] = True
    bad[0, :, 7, 3] = True
    same = ~bad & np.isfinite(y).reshape(bad.shape)
    same[0, :, 7] = False                    # the scale of the values' pieces may change there
    same = same.reshape(y.shape)
    assert not np.isfinite(y2[bad.reshape(y.shape)]).any() and np.array_equal(y2[same], y[same])
    assert np.isnan(lse2[3, 5]).all() and np.array_equal(np.delete(lse2[0], 7, 0), np.delete(lse[0], 7, 0))
    au.within("lse", lse2[0, 7], lse[0, 7].astype(np.float64), 4 * au.U * np.abs(lse[0, 7]) + 4 * au.U)
    f = np.float64
    clean = kv.copy()
    clean.reshape(states.shape)[0, 69, 1, 7, 3] = 0
    one = {**a, "B": 1}
    wy, _ = ops.cross_attention_fwd(q[:129].astype(f), clean[:70].astype(f), klen[:1], one)
    by = au.cross_bounds(q[:129], clean[:70], klen[:1], dy[:129], one)[0]
    keep = ~bad[0].reshape(129, -1)
    au.within("y", y2[:129][keep], wy[keep], by[keep])
