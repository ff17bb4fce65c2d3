"""The oracle's recurrence where values are not finite."""

import numpy as np

import decoder_util as du
from oracle import ops


def test_the_oracle_cuts_off_what_is_not_finite():
    a, fx, h0, fr, dh = du.scan_case(54, 2, 12, 3, True, True)
    fx, h0, dh = (t.astype(np.float64) for t in (fx, h0, dh))
    fr[:] = 0
    fr[5] = 1
    clean = ops.scan_fwd(fx, a, h0, fr)
    bad = fx.copy()
    bad[3, 1] = np.nan
    h = ops.scan_fwd(bad, a, h0, fr)
    assert np.isnan(h[3:5, 1]).all()
    h[3:5, 1] = clean[3:5, 1]
    assert np.array_equal(h, clean)
    back = ops.scan_bwd(fx, clean, dh, a, h0, fr)
    bad = dh.copy()
    bad[7, 2] = np.inf
    got = ops.scan_bwd(fx, clean, bad, a, h0, fr)
    ok = np.ones(got[0].shape, bool)
    ok[5:8, [2, 5]] = False
    assert np.array_equal(got[0][ok], back[0][ok]) and np.array_equal(got[1], back[1])
    fx[8, 0], fx[6, 3] = -np.inf, np.nan      # a gate of zero behind a NaN
    h = ops.scan_fwd(fx, a, h0, fr)
    assert np.isnan(h[6:8, 0]).all() and h[8, 0] == fx[8, 3] and np.isfinite(h[8:]).all()
    dfx = ops.scan_bwd(fx, h, dh, a, h0, fr)[0]
    assert abs(dfx[8, 0]) < 1e-200 and np.isfinite(dfx[8:]).all() and np.isnan(dfx[6:8, 0]).all()
