"""Gated recurrences whose gates, values or gradients are not finite: a row that starts afresh, or a gate of
zero, keeps them from the rows beyond it, in the same lane's run of rows, in another run of its wave, in
another wave and in another slice, in both directions."""

import numpy as np
import pytest

import attention_util as au
import decoder_util as du
from test_gpu_decoder_ops import scan_bwd, scan_fwd

pytestmark = pytest.mark.gpu

# B T C slices, a row with a NaN, the row behind it that starts afresh.  Up to 1024 rows, 16 columns a
# workgroup, a wave has 4 runs of 16 rows (of 8 backward); above, 64 columns and one run.
CUTS = [
    (2, 200, 66, 1, 3, 5), (2, 200, 66, 1, 3, 20), (2, 200, 66, 1, 37, 45), (2, 200, 66, 1, 3, 70),
    (2, 200, 66, 1, 130, 198), (2, 200, 66, 5, 3, 5), (2, 200, 66, 5, 45, 59), (2, 200, 66, 5, 3, 90),
    (2, 200, 66, 64, 3, 5), (2, 200, 66, 1, 198, 199), (1, 1500, 130, 1, 3, 5), (1, 1500, 130, 1, 3, 20),
    (1, 1500, 130, 1, 100, 400), (1, 1500, 130, 5, 3, 5), (1, 1500, 130, 5, 20, 290), (1, 1500, 130, 5, 20, 700),
    (2, 200, 66, 5, 1, 90), (2, 1500, 130, 64, 1000, 1003), (2, 1500, 130, 11, 1498, 1499),
]


def case(B, T, C, seed=54):
    a, fx, h0, fr, dh = du.scan_case(seed, B, T, C, True, True)
    fr[:] = 0
    return a, fx, h0, fr, dh


@pytest.mark.parametrize("cut", CUTS, ids=str)
def test_a_gate_that_is_no_number(cut):
    B, T, C, slices, at, cut_at = cut
    a, fx, h0, fr, dh = case(B, T, C)
    first = at - min(at, 2)                          # the row's own document: first .. cut_at
    fr[[first, cut_at]] = first > 0, 1
    bad = fx.copy()
    bad[at, :C:3] = np.nan
    hit = np.zeros(C, bool)
    hit[::3] = True
    clean = scan_fwd(a, fx, h0, fr, slices)
    h = scan_fwd(a, bad, h0, fr, slices)
    reached = np.zeros((B * T, C), bool)
    reached[at:cut_at] = hit
    assert np.isnan(h[reached]).all() and np.array_equal(h[~reached], clean[~reached])
    want = scan_bwd(a, fx, h0, fr, clean, dh, slices)
    got = scan_bwd(a, bad, h0, fr, h, dh, slices)
    df, dx = (np.split(t, 2, 1) for t in (got[0], want[0]))
    # the NaN's row and those before it, back to where its document starts, and df of those behind it,
    # whose state before is NaN
    back = np.zeros((B * T, C), bool)
    back[first:at + 1] = hit
    for mine, clean_grad, r in zip(df, dx, (back | reached, back)):
        assert np.isnan(mine[r]).all() and np.array_equal(mine[~r], clean_grad[~r])
    if first:
        assert np.array_equal(got[1], want[1])
    else:
        assert np.isnan(got[1][0, hit]).all() and np.array_equal(got[1][0, ~hit], want[1][0, ~hit])
        assert np.array_equal(got[1][1:], want[1][1:])


@pytest.mark.parametrize("cut", CUTS, ids=str)
def test_any_count_of_slices_gives_the_same(cut):
    """Where a gate is no number, too: the same rows are none, and the others agree within the bounds of two
    calls, which are those of the values without the NaN."""
    B, T, C, slices, at, cut_at = cut
    a, fx, h0, fr, dh = case(B, T, C, 55)
    fr[cut_at] = 1
    bad = fx.copy()
    bad[at, :C:2] = np.nan
    clean = scan_fwd(a, fx, h0, fr, 1)
    bounds = (du.scan_bound(a, fx, h0, fr),) + du.scan_back_bounds(a, fx, h0, fr, clean, dh)
    h = scan_fwd(a, bad, h0, fr, 1)
    one, other = ([scan_fwd(a, bad, h0, fr, n)] + scan_bwd(a, bad, h0, fr, h, dh, n) for n in (1, slices))
    for name, x, y, b in zip(("h", "dfx", "dh0"), one, other, bounds):
        au.within(name, y, x, 2 * b)


@pytest.mark.parametrize("shape", [(2, 200, 66, 1), (2, 200, 66, 5), (1, 1500, 130, 1), (1, 1500, 130, 64)], ids=str)
def test_gradients_at_a_gate_of_zero(shape):
    """A state that is no number does not count there, for the gate's own gradient either."""
    B, T, C, slices = shape
    a, fx, h0, fr, dh = case(B, T, C, 56)
    fx[[20, 61], :C], fx[60, :C] = -np.inf, -200.0
    clean = scan_fwd(a, fx, h0, fr, slices)
    want = scan_bwd(a, fx, h0, fr, clean, dh, slices)
    bad, nan_state = fx.copy(), h0.copy()
    bad[10, C::2], bad[59, C::3], nan_state[0] = np.nan, np.inf, np.nan
    h = scan_fwd(a, bad, nan_state, fr, slices)
    assert np.array_equal(h[20:59], clean[20:59]) and np.array_equal(h[60:], clean[60:])
    got = scan_bwd(a, bad, nan_state, fr, h, dh, slices)
    rows = np.r_[20:59, 60:B * T]
    assert np.array_equal(got[0][rows], want[0][rows]) and not got[0][[20, 60], :C].any()
    assert np.array_equal(got[0][:, C:], want[0][:, C:]) and np.array_equal(got[1], want[1])
