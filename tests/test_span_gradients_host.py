"""The cap's factor in fp32, from either side, and what the bounds of one-sided scores tell apart."""

import numpy as np
import pytest

from oracle import ops
from span_gradients_util import U, one_sided_bounds, one_sided_case


@pytest.mark.parametrize("x", [-9.0, -6.0, -3.0, -1.0, 1.0, 3.0, 6.0, 9.0])
def test_the_factor_by_the_magnitude_keeps_its_bits(x):
    """4 r (1 - r) with r = 1 / (1 + exp(2 |x|)) in fp32; by the signed x, r goes to 1 and loses them."""
    one, want = np.float32(1), 1 - np.tanh(np.float64(x)) ** 2

    def factor(x):
        r = one / (one + np.exp(np.float32(2) * np.float32(x)))
        return float(np.float32(4) * (r - r * r))
    bound = (4 * abs(x) + 6) * U + 2 * U        # (the product r r rounds here)
    assert abs(factor(abs(x)) - want) < bound * want
    assert x > -3 or abs(factor(x) - want) > 8 * bound * want


@pytest.mark.parametrize("low,high", [(-10, -5), (5, 10), (-3, -1)])
def test_the_bounds_separate_a_factor_that_is_off(low, high):
    """Planted in the oracle: a factor half a percent off."""
    a, q, kv, span, mod, dy = one_sided_case(181, 64, low, high)
    f = np.float64
    args = [t.astype(f) for t in (q, kv)] + [span, dy.astype(f), a, mod]
    want = ops.span_attention_bwd(*args)
    scores = ops._span_scores

    def planted(*xs):
        S, turn = scores(*xs)
        return S, turn * 1.005
    ops._span_scores = planted
    try:
        got = ops.span_attention_bwd(*args)
    finally:
        ops._span_scores = scores
    bq, bk = one_sided_bounds(q, kv, span, mod, dy, a)
    assert (np.abs(got[0] - want[0]) > bq).mean() > 0.5
    dk = np.arange(kv.shape[1]) < kv.shape[1] // 2
    assert (np.abs(got[1] - want[1]) > bk)[:, dk].mean() > 0.5
