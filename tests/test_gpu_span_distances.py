"""Distance bias of states that lie far into a sequence."""

import numpy as np
import pytest

import attention_util as au
import decoder_util as du
import hip_util as hu
from oracle import ops
from test_gpu_far_offsets import Far, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Tq,dh,cap", [(40, 8, 0.0), (300, 8, 3.0), (40, 72, 3.0), (300, 72, 0.0), (3, 16, 0.0)])
def test_distances_across_two_to_the_24(Tq, dh, cap):
    """Places up to 2^24, states behind them: distances of a few rows are exact there.

    Most of the 700 states are so far from a query that their probability is near 2^-126 or below.  The
    exponential instruction gives 0 for results below 2^-126, so such a term p is missing in whole: to the bounds
    of dv and dk come sum 2^-126 |dY| and sum 2^-126 |dP - delta| |q| / sqrt(dh) over the queries."""
    near, far_rows = 700, (1 << 24) + 350
    off = far_rows - near
    a, q, kv, span, mod, dy = du.span_case(182, 1, Tq, near, 1, 1, dh, "all", cap, True)
    mod[-1] = 0.7
    span[:, 2] = (1 << 24) - off - np.random.default_rng(183).integers(0, 30, Tq)
    span[::3, 2] = (1 << 24) - off
    f = np.float64
    y, lse = ops.span_attention_fwd(q.astype(f), kv.astype(f), span, a, mod)
    wq, wk, _ = ops.span_attention_bwd(q.astype(f), kv.astype(f), span, dy.astype(f), a, mod)
    by, bl, bq, bk = du.span_bounds(q, kv, span, mod, dy, a)
    v, d = kv[:, dh:].astype(f), dy.astype(f)
    slope = np.abs(d @ v.T - (d * y).sum(-1, keepdims=True)) / np.sqrt(dh)
    bk = bk + 2.0 ** -126 * np.concatenate([slope.T @ np.abs(q.astype(f)),
                                            np.broadcast_to(np.abs(d).sum(0), v.shape)], 1)
    far, dkv = Far(far_rows, 2 * dh), Far(far_rows, 2 * dh)
    far.put(off, kv)
    ins = [hu.Array(q), far, hu.Array((span + off).astype(np.int32)), hu.Array(mod)]
    y_, l_, dq = hu.empty(q.shape), hu.empty(lse.shape), hu.empty(q.shape)
    shape = du.span_attrs(dict(a, Tk=far_rows))
    run("span_attention_fwd", ins, [y_, l_], shape + [1])
    au.within("y", y_.get(), y, by)
    au.within("lse", l_.get(), lse, bl)
    run("span_attention_bwd", ins + [y_, l_, hu.Array(dy)],
        [dq, dkv, hu.empty(lse.shape), hu.empty((1, -(-Tq // 32), 2), np.int32)], shape + [1, 1])
    au.within("dq", dq.get(), wq, bq)
    au.within("dkv", dkv.get(off, near), wk, bk)
    assert not dkv.get(off - 5000, 5000).any()
