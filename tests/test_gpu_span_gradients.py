"""Gradients of capped scores far below and far above zero."""

import numpy as np
import pytest

import attention_util as au
from oracle import ops
from span_gradients_util import one_sided_bounds, one_sided_case
from test_gpu_span_attention import span_bwd, span_fwd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("low,high", [(-10, -5), (-7, -0.7), (-3, -1), (5, 10), (1, 3), (-9, 9)])
@pytest.mark.parametrize("dh", [32, 64, 128, 200])
def test_one_sided_scores_under_the_cap(dh, low, high):
    """The cap's factor keeps its bits on either side, however small it is."""
    a, q, kv, span, mod, dy = one_sided_case(181, dh, low, high)
    f = np.float64
    y, lse = span_fwd(a, q, kv, span, mod)
    dq, dkv, _ = span_bwd(a, q, kv, span, mod, y, lse, dy)
    wq, wk, _ = ops.span_attention_bwd(q.astype(f), kv.astype(f), span, dy.astype(f), a, mod)
    bq, bk = one_sided_bounds(q, kv, span, mod, dy, a)
    au.within("dq", dq, wq, bq)
    au.within("dkv", dkv, wk, bk)
