"""Span attention in the kernels that test_gpu_span_attention leaves out, above all the forward with 256
columns a workgroup.  Bounds: decoder_util."""

import numpy as np
import pytest

import attention_util as au
import decoder_util as du
import span_variants_util as sv
from oracle import ops
from test_gpu_span_attention import check_span, span_bwd, span_fwd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", sv.SPAN, ids=str)
def test_span_attention(case):
    check_span(*du.span_case(171, *case))


@pytest.mark.parametrize("dh,cap", [(128, 3.0), (85, 0.0)])
def test_wide_forward_in_slices(dh, cap):
    check_span(*du.span_case(172, 16, 140, 150, 32, 32, dh, "any", cap, True), slices=(3, (2, 2)))


@pytest.mark.parametrize("dh,cap", [(128, 0.0), (128, 4.0), (96, 4.0), (101, 0.0)])
def test_wide_forward_beside_what_is_not_finite(dh, cap):
    """States with a NaN or an infinity reach the queries that see them and no other; spans that reach
    outside the states give NaN, empty ones zeros."""
    B, T, H = 16, 140, 32
    a, q, kv, span, mod, dy = du.span_case(173, B, T, T, H, H, dh, "any", cap, True)
    assert sv.span_kernels(B, T, T, H, H, dh, "any", cap, True)[0][0] == "wide"
    outside = np.array([3, 2 * T + 131])
    span[outside] = (-1, 40, 0), (100, T + 1, 0)
    bad = kv.reshape(B, T, 2, H, dh).copy()
    hits = np.zeros((B, H, T), bool)                 # states that are not finite
    g = np.random.default_rng(174)
    for n, (b, h, j) in enumerate(((0, 0, 5), (0, 0, 77), (2, 31, 139), (15, 7, 0), (9, 16, 64))):
        bad[b, j, n % 2, h, g.integers(dh)] = (np.nan, np.inf, -np.inf)[n % 3]
        hits[b, h, j] = True
    zero = np.where(np.isfinite(bad), bad, 0).reshape(kv.shape)
    bad = bad.reshape(kv.shape)
    sp = span.reshape(B, T, 3)
    j = np.arange(T)
    seen = (j >= sp[..., :1]) & (j < sp[..., 1:2])
    off = np.zeros((B, T), bool)
    off.reshape(-1)[outside] = True
    seen &= ~off[..., None]
    none = (seen[:, None] & hits[:, :, None]).any(-1) | off[:, None]          # [B, H, T]
    y, lse = span_fwd(a, q, bad, span, mod)
    f = np.float64
    clean = span.copy()
    clean[outside] = 0
    wy, wl = ops.span_attention_fwd(q.astype(f), zero.astype(f), clean, a, mod)
    by, bl, bq, bk = du.span_bounds(q, zero, clean, mod, dy, a)
    rows = none.transpose(0, 2, 1)[..., None].repeat(dh, -1).reshape(q.shape)
    assert hits.any() and np.isnan(y[rows]).all() and np.isnan(lse[none]).all()
    au.within("y", y[~rows], wy[~rows], by[~rows])
    au.within("lse", lse[~none], wl[~none], bl[~none])
    dq, dkv, _ = span_bwd(a, q, bad, span, mod, y, lse, dy)
    wq, wk, _ = ops.span_attention_bwd(q.astype(f), zero.astype(f), clean, dy.astype(f), a, mod)
    assert np.isnan(dq[rows]).all()
    au.within("dq", dq[~rows], wq[~rows], bq[~rows])
    reached = (seen[:, None] & none[..., None]).any(2)                        # [B, H, state]
    reached = np.broadcast_to(reached.transpose(0, 2, 1)[:, :, None, :, None], (B, T, 2, H, dh)).reshape(kv.shape)
    au.within("dkv", dkv[~reached], wk[~reached], bk[~reached])
    assert np.isnan(dkv[reached]).all()
