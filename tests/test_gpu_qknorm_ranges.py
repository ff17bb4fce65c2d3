"""Per-head norms at the limits of their documented ranges and in every variant of their kernels, on the
device against the 64-bit oracle.  Error bounds: attention_util."""

import numpy as np
import pytest

import attention_util as au
from oracle import ops
from paper_2010_14109_amd import ooc
from test_gpu_attention_ops import outputs

pytestmark = pytest.mark.gpu


def check(a, x, gain, where, dy):
    attrs, f = au.qknorm_attrs(x, a), np.float64
    (y,) = outputs("qknorm_fwd", [x, gain] + where, [x.shape], attrs)
    au.within("y", y, ops.qknorm_fwd(x.astype(f), gain.astype(f), *where, a=a),
              au.qknorm_bound(x, gain, where, a))
    slices = ooc.qknorm_slices(len(x))
    dx, dgain, _ = outputs("qknorm_bwd", [x, gain] + where + [dy],
                           [x.shape, gain.shape, (slices,) + gain.shape], attrs + [slices])
    want = ops.qknorm_bwd(x.astype(f), gain.astype(f), dy.astype(f), *where, a=a)
    bx, bg = au.qknorm_back_bound(x, gain, where, dy, a, slices)
    au.within("dx", dx, want[0], bx)
    au.within("dgain", dgain, want[1], bg)


@pytest.mark.parametrize("dh", [1, 64, 85, 340, 341, 400, 1023, 1024])
@pytest.mark.parametrize("size", [1e18, 1e-18])
def test_largest_and_smallest_values(dh, size):
    """Every value of a row at the documented limit: the sum of dh squares must not pass fp32's range.
    And values whose squares vanish: the norm divides by sqrt(1e-5)."""
    rot = dh // 4 * 2
    a, x, gain, where, dy = au.qknorm_case(25, 9, 2, 1, dh, rot, 1, 3, False)
    x = (size * (1 - 0.5 * np.random.default_rng(26).random(x.shape))).astype(np.float32) * np.sign(x)
    x[:3] = np.float32(size)
    x[4, :dh] = 0
    check(a, x, gain, where, dy)
