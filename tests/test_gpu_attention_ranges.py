"""Cross attention over states of unlike sizes, on the device against the 64-bit oracle, through each of
its forward kernels.  Error bounds: attention_util."""

import numpy as np
import pytest

import attention_util as au
from test_gpu_attention_ops import check_cross, cross_fwd
from oracle import ops

pytestmark = pytest.mark.gpu

#: B Tq Tk H Hkv dh klen of a call that each forward kernel takes
KERNELS = {
    "few": (32, 3, 300, 16, 8, 64, None),
    "few, odd width": (64, 1, 300, 8, 4, 85, None),
    "128 columns": (2, 150, 300, 2, 1, 64, [300, 131]),
    "128 columns, pairs": (1, 70, 200, 2, 2, 96, [190]),
    "64 columns": (1, 70, 200, 1, 1, 160, [190]),
    "256 columns": (64, 129, 140, 8, 8, 32, None),
}
#: factors of the values of the first 64 states and of the others, and whether the first have all
#: probabilities vanish
SIZES = [(0.0, 2.0 ** -16, False), (0.0, 2.0 ** -30, False), (0.0, 2.0 ** -50, False),
         (0.0, 2.0 ** -90, False), (2.0 ** -70, 2.0 ** 70, False), (2.0 ** -64, 2.0 ** 64, False),
         (2.0 ** 70, 2.0 ** -70, True), (2.0 ** 20, 2.0 ** -40, True), (1.0, 0.0, False),
         (2.0 ** 90, 2.0 ** -90, False), (1.0, 2.0 ** -60, True)]


@pytest.mark.parametrize("sizes", SIZES, ids=str)
@pytest.mark.parametrize("kernel", KERNELS)
def test_values_of_unlike_sizes(kernel, sizes):
    """The output is accurate relative to what it sums, and lse does not depend on the values."""
    a, q, kv, klen, dy = au.cross_case(91, *KERNELS[kernel])
    first, later, vanish = sizes
    states = kv.reshape(a["B"], a["Tk"], 2, a["Hkv"], a["dh"])
    states[:, :64, 1] *= np.float32(first)
    states[:, 64:, 1] *= np.float32(later)
    if vanish:                       # scores 400 and more apart: weights of 0 in fp32, and in effect
        q[:, ::a["dh"]] = a["dh"] ** 0.5
        states[:, :64, 0, :, 0] = -450
        klen = np.maximum(klen, 65)  # (a sequence of the first states alone would look at them)
    y, lse = cross_fwd(a, q, kv, klen)
    f = np.float64
    wy, wl = ops.cross_attention_fwd(q.astype(f), kv.astype(f), klen, a)
    by, bl, _, _ = au.cross_bounds(q, kv, klen, dy, a)
    au.within("lse", lse, wl, bl)
    au.within("y", y, wy, by)


@pytest.mark.parametrize("kernel", KERNELS)
def test_gradients_of_unlike_sizes(kernel):
    """Whole gradients, which recompute the probabilities from lse, where the first values are zero."""
    a, q, kv, klen, dy = au.cross_case(92, *KERNELS[kernel])
    states = kv.reshape(a["B"], a["Tk"], 2, a["Hkv"], a["dh"])
    states[:, :64, 1] = 0
    states[:, 64:, 1] *= np.float32(2.0 ** -50)
    check_cross(a, q, kv, klen, dy * np.float32(2.0 ** 40))
