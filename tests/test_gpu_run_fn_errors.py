"""``ooc.run_fn`` beside other users of the HIP runtime."""

import ctypes

import numpy as np
import pytest

import hip_util as hu
from paper_2010_14109_amd import ooc

pytestmark = pytest.mark.gpu


def test_an_earlier_error_is_not_the_launchs():
    """An allocation that fails leaves its error pending: the next operation runs, and clears it."""
    x, y = hu.Array(np.linspace(-1, 1, 64, dtype=np.float32)), hu.empty(64)
    p = ctypes.c_void_p()
    assert hu.hip().hipMalloc(ctypes.byref(p), ctypes.c_size_t(1 << 55)) != 0 and not p.value
    assert hu.hip().hipPeekAtLastError() != 0
    hu.call("relu_fwd", [x, y], [ooc.R, ooc.W], [64])
    assert hu.hip().hipPeekAtLastError() == 0
    hu.synchronize()
    assert np.array_equal(y.get(), np.maximum(x.get(), 0))
