"""Cross attention over states of unlike sizes, on the device against the 64-bit oracle, through each of
its forward kernels.  Error bounds: attention_util."""

import numpy as np
import pytest

import attention_util as au
from test_gpu_attention_ops import check_cross, cross_bwd, cross_fwd
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
    "256 columns, eight waves": (64, 129, 140, 8, 8, 72, None),
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


# ---------------------------------------------------------------- bits of small terms
# The bounds below count what include/ooc.h states: two pieces of a value are off by 2^-23 of it (2 u) or
# 2^-39 of the largest value it is read with, the pieces of a probability by 2^-23 of it or 2^-35 of the
# largest, and the products of two low pieces, 2^-22 (4 u) at most, are left out.  Each matrix instruction
# (3 for 16 terms, in two halves) and each addition rounds once more.

def uniform(kernel, seed=93, lengths=None):
    """A case whose scores are all zero: every probability is 1 / klen."""
    B, Tq, Tk, H, Hkv, dh, klen = KERNELS[kernel]
    if lengths is not None:
        klen = np.resize(lengths, B)
    a, q, kv, klen, dy = au.cross_case(seed, B, Tq, Tk, H, Hkv, dh, klen)
    return a, np.zeros_like(q), kv, np.maximum(klen, 1), dy


@pytest.mark.parametrize("lengths", [[1], [2, 3], [33, 5], [64, 100, 17], [140]], ids=str)
@pytest.mark.parametrize("kernel", KERNELS)
def test_means_of_few_states(kernel, lengths):
    """y is the mean of klen states and lse their count's logarithm, as exactly as fp32 has them."""
    a, q, kv, klen, dy = uniform(kernel, lengths=lengths)
    y, lse = cross_fwd(a, q, kv, klen)
    f = np.float64
    wy, wl = ops.cross_attention_fwd(q.astype(f), kv.astype(f), klen, a)
    size, _ = ops.cross_attention_fwd(q.astype(f), np.abs(kv.astype(f)), klen, a)
    n = np.repeat(klen, a["Tq"])[:, None]
    top = np.abs(kv).max()
    # pieces of the values, instructions, the join's weights, quotient and products
    au.within("y", y, wy, (2 + 6 * np.ceil(n / 16) + 40) * au.U * size + 2.0 ** -39 * top)
    au.within("lse", lse, wl, (klen / 16 + 16)[:, None, None] * au.U + 4 * au.U * np.abs(wl))
    dq, dkv, _ = cross_bwd(a, q, kv, klen, y, lse, dy)
    _, wk, _ = ops.cross_attention_bwd(q.astype(f), kv.astype(f), klen, dy.astype(f), a)
    _, size, _ = ops.cross_attention_bwd(q.astype(f), kv.astype(f), klen, np.abs(dy.astype(f)), a)
    half = kv.shape[1] // 2
    rows = a["Tq"] * a["H"] // a["Hkv"]
    assert not dkv[:, :half].any()               # dk sums multiples of q
    # pieces of dy and of the probabilities, exp(-lse) with its argument's rounding, instructions, joins
    au.within("dv", dkv[:, half:], wk[:, half:],
              (2 + 2 + 4 + 40 + 8 * np.log(n.max()) + 6 * rows / 16) * au.U * size[:, half:]
              + rows * 2.0 ** -39 * np.abs(dy).max())


@pytest.mark.parametrize("outlier", [2.0 ** 17, 2.0 ** 24])
@pytest.mark.parametrize("kernel", KERNELS)
def test_a_large_column_of_values(kernel, outlier):
    """One head column far above the others: those lose what lies 2^-39 below it."""
    a, q, kv, klen, _ = uniform(kernel, seed=94)
    kv.reshape(a["B"], a["Tk"], 2, a["Hkv"], a["dh"])[:, :, 1, :, 5] *= np.float32(outlier)
    y, _ = cross_fwd(a, q, kv, klen)
    f = np.float64
    wy, _ = ops.cross_attention_fwd(q.astype(f), kv.astype(f), klen, a)
    size, _ = ops.cross_attention_fwd(q.astype(f), np.abs(kv.astype(f)), klen, a)
    n = np.repeat(klen, a["Tq"])[:, None]
    au.within("y", y, wy, (2 + 6 * np.ceil(n / 16) + 40) * au.U * size + 2.0 ** -39 * np.abs(kv).max())


@pytest.mark.parametrize("ratio", [14.0, 16.0, 18.3, 20.6, 22.7, 24.4])
@pytest.mark.parametrize("kernel", KERNELS)
def test_a_state_of_zeros_that_takes_the_weight(kernel, ratio):
    """State 0 has zero values and nearly all probability, every other 2^-ratio of it: y is what the
    others leave.  (All of one sign, as the pieces of equal probabilities err to one side.)"""
    B, Tq, Tk, H, Hkv, dh, _ = KERNELS[kernel]
    a, q, kv, klen, _ = au.cross_case(95, B, Tq, Tk, H, Hkv, dh, Tk)
    f = np.float64
    states = kv.reshape(B, Tk, 2, Hkv, dh)
    q[:] = 0
    q[:, ::dh] = 1
    states[:, :, 0] = 0
    states[:, 0, 0, :, 0] = ratio * np.log(2) * dh ** 0.5
    states[:, :, 1] = 1 + np.abs(states[:, :, 1])
    states[:, 0, 1] = 0
    y, _ = cross_fwd(a, q, kv, klen)
    wy, _ = ops.cross_attention_fwd(q.astype(f), kv.astype(f), klen, a)
    # the score's two pieces and three factors (5 u of it, a base-2 logarithm of `ratio`) and the sum
    # with the maximum (20 u), exp2 and sums, pieces, instructions, quotient and joins
    c = np.log(2) * (5 * ratio + 20) + 12 + 8 + 6 * np.ceil(Tk / 16) + 40
    au.within("y", y, wy, (c * au.U + 2.0 ** (ratio - 36)) * wy + 2.0 ** (-39 - ratio) * np.abs(kv).max())


@pytest.mark.parametrize("ratio", [6.0, 8.3, 10.6, 12.7, 14.4])
@pytest.mark.parametrize("kernel", KERNELS)
def test_a_query_without_gradient_that_takes_a_state(kernel, ratio):
    """Query 0 looks at state 1 alone and has a zero gradient: dv of state 1 is what the other queries
    leave, whose probabilities there are 2^-ratio / Tk or so."""
    B, Tq, Tk, H, Hkv, dh, _ = KERNELS[kernel]
    a, q, kv, klen, dy = au.cross_case(96, B, max(Tq, 2), Tk, H, Hkv, dh, Tk)
    f = np.float64
    q[:] = 0
    heads = q.reshape(B, -1, H, dh)
    heads[:, :, :, 0] = -1
    heads[:, 0, :, 0] = 40 / ratio
    kv.reshape(B, Tk, 2, Hkv, dh)[:, :, 0] = 0
    kv.reshape(B, Tk, 2, Hkv, dh)[:, 1, 0, :, 0] = ratio * np.log(2) * dh ** 0.5
    dy[:] = 1 + np.abs(dy)
    dy.reshape(B, -1, H, dh)[:, 0] = 0
    wy, wl = ops.cross_attention_fwd(q.astype(f), kv.astype(f), klen, a)
    _, wk, _ = ops.cross_attention_bwd(q.astype(f), kv.astype(f), klen, dy.astype(f), a)
    _, dkv, _ = cross_bwd(a, q, kv, klen, wy.astype(np.float32), wl.astype(np.float32), dy)
    got, want = (t.reshape(B, Tk, 2, -1)[:, 1, 1] for t in (dkv, wk))
    # score, lse and exp2 with their arguments' roundings, pieces, instructions, joins
    c = np.log(2) * (5 * ratio + 20) + 8 * np.log(Tk) + 8 + 6 * (a["Tq"] * H // Hkv) / 16 + 40
    lost = np.abs(dy).reshape(B, -1, Hkv, H // Hkv, dh).sum((1, 3)).reshape(B, -1) * 2.0 ** -35
    au.within("dv", got, want, c * au.U * want + lost)


#: factors of the keys, of the values (first 64 states, the others), of the queries and of their
#: gradients (first 64 positions, the others)
UNLIKE = [((2.0 ** -60, 2.0 ** 30), (1, 1), (2.0 ** -30, 2.0 ** -30), (1, 1)),
          ((2.0 ** 30, 2.0 ** -60), (1, 1), (2.0 ** -30, 2.0 ** -30), (1, 1)),
          ((1, 1), (2.0 ** -70, 2.0 ** 70), (1, 1), (2.0 ** -60, 2.0 ** -60)),
          ((1, 1), (2.0 ** 70, 2.0 ** -70), (1, 1), (2.0 ** -60, 2.0 ** -60)),
          ((1, 1), (1, 1), (1, 1), (2.0 ** -50, 2.0 ** 50)), ((1, 1), (1, 1), (1, 1), (2.0 ** 50, 2.0 ** -50)),
          ((1, 1), (1, 1), (1, 1), (0, 2.0 ** -80)), ((0, 1), (0, 1), (0, 1), (0, 1)),
          ((2.0 ** -90, 2.0 ** -95), (2.0 ** 80, 2.0 ** 90), (2.0 ** 85, 2.0 ** 95), (2.0 ** -90, 2.0 ** -80)),
          ((2.0 ** -40, 2.0 ** 40), (2.0 ** 40, 2.0 ** -40), (2.0 ** -40, 2.0 ** -100), (2.0 ** -40, 2.0 ** 40))]


@pytest.mark.parametrize("sizes", UNLIKE, ids=str)
@pytest.mark.parametrize("dh", [24, 64, 85, 200])
def test_whole_gradients_of_unlike_sizes(dh, sizes):
    """Every operand of unlike sizes along its rows, alike within the 64 that share a scale (from the first
    of a head or slice on): all gradients relative to what they sum."""
    a, q, kv, klen, dy = au.cross_case(97, 2, 150, 170, 4, 2, dh, [170, 90])
    states = kv.reshape(2, 170, 2, 2, dh)
    for part, t in ((slice(0, 64), 0), (slice(64, None), 1)):
        states[:, part, 0] *= np.float32(sizes[0][t])
        states[:, part, 1] *= np.float32(sizes[1][t])
        q.reshape(2, 150, -1)[:, part] *= np.float32(sizes[2][t])
        dy.reshape(2, 150, -1)[:, part] *= np.float32(sizes[3][t])
    check_cross(a, q, kv, klen, dy, slices=(None, (1, 1)))


@pytest.mark.parametrize("size", [12, 23, 26, 100])
@pytest.mark.parametrize("later", [2.0 ** -20, 2.0 ** 20])
@pytest.mark.parametrize("kernel", KERNELS)
def test_scores_of_any_size(kernel, later, size):
    """Scores that differ by 2^size / sqrt(dh) and more, to both sides of zero: each query has one state, or
    two of the same key in tiles whose values are unlike, and lse is its score."""
    a, q, kv, klen, _ = au.cross_case(98, *KERNELS[kernel])
    B, Tq, Tk, H, Hkv, dh = au.cross_shape(a)
    g = np.random.default_rng(99)
    rank = 1.0 + g.permutation(Tk)               # whole numbers: exact in one fp16 piece
    top, low = np.argmax(rank[:64]), np.argmin(rank[:64])
    rank[top], rank[low] = Tk + 1, 0.5
    rank[64 + 6], rank[64 + 7] = rank[top], rank[low]
    states = kv.reshape(B, Tk, 2, Hkv, dh)
    states[:, :, 0] = 0
    states[:, :, 0, :, 0] = (rank * 2.0 ** (size // 2))[None, :, None]
    states[:, 64:, 1] *= np.float32(later)
    q[:] = 0
    q.reshape(B, Tq, H, dh)[..., 0] = g.choice([-1.0, 1.0], (B, Tq, H)) * 2.0 ** (size - size // 2)
    y, lse = cross_fwd(a, q, kv, klen)
    f = np.float64
    wy, wl = ops.cross_attention_fwd(q.astype(f), kv.astype(f), klen, a)
    abs_v = kv.astype(f).copy()
    abs_v.reshape(states.shape)[:, :, 1] = np.abs(states[:, :, 1])
    weight, _ = ops.cross_attention_fwd(q.astype(f), abs_v, klen, a)
    # pieces, instructions and joins as in the means above; the score's scale is a product of three
    au.within("y", y, wy, (2 + 6 * np.ceil(Tk / 16) + 40) * au.U * weight + 2.0 ** -39 * np.abs(states[:, :, 1]).max())
    au.within("lse", lse, wl, 8 * au.U * np.abs(wl) + 16 * au.U)
