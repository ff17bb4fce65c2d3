"""Which kernel of attend.hip and rope.hip a call is given to, by their rules, and cases that together
with those of test_gpu_attention_ops reach every one."""

FEW_ROWS = 16


def width(dh):
    return next(d for d in (32, 64, 96, 128, 256) if dh <= d)


def cross_kernels(B, Tq, Tk, H, Hkv, dh, *_):
    """(forward, dq, dkv) as (kernel, padded width, whether dh fills it)."""
    rows, d = Tq * (H // Hkv), width(dh)
    halves = -(-rows // 128)
    if rows <= FEW_ROWS and dh <= 128:
        fwd = "few"
    elif dh <= 128 and (halves % 2 == 0 or halves >= 10) and B * Hkv * -(-halves // 2) >= 512:
        fwd = "wide"
    else:
        fwd = "narrow"
    pair = "" if dh <= 64 else "_pair"
    return [(k, d, dh == d) for k in (fwd, "dq" + pair, "dkv" + pair)]


def all_cross_kernels():
    return ({(k, d, e) for k in ("few", "narrow", "wide") for d in (32, 64, 96, 128) for e in (True, False)}
            | {("narrow", 256, e) for e in (True, False)}
            | {(k, d, e) for k in ("dq", "dkv") for d in (32, 64) for e in (True, False)}
            | {(k + "_pair", d, e) for k in ("dq", "dkv") for d in (96, 128, 256) for e in (True, False)})


#: (fours of columns at most, lanes a head, fours a lane)
GROUPS = [(8, 8, 1), (16, 16, 1), (24, 8, 3), (32, 32, 1), (48, 16, 3), (64, 64, 1), (96, 32, 3),
          (128, 64, 2), (192, 64, 3), (256, 64, 4)]


def norm_kernel(rows, h1, h2, dh, rot, layout, rest, *_):
    """(odd, lanes a head, fours a lane) of both directions."""
    cols = (h1 + h2) * dh + rest
    odd = bool(dh % 4 or cols % 4 or rot % (8 if layout else 4))
    return (odd,) + next((g, k) for most, g, k in GROUPS if (dh + 3) // 4 <= most)


def all_norm_kernels():
    return {(odd, g, k) for odd in (False, True) for _, g, k in GROUPS}


CROSS = [
    # B Tq Tk H Hkv dh klen
    (32, 129, 70, 16, 16, 24, None), (32, 200, 90, 16, 16, 32, None), (32, 130, 100, 16, 16, 40, None),
    (32, 256, 64, 16, 16, 64, None), (16, 140, 65, 32, 32, 85, None), (32, 129, 77, 16, 16, 96, None),
    (16, 131, 70, 32, 32, 101, None), (32, 150, 97, 16, 16, 128, None),
    # shared key heads, ten and more halves of 128 rows, an odd count among them
    (26, 330, 75, 16, 4, 64, None), (52, 1217, 33, 2, 2, 48, None),
    # a few queries, and the widths from 97 to 127 of every kernel
    (3, 2, 300, 8, 4, 32, [300, 0, 77]), (2, 1, 200, 6, 2, 96, [200, 65]), (2, 5, 130, 4, 2, 110, [130, 64]),
    (2, 90, 130, 2, 1, 127, [130, 1]), (1, 300, 300, 2, 2, 97, 299), (2, 40, 33, 3, 3, 119, [33, 0]),
]

QKNORM = [
    # rows h1 h2 dh rot layout rest far
    (37, 3, 2, 101, 100, 1, 5, True), (30, 2, 1, 127, 42, 0, 127, False), (22, 2, 1, 160, 80, 1, 160, True),
    (40, 1, 1, 200, 0, 1, 0, False), (15, 2, 1, 253, 252, 0, 3, True), (19, 2, 2, 256, 18, 1, 0, False),
    (11, 1, 2, 400, 200, 1, 8, True), (9, 1, 1, 398, 398, 1, 2, False), (13, 1, 1, 384, 64, 0, 0, False),
    (12, 2, 0, 510, 34, 1, 6, True), (10, 1, 1, 512, 512, 0, 4, True), (8, 1, 1, 600, 120, 1, 0, False),
    (7, 1, 1, 767, 766, 1, 1, True), (9, 2, 1, 768, 32, 0, 768, True), (16, 2, 1, 170, 84, 0, 1, False),
    (18, 1, 1, 24, 8, 1, 8, True), (300, 4, 4, 128, 128, 1, 0, True),
]
