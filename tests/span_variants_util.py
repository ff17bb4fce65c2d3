"""Which kernel of attend_kernels.h a span attention is given to, by the rules, and cases that together with
those of test_gpu_span_attention reach every one."""

from variants_util import FEW_ROWS, width


def span_kernels(B, Tq, Tk, H, Hkv, dh, kind, cap, bias):
    """(forward, dq, dkv) as (kernel, padded width, whether dh fills it, whether scores are capped)."""
    rows, d = Tq * (H // Hkv), width(dh)
    halves = -(-rows // 128)
    if rows <= FEW_ROWS and dh <= 128:
        fwd = "few"
    elif 64 < dh <= 128 and (halves % 2 == 0 or halves >= 10) and B * Hkv * -(-halves // 2) >= 512:
        fwd = "wide"
    else:
        fwd = "narrow"
    pair = "" if dh <= 64 else "_pair"
    return [(k, d, dh == d, cap > 0) for k in (fwd, "dq" + pair, "dkv" + pair)]


def all_span_kernels():
    widths = ({(k, d) for k in ("few", "narrow") for d in (32, 64, 96, 128)} | {("narrow", 256)}
              | {("wide", d) for d in (96, 128)} | {(k, d) for k in ("dq", "dkv") for d in (32, 64)}
              | {(k + "_pair", d) for k in ("dq", "dkv") for d in (96, 128, 256)})
    return {(k, d, exact, cap) for k, d in widths for exact in (True, False) for cap in (True, False)}


SPAN = [
    # B Tq Tk H Hkv dh kind cap bias
    # 256 columns a workgroup: one round of them, shared key heads, ten and more halves of 128 rows
    (16, 140, 140, 32, 32, 128, "docs", 3, False), (16, 130, 140, 32, 32, 128, "any", 0, True),
    (16, 140, 140, 32, 32, 96, "window", 4, True), (32, 129, 150, 16, 16, 96, "any", 0, False),
    (16, 140, 70, 32, 32, 85, "any", 2, True), (26, 330, 340, 16, 4, 72, "docs", 0, True),
    (16, 131, 131, 32, 32, 101, "prefix", 5, False), (52, 1217, 90, 2, 2, 119, "any", 0, False),
    # a few rows
    (3, 2, 300, 8, 4, 32, "any", 3, False), (3, 2, 300, 8, 4, 32, "any", 0, True), (2, 3, 200, 6, 2, 45, "any", 0, False),
    (2, 5, 130, 4, 2, 110, "any", 2, True), (2, 1, 1200, 6, 2, 119, "window", 0, True), (3, 4, 150, 3, 3, 80, "any", 4, False),
    (2, 2, 260, 12, 2, 96, "any", 0, True), (2, 7, 90, 2, 1, 96, "causal", 3, False),
    (2, 3, 400, 8, 4, 64, "window", 0, True), (1, 4, 513, 4, 1, 128, "any", 0, True),
    # the others
    (1, 200, 200, 2, 1, 96, "docs", 0, True), (2, 140, 150, 2, 2, 256, "any", 3, True),
    (2, 130, 130, 3, 1, 70, "any", 3, True), (1, 200, 230, 2, 2, 85, "docs", 2, False),
    (2, 150, 150, 4, 2, 101, "prefix", 0, True), (1, 257, 257, 3, 3, 127, "any", 4, True),
    (2, 140, 90, 2, 1, 110, "window", 3, False), (1, 333, 333, 2, 1, 97, "any", 0, False),
]
