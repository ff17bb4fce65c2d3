"""The tests on the device run every kernel of attend.hip and rope.hip's norms."""

import os
import re

import variants_util as vu
import test_gpu_attention_ops as gpu

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2010_14109_amd", "csrc")


def test_every_attention_kernel_is_run():
    run = {k for c in gpu.CROSS + vu.CROSS for k in vu.cross_kernels(*c)}
    assert run == vu.all_cross_kernels()


def test_every_norm_kernel_is_run():
    assert {vu.norm_kernel(*c) for c in gpu.QKNORM + vu.QKNORM} == vu.all_norm_kernels()


def test_the_rules_are_those_of_the_sources():
    """The numbers that variants_util repeats."""
    with open(os.path.join(CSRC, "attend.hip")) as f:
        text = f.read()
    assert f"kFewRows = {vu.FEW_ROWS};" in text
    assert "(halves % 2 == 0 || halves >= 10) && a.B * a.Hkv * ceil_div(halves, 2) >= 512" in text
    with open(os.path.join(CSRC, "rope.hip")) as f:
        text = f.read()
    rows = re.findall(r"q <= (\d+)\) CALL\(ODD, (\d+), (\d+)\)", text)
    assert [tuple(map(int, r)) for r in rows] == vu.GROUPS[:-1]
