"""The tests on the device run every kernel of span attention."""

import os

import pytest

import span_variants_util as sv
import test_gpu_span_attention as gpu
from variants_util import FEW_ROWS

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2010_14109_amd", "csrc")


def test_every_kernel_is_run():
    run = {k for c in gpu.SPAN + sv.SPAN for k in sv.span_kernels(*c)}
    assert run == sv.all_span_kernels() and len(run) == 84


@pytest.mark.parametrize("cap", [0, 3])
def test_the_wide_kernels_are_run_from_these_cases(cap):
    """At least two of them each with and without the bias, and with whole rounds and odd halves."""
    wide = [c for c in sv.SPAN if sv.span_kernels(*c)[0][0] == "wide" and (c[7] > 0) == (cap > 0)]
    assert {c[8] for c in wide} == {True, False} and len(wide) >= 4


def test_the_rules_are_those_of_the_sources():
    with open(os.path.join(CSRC, "attend.hip")) as f:
        text = f.read()
    assert f"kFewRows = {FEW_ROWS};" in text
    assert "return a.Tq * (a.H / a.Hkv) <= kFewRows && a.dh <= 128;" in text
    assert "if (spans && a.dh <= 64) return false;" in text
    assert "a.dh <= 128 && (halves % 2 == 0 || halves >= 10) && a.B * a.Hkv * ceil_div(halves, 2) >= 512" in text
