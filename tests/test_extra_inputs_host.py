"""Synthetic inputs are made by what layers take them for, not by what they are called."""

import numpy as np
import pytest

from paper_2010_14109_amd import synth
from test_decoder_ops_host import small_packed


def renamed(spec, names):
    for L in spec["layers"]:
        for key in ("span", "mod", "fresh", "seed", "scale"):
            if L.get(key) in names:
                L[key] = names[L[key]]
    for v in spec["inputs"]:
        v["name"] = names.get(v["name"], v["name"])
    return spec


def test_names_do_not_matter():
    names = {"span": "a", "mod": "b", "fresh": "c", "seed": "d", "scale": "e"}
    want = synth.make_extra_inputs(small_packed())
    got = synth.make_extra_inputs(renamed(small_packed(), names))
    assert set(got) == set(names.values())
    for n, m in names.items():
        assert got[m].dtype == want[n].dtype and np.array_equal(got[m], want[n]), n


def test_inputs_that_no_such_layer_takes_are_as_ever():
    """f32 standard normal, i32 of two axes tokens, whatever they are called; others are refused."""
    spec = small_packed()
    plain = dict(spec, layers=[], inputs=[
        {"name": "my_mod", "shape": [6], "dtype": "f32"}, {"name": "scale", "shape": [1], "dtype": "f32"},
        {"name": "makespan", "shape": [22, 3], "dtype": "i32"}])
    g = np.random.Generator(np.random.PCG64(2))
    e = synth.make_extra_inputs(plain)
    assert np.array_equal(e["my_mod"], g.standard_normal(6, np.float32))
    assert np.array_equal(e["scale"], g.standard_normal(1, np.float32))
    assert np.array_equal(e["makespan"], g.integers(0, 13, (22, 3)).astype(np.int32))
    for v in ({"name": "seed", "shape": [2], "dtype": "i32"}, {"name": "fresh", "shape": [22], "dtype": "i32"}):
        with pytest.raises(ValueError, match="no synthetic values"):
            synth.make_extra_inputs(dict(plain, inputs=[v]))


def test_a_layer_without_a_cap_has_slopes_alone():
    spec = small_packed()
    first = next(L for L in spec["layers"] if L["op"] == "span_attention")
    second = dict(first, name="again", cap=False, mod="slopes")
    spec["layers"].append(second)
    spec["inputs"].append({"name": "slopes", "shape": [4], "dtype": "f32"})
    e = synth.make_extra_inputs(spec)
    assert e["mod"][0] == 2 and np.array_equal(e["slopes"], e["mod"][1:])
