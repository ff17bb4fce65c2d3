"""Network descriptions whose tensors hold other numbers of sequences than the network's input."""

import numpy as np
import pytest

from paper_2010_14109_amd import netdef, synth
from test_attention_ops_host import small_seq2seq


def resized(spec, **shapes):
    return dict(spec, inputs=[dict(v, shape=shapes.get(v["name"], v["shape"])) for v in spec["inputs"]])


def test_a_source_of_other_sequences_is_refused(lib):
    """2 x 14 source tokens beside 4 x 5 target tokens: the rows divide by 4, the sequences do not."""
    spec = small_seq2seq(batch=4, layers=1)
    with pytest.raises(ValueError, match="sequences"):
        netdef.Net(resized(spec, src=[2, 14], src_pos=[28], src_len=[4]))
    netdef.Net(spec)


def test_rows_that_do_not_divide_into_the_sequences_are_refused(lib):
    """States given as an input of rows, for attention and for cross attention."""
    def net(rows, op):
        layers = [{"name": "e", "op": "embed", "in": ["x"], "vocab": 9, "d": 12},
                  {"name": "states", "op": "linear", "in": ["mem"], "in_features": 24, "out_features": 24},
                  {"name": "q", "op": "linear", "in": ["e"], "in_features": 12, "out_features": 12}]
        if op == "cross_attention":
            layers += [{"name": "a", "op": op, "in": ["q", "states"], "heads": 2, "kv_heads": 2, "klen": "n"}]
        else:
            layers += [{"name": "a", "op": op, "in": ["states"], "heads": 2, "causal": False}]
        layers += [{"name": "head", "op": "linear", "in": ["a"], "in_features": 12 if op != "attention" else 8,
                    "out_features": 9}]
        return netdef.Net({"name": "t", "input": [4, 5], "tokens": True, "classes": 9, "layers": layers,
                           "logits": "head", "init": "normal", "optimizer": {"lr": 0.1, "momentum": 0.0},
                           "inputs": [{"name": "mem", "shape": [rows, 24], "dtype": "f32"},
                                      {"name": "n", "shape": [4], "dtype": "i32"}]})
    for op in ("cross_attention", "attention"):
        net(28, op)
        with pytest.raises(ValueError, match="sequences"):
            net(27, op)


def test_inputs_without_a_meaning_are_refused():
    """Synthetic inputs follow names and types; one that fits none is not filled with guesses."""
    spec = small_seq2seq(layers=1)
    good = synth.make_extra_inputs(resized(spec))
    assert good["src"].dtype == np.int32
    for v in ({"name": "offsets", "shape": [3], "dtype": "i32"}, {"name": "mask", "shape": [3, 7], "dtype": "u8"},
              {"name": "other_len", "shape": [3], "dtype": "i32"}):
        with pytest.raises(ValueError, match=v["name"]):
            synth.make_extra_inputs(dict(spec, inputs=spec["inputs"] + [v]))
    states = synth.make_extra_inputs(dict(spec, inputs=spec["inputs"] + [
        {"name": "memory_in", "shape": [21, 6], "dtype": "f32"}]))["memory_in"]
    assert states.dtype == np.float32 and states.shape == (21, 6) and states.std() > 0.5
