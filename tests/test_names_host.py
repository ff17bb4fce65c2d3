"""Network descriptions in which one name would stand for two tensors."""

import pytest

from paper_2010_14109_amd import netdef
from test_attention_ops_host import small_seq2seq


def test_an_input_named_like_any_tensor_is_refused(lib):
    """Parameters, statistics, gradients and the loss among them, whether or not the network names them."""
    spec = small_seq2seq(layers=1)
    for name in netdef.Net(spec, keep_grads=True).names:
        wrong = dict(spec, inputs=spec["inputs"] + [{"name": name, "shape": [4], "dtype": "i32"}])
        with pytest.raises(ValueError, match="two tensors"):
            netdef.Net(wrong, keep_grads=True)


def test_two_layers_of_one_name_are_refused(lib):
    spec = small_seq2seq(layers=1)
    again = [L for L in spec["layers"] if L["name"] == "e1.gelu"]
    with pytest.raises(ValueError, match="two tensors"):
        netdef.Net(dict(spec, layers=spec["layers"][:-1] + again + spec["layers"][-1:]))


def test_queries_and_states_of_one_tensor_are_refused(lib):
    """Their gradients would be one variable."""
    spec = small_seq2seq(layers=1, heads=4, kv_heads=2, seq=7, src_seq=7)
    for L in spec["layers"]:
        if L["op"] == "cross_attention":
            L["in"] = [L["in"][1]] * 2
    with pytest.raises(ValueError, match="two tensors"):
        netdef.Net(spec)
