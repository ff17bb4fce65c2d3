"""Salts of dropout and joins in network descriptions."""

import pytest

from paper_2010_14109_amd import netdef
from test_decoder_ops_host import small_packed


def dropping(spec):
    return [L for L in spec["layers"] if L["op"] in ("dropout", "join")]


def salts(net):
    """(operation, salt) of every call that drops, forward and backward."""
    at = {"dropout": 2, "join_fwd": 4, "join_bwd": 4}
    return [(op, a[at[op]]) for op, a in zip(net.fn_ops, net.fn_attrs) if op in at]


def test_a_salt_left_out_twice_is_refused(lib):
    spec = small_packed()
    assert len(dropping(spec)) >= 4
    whole = salts(netdef.Net(spec))
    for L in dropping(spec)[1:3]:
        del L["salt"]
    with pytest.raises(ValueError, match="same words as"):
        netdef.Net(spec)
    dropping(spec)[2]["salt"] = 0               # the one the other has by default
    with pytest.raises(ValueError, match="same words as"):
        netdef.Net(spec)
    dropping(spec)[2]["salt"] = 77
    one = salts(netdef.Net(spec))               # one alone has salt 0
    assert len(one) == len(whole) and {s for _, s in one} >= {0, 77}


def test_seeds_keep_salts_apart(lib):
    spec = small_packed()
    for L in dropping(spec)[:2]:
        del L["salt"]
    dropping(spec)[1]["seed"] = "other"
    spec["inputs"].append({"name": "other", "shape": [2], "dtype": "i32"})
    netdef.Net(spec)


def test_the_same_salt_may_be_asked_for(lib):
    spec = small_packed()
    for L in dropping(spec):
        L["salt"] = 5
    assert {s for _, s in salts(netdef.Net(spec))} == {5}
    del dropping(spec)[-1]["salt"]              # another one than the others'
    netdef.Net(spec)


def test_layers_that_drop_nothing_need_none(lib):
    spec = small_packed(p=0.0)
    for L in dropping(spec):
        L.pop("salt", None)
    netdef.Net(spec)
