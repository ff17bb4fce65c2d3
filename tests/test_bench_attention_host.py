"""``bench.py``'s figures of the attention-side operators (no GPU)."""


import bench
from paper_2010_14109_amd import netdef, synth
from test_attention_ops_host import small_seq2seq


def test_padding_is_not_work(lib):
    """A step's cross attention is credited with the states that its sequences have."""
    spec = small_seq2seq(layers=1)
    net = netdef.Net(spec)
    extra = synth.make_extra_inputs(spec)
    assert extra["src_len"].sum() < 3 * 7
    table = bench.kernel_table(net, [1.0] * len(net.fn_ops), extra)
    d, seq = 24, 5                     # all heads' columns, positions of a sequence
    for op, products in (("cross_attention_fwd", 2), ("cross_attention_bwd", 5)):
        assert table[op]["work"] == products * 2 * d * seq * int(extra["src_len"].sum())
    assert bench.fn_work("cross_attention_fwd", [2, 3, 5, 4, 2, 8, 1], 6) == ("flop", 2 * 2 * 4 * 3 * 6 * 8)


def test_roof_of_fp16_pieces():
    """Cross attention runs three fp16 products for each fp32 product, everything else six bf16 ones."""
    dom = {"unit": "flop", "rate": 200.0}
    r = bench.roofline(dom, "cross_attention_bwd")
    assert r["peak"] == round(2500 / 3, 1) and "3 fp16" in r["peak_of"] and r["frac"] == round(600 / 2500, 4)
    for op in ("conv_fwd", "attention_bwd", "linear_bwd_w"):
        assert bench.roofline(dom, op) == bench.roofline(dom)


def test_partial_results_are_not_algorithmic(lib):
    """Neither direction's partial results (``.part``, ``.bpart``) count as compulsory bytes."""
    net = netdef.Net(small_seq2seq(batch=1, src_seq=700, seq=300, layers=1))
    sizes = dict(zip(net.names, net.var_bytes))
    assert any(n.endswith("cross.part") for n in sizes) and any(n.endswith("cross.bpart") for n in sizes)
    q, kv, y = sizes["d1.qn"], sizes["d1.kn"], sizes["d1.cross"]
    lse = sizes["d1.cross.lse"]
    assert bench.algorithmic_bytes(net, "cross_attention_fwd") == q + kv + y + 4 + lse
    # q, kv, lengths, y, lse, dy read; dq, dkv and delta written
    assert bench.algorithmic_bytes(net, "cross_attention_bwd") == 4 * q + 2 * kv + 4 + 2 * lse
