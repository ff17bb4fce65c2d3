"""Dropout, block joins and gated recurrences without a GPU: the oracle's formulas against published
values, differences and plain loops, and everything the library refuses."""

import ctypes as C

import numpy as np
import pytest

import bench
import decoder_util as du
from oracle import ops
from oracle.lower import lower
from paper_2010_14109_amd import netdef, ooc, synth
from test_attention_ops_host import difference

R, W, RW = ooc.R, ooc.W, ooc.RW


# ---------------------------------------------------------------- the oracle's formulas
def test_the_generator_gives_its_published_words():
    """The known answers that were published with the generator, for three counters and keys."""
    full = 0xFFFFFFFF
    assert ops.philox([0], 0, [0, 0]).tolist() == [[0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]]
    assert ops.philox([full << 32 | full], full << 32 | full, [full, full]).tolist() == \
        [[0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]]
    assert ops.philox([0x85a308d3243f6a88], 0x0370734413198a2e, [0xa4093822, 0x299f31d0]).tolist() == \
        [[0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]]


def test_dropout_keeps_its_share():
    a = {"drop": int(0.1 * 2 ** 32), "salt": 1}
    m = ops.dropout_factor((1000, 400), [1, 2], a)
    kept = (m > 0).mean()
    assert abs(kept - 0.9) < 5 * np.sqrt(0.09 / m.size) and np.allclose(m[m > 0], 1 / 0.9, rtol=1e-9)
    assert (ops.dropout_factor((1000, 400), [1, 3], a) != m).mean() > 0.15


@pytest.mark.parametrize("groups,p,stream", [(1, 0.0, True), (3, 0.4, True), (2, 0.2, False)])
def test_join_gradients_against_differences(groups, p, stream):
    a, v = du.join_case(1, 6, 11, groups, p)
    f = {k: t.astype(np.float64) for k, t in v.items()}
    seed = v["seed"]
    if not stream:
        f["dh"] = np.zeros_like(f["dh"])

    def loss(**kw):
        t = dict(f, **kw)
        h, n, _ = ops.join_fwd(t["x"], t["f"], t["post"], t["gate"], t["pre"], t["scale"], a, seed)
        return (h * f["dh"]).sum() + (n * f["dn"]).sum()
    h = ops.join_fwd(f["x"], f["f"], f["post"], f["gate"], f["pre"], f["scale"], a, seed)[0]
    grads = ops.join_bwd(f["f"], h, f["post"], f["gate"], f["pre"], f["scale"],
                         f["dh"] if stream else None, f["dn"], a, seed)
    g = np.random.default_rng(2)
    for name, grad in zip(("x", "f", "post", "gate", "pre"), grads):
        d = g.standard_normal(f[name].shape)
        assert np.isclose(difference(lambda t: loss(**{name: t}), f[name], d), (grad * d).sum(),
                          rtol=1e-6, atol=1e-7), name


@pytest.mark.parametrize("carry,fresh", [(False, False), (True, True)])
def test_scan_against_plain_loops_and_differences(carry, fresh):
    a, fx, h0, fr, dh = du.scan_case(3, 2, 9, 4, carry, fresh)
    if fresh:
        fr[[3, 14]] = 1
    fx, dh = fx.astype(np.float64), dh.astype(np.float64)
    h0 = None if h0 is None else h0.astype(np.float64)
    h = ops.scan_fwd(fx, a, h0, fr)
    for b in range(2):
        for c in range(4):
            s = h0[b, c] if carry else 0.0
            for t in range(9):
                r = b * 9 + t
                if fresh and fr[r]:
                    s = 0.0
                gate = 1 / (1 + np.exp(-fx[r, c]))
                s = gate * s + (1 - gate) * fx[r, 4 + c]
                assert np.isclose(h[r, c], s, rtol=1e-12)
    dfx, dh0 = ops.scan_bwd(fx, h, dh, a, h0, fr)
    g = np.random.default_rng(4)
    d = g.standard_normal(fx.shape)
    num = difference(lambda t: (ops.scan_fwd(t, a, h0, fr) * dh).sum(), fx, d)
    assert np.isclose(num, (dfx * d).sum(), rtol=1e-7)
    if carry:
        d = g.standard_normal(h0.shape)
        num = difference(lambda t: (ops.scan_fwd(fx, a, t, fr) * dh).sum(), h0, d)
        assert np.isclose(num, (dh0 * d).sum(), rtol=1e-7)


def test_the_bounds_separate_planted_mistakes():
    """Planted in the oracle: a join without its 1e-5, a recurrence that misses one row."""
    a, v = du.join_case(5, 20, 64, 1, wide=True)
    h, n, _ = du.join_oracle(a, v)
    off = dict(v, f=v["f"] * np.float32(1 + 1e-4))
    bh, bn, _ = du.join_bounds(a, v)
    h1, n1, _ = du.join_oracle(a, off)
    assert (np.abs(h1 - h) > bh).any() and (np.abs(n1 - n) > bn).any()
    a, fx, h0, fr, dh = du.scan_case(6, 1, 50, 8, True, False)
    h = du.scan_oracle(a, fx, h0, fr)
    fx1 = fx.copy()
    fx1[20, 8:] = 0
    assert (np.abs(du.scan_oracle(a, fx1, h0, fr) - h) > du.scan_bound(a, fx, h0, fr)).any(1)[20:30].all()


# ---------------------------------------------------------------- what is refused
def refused(op, sizes, access, attrs, match):
    ctx = ooc.Context(-1)
    try:
        ids = [ctx.add_var(n, ooc.TEMP if a & W else ooc.INPUT) for n, a in zip(sizes, access)]
        with pytest.raises(ooc.OocError, match=match) as e:
            ctx.add_fn(op, ids, access, attrs)
        assert e.value.status == ooc.E_INVALID
    finally:
        ctx.close()


def accepted(op, sizes, access, attrs):
    ctx = ooc.Context(-1)
    try:
        ids = [ctx.add_var(n, ooc.TEMP if a & W else ooc.INPUT) for n, a in zip(sizes, access)]
        ctx.add_fn(op, ids, access, attrs)
    finally:
        ctx.close()


def vary(op, sizes, access, attrs, bad_attrs):
    """The call as given is taken; each size off by 4, each access, one variable fewer or more, one
    attribute fewer, and the attributes named are not."""
    accepted(op, sizes, access, attrs)
    for j in range(len(sizes)):
        refused(op, [s + 4 * (i == j) for i, s in enumerate(sizes)], access, attrs, op.upper())
        refused(op, sizes, [(R + W - s if i == j else s) for i, s in enumerate(access)], attrs, op.upper())
    refused(op, sizes[:-1], access[:-1], attrs, op.upper())
    refused(op, sizes + [16], access + [W], attrs, op.upper())
    refused(op, sizes, access, attrs[:-1], op.upper())
    for j, x in bad_attrs:
        refused(op, sizes, access, attrs[:j] + [x] + attrs[j + 1:], op.upper())


def test_dropout_refusals(lib):
    vary("dropout", [400, 8, 400], [R, R, W], [100, 7, 3],
         [(0, 0), (0, 101), (0, -1), (0, 1 << 40), (1, 1 << 32), (1, -1), (2, -1)])


@pytest.mark.parametrize("drop", [0, 9])
def test_join_refusals(lib, drop):
    x, v, g = 6 * 10 * 4, 40, 2 * 40
    seed = [8] if drop else []
    sizes = [x, x, v, g, v, 4] + seed + [x, x, 48]
    access = [R] * (6 + len(seed)) + [W] * 3
    bad = [(0, 0), (0, 7), (0, 1 << 23), (1, 0), (1, 8193), (2, 0), (2, 4), (2, 65534), (3, 1 << 32),
           (3, 0 if drop else 9), (4, -1)]
    vary("join_fwd", sizes, access, [6, 10, 2, drop, 3], bad)
    for stream in (0, 1):
        sizes = [x, x, 48, v, g, v, 4] + seed + [x] * stream + [x, x, x, v, g, v, 2 * 3 * 3 * 40]
        access = [R] * (8 + len(seed) + stream) + [W] * 6
        vary("join_bwd", sizes, access, [6, 10, 2, drop, 3, stream, 3],
             bad + [(5, 1 - stream), (5, 2), (6, 0), (6, 4)])


@pytest.mark.parametrize("carry,fresh,slices", [(0, 0, 1), (1, 1, 2), (1, 0, 1), (0, 1, 3)])
def test_scan_refusals(lib, carry, fresh, slices):
    h, st = 3 * 5 * 7 * 4, 3 * 7 * 4
    part = [3 * slices * 2 * 7 * 4] if slices > 1 else []
    ins = [2 * h] + [st] * carry + [60] * fresh
    bad = [(0, 0), (1, 0), (2, 0), (0, 4), (1, (1 << 28) + 1), (2, (1 << 24) + 1), (0, 1 << 24),
           (3, 1 - carry), (3, 2), (4, 1 - fresh), (4, 2), (5, 0), (5, 6), (5, 65)]
    attrs = [3, 5, 7, carry, fresh, slices]
    vary("scan_fwd", ins + [h] + part, [R] * len(ins) + [W] * (1 + len(part)), attrs, bad)
    outs = [2 * h] + [st] * carry + part
    vary("scan_bwd", ins + [h, h] + outs, [R] * (len(ins) + 2) + [W] * len(outs), attrs, bad)


def test_slice_counts(lib):
    assert ooc.join_slices(12288, 1024, 24) == (32, 24 * 32 * 3 * 1024 * 4)
    assert ooc.join_slices(1, 1, 1) == (1, 12) and ooc.join_slices(24, 5, 24)[0] == 1
    assert ooc.scan_slices("scan_fwd", [24, 512, 1024]) == (1, 0)
    assert ooc.scan_slices("scan_bwd", [1, 1, 1]) == (1, 0)
    s, part = ooc.scan_slices("scan_fwd", [1, 1 << 20, 64])
    assert 1 < s <= 64 and part == s * 2 * 64 * 4
    for rows, d, groups in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (6, 1, 4), (1 << 23, 1, 1), (1, 8193, 1)):
        with pytest.raises(ooc.OocError, match="ooc_join_slices"):
            ooc.join_slices(rows, d, groups)
    for op, a in (("scan_fwd", [0, 1, 1]), ("join_fwd", [1, 1, 1]), ("scan_bwd", [1, 1]),
                  ("scan_fwd", [1 << 23, 1, 1])):
        with pytest.raises(ooc.OocError, match="ooc_scan_slices"):
            ooc.scan_slices(op, a)
    n, b = C.c_int64(), C.c_uint64()
    a = (C.c_int64 * 3)(1, 1, 1)
    assert lib.ooc_join_slices(1, 1, 1, None, C.byref(b)) == ooc.E_INVALID
    assert lib.ooc_join_slices(1, 1, 1, C.byref(n), None) == ooc.E_INVALID
    assert lib.ooc_scan_slices(41, None, 3, C.byref(n), C.byref(b)) == ooc.E_INVALID
    assert lib.ooc_scan_slices(41, a, 3, None, C.byref(b)) == ooc.E_INVALID
    assert lib.ooc_scan_slices(41, a, 3, C.byref(n), None) == ooc.E_INVALID


# ---------------------------------------------------------------- span attention
@pytest.mark.parametrize("kind,cap,bias", [("causal", 0, False), ("any", 1.5, True), ("docs", 0, True),
                                           ("none", 2.0, False)])
def test_span_attention_against_plain_loops_and_differences(kind, cap, bias):
    a, q, kv, span, mod, dy = du.span_case(7, 2, 5, 7, 4, 2, 3, kind, cap, bias)
    q, kv, dy, mod = (t.astype(np.float64) for t in (q, kv, dy, mod))
    y, lse = ops.span_attention_fwd(q, kv, span, a, mod)
    for b in range(2):
        for h in range(4):
            for i in range(5):
                lo, hi, at = span[b * 5 + i]
                e = {}
                for j in range(max(lo, 0), min(hi, 7)):
                    s = q[b * 5 + i, 3 * h:3 * h + 3] @ kv[b * 7 + j, 3 * (h // 2):3 * (h // 2) + 3] / np.sqrt(3)
                    s = mod[0] * np.tanh(s / mod[0]) if cap else s
                    e[j] = np.exp(s - (mod[-4 + h] * abs(at - j) if bias else 0))
                want = sum((w * kv[b * 7 + j, 6 + 3 * (h // 2):9 + 3 * (h // 2)] for j, w in e.items()),
                           np.zeros(3)) / (sum(e.values()) or 1)
                assert np.allclose(y[b * 5 + i, 3 * h:3 * h + 3], want, rtol=1e-11, atol=1e-13)
                assert np.isclose(lse[b, h, i], np.log(sum(e.values())) if e else -np.inf)
    dq, dkv, delta = ops.span_attention_bwd(q, kv, span, dy, a, mod)
    assert np.allclose(delta.transpose(0, 2, 1).reshape(10, 4), (dy * y).reshape(10, 4, 3).sum(-1), atol=1e-13)
    g = np.random.default_rng(8)
    for _ in range(3):
        vq, vk = g.standard_normal(q.shape), g.standard_normal(kv.shape)
        num = difference(lambda t: (ops.span_attention_fwd(t, kv, span, a, mod)[0] * dy).sum(), q, vq)
        assert np.isclose(num, (dq * vq).sum(), rtol=1e-6, atol=1e-8)
        num = difference(lambda t: (ops.span_attention_fwd(q, t, span, a, mod)[0] * dy).sum(), kv, vk)
        assert np.isclose(num, (dkv * vk).sum(), rtol=1e-6, atol=1e-8)


def test_the_span_bounds_separate_planted_mistakes():
    """Planted in the oracle: a state more or fewer in each span, a cap and slopes 0.1 % off."""
    a, q, kv, span, mod, dy = du.span_case(9, 1, 60, 60, 2, 1, 16, "causal", 2.0, True)
    mod[1:] = 1 / 64      # far states count
    f = np.float64
    q64, kv64, d64 = q.astype(f), kv.astype(f), dy.astype(f)
    y, lse = ops.span_attention_fwd(q64, kv64, span, a, mod)
    dq, dkv, _ = ops.span_attention_bwd(q64, kv64, span, d64, a, mod)
    by, bl, bq, bk = du.span_bounds(q, kv, span, mod, dy, a)
    for other, m in ((span - [0, 1, 0], mod), (span + [1, 0, 0], mod), (span, mod * np.float32(1.001))):
        y1, l1 = ops.span_attention_fwd(q64, kv64, other, a, m)
        g1 = ops.span_attention_bwd(q64, kv64, other, d64, a, m)
        for got, want, bound in ((y1, y, by), (g1[0], dq, bq), (g1[1], dkv, bk)):
            assert (np.abs(got - want) > bound).mean() > 0.5


@pytest.mark.parametrize("cap,bias", [(0, 0), (1, 0), (0, 1), (1, 1)])
@pytest.mark.parametrize("slices", [(1, 1, 1), (2, 1, 3)], ids=str)
def test_span_attention_refusals(lib, cap, bias, slices):
    B, Tq, Tk, H, Hkv, dh = shape = [2, 5, 7, 4, 2, 8]
    q, kv, lse = B * Tq * H * dh * 4, B * Tk * 2 * Hkv * dh * 4, B * H * Tq * 4
    mod = [4 * (cap + bias * H)] if cap or bias else []
    sf, sq, sk = slices
    bad = [(0, 0), (1, 0), (2, 0), (3, 0), (4, 3), (5, 257), (6, 1 - cap), (6, 2), (7, 1 - bias), (7, 2), (8, 0), (8, 65)]
    if not (cap and bias):      # one flag for the other needs another mod
        bad = [(j, x) for j, x in bad if not (j in (6, 7) and x < 2 and not mod)]
    ins = [q, kv, B * Tq * 12] + mod
    part = [sf * (q + lse)] if sf > 1 else []
    vary("span_attention_fwd", ins + [q, lse] + part, [R] * len(ins) + [W] * (2 + len(part)),
         shape + [cap, bias, sf], bad + [(8, 8)])
    n = max(sq * q if sq > 1 else 0, sk * kv if sk > 1 else 0)
    outs = [q, kv, lse, B * 8] + ([n] if n else [])
    vary("span_attention_bwd", ins + [q, lse, q] + outs, [R] * (len(ins) + 3) + [W] * len(outs),
         shape + [cap, bias, sq, sk], bad + [(8, 8), (9, 0), (9, 11)])
    assert ooc.attention_slices("span_attention_fwd", shape) == ooc.attention_slices("cross_attention_fwd", shape)
    assert ooc.attention_slices("span_attention_bwd", shape) == ooc.attention_slices("cross_attention_bwd", shape)


# ---------------------------------------------------------------- networks
def small_packed(**kw):
    args = dict(batch=2, seq=11, d=24, heads=4, kv_heads=2, ffn=20, layers=2, vocab=13, p=0.2, cap=2.0)
    args.update(kw)
    return synth.packed(**args)


@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("kw", [{}, dict(p=0.0, cap=0.0, layers=3), dict(batch=1, seq=1), dict(batch=1, seq=700)],
                         ids=str)
def test_sequence_matches_the_oracle(lib, kw, keep):
    spec = small_packed(**kw)
    mine = netdef.Net(spec, keep_grads=keep)
    ref = lower(spec, keep_grads=keep, slices=mine.slices)
    assert mine.names == [v["name"] for v in ref["vars"]]
    assert mine.var_bytes == [v["bytes"] for v in ref["vars"]]
    assert mine.var_kinds == [v["kind"] for v in ref["vars"]]
    opname = {"add_fwd": "add", "add_grad": "add", "acc_grad": "acc"}
    assert mine.fn_ops == [opname.get(f["op"], f["op"]) for f in ref["fns"]]
    assert mine.fn_vars == [f["vars"] for f in ref["fns"]]
    ctx = ooc.Context(-1)
    mine.register(ctx)
    ctx.build_schedule()
    ctx.close()


def gated_and_carried():
    """A network with what ``packed`` leaves out: a gate from another layer, states handed in."""
    spec = small_packed(layers=1)
    for L in spec["layers"]:
        if L["op"] == "scan":
            L["state"] = "state"
        if L["name"] == "b1.join2":
            L["gate"] = "gates"
    i = next(i for i, L in enumerate(spec["layers"]) if L["name"] == "b1.join2")
    spec["layers"].insert(i, {"name": "gates", "op": "linear", "in": ["cond"], "in_features": 3,
                              "out_features": 24})
    spec["inputs"] += [{"name": "state", "shape": [2, 24], "dtype": "f32"},
                       {"name": "cond", "shape": [2, 3], "dtype": "f32"}]
    return spec


@pytest.mark.parametrize("build", [lambda: small_packed(), gated_and_carried], ids=["packed", "gated"])
def test_oracle_gradients_by_differences(lib, build):
    """The wiring: the loss's change along a direction of every parameter is the gradients'."""
    from oracle.interp import run
    spec = build()
    mine = netdef.Net(spec, keep_grads=True)
    reg = lower(spec, keep_grads=True, slices=mine.slices)
    assert mine.names == [v["name"] for v in reg["vars"]]
    x, labels = synth.make_inputs(spec, 0)
    extra = synth.make_extra_inputs(spec)
    g = np.random.default_rng(4)
    shapes = {n: mine.meta[n][0] for n in mine.param_names()}
    start = synth.make_params(spec, 1)
    assert {n: v.shape for n, v in start.items()} == shapes
    params = {n: start[n].astype(np.float64) + 0.3 * g.standard_normal(s) for n, s in shapes.items()}
    out = run(reg, x, labels, params, inputs=extra)
    for name in params:
        v = g.standard_normal(params[name].shape)

        def loss(t):
            return run(reg, x, labels, dict(params, **{name: params[name] + t * v}),
                       inputs=extra)["loss"][-1]
        num = (loss(1e-5) - loss(-1e-5)) / 2e-5
        assert np.isclose(num, (out["d:" + name] * v).sum(), rtol=1e-4, atol=1e-8), name


def test_wrong_descriptions_are_refused():
    def broken(change, inputs=None):
        spec = small_packed()
        for L in spec["layers"]:
            change(L)
        for v in spec["inputs"]:
            if inputs and v["name"] in inputs:
                v.update(inputs[v["name"]])
        return spec

    def of(op, **kw):
        return lambda L: L.update(kw) if L["op"] == op else None

    def nothing(L):
        pass
    for change, inputs, what in (
            (of("span_attention", span="fresh"), None, "must be an input"),
            (of("span_attention", span="embed"), None, "must be an input"),
            (of("span_attention", mod="scale"), None, "must be an input"),
            (of("span_attention", kv_heads=4), None, "widths"),
            (of("span_attention", cap=False), None, "must be an input"),
            (of("scan", fresh="span"), None, "must be an input"),
            (of("scan", state="mod"), None, "must be an input"),
            (of("dropout", p=1.0), None, "p must lie"), (of("dropout", p=-0.1), None, "p must lie"),
            (of("dropout", p=0.0), None, "nothing is dropped"),
            (of("dropout", seed="scale"), None, "must be an input"),
            (of("join", p=1.0), None, "p must lie"), (of("join", scale="mod"), None, "must be an input"),
            (of("join", gate="mod"), None, "gate"), (of("join", gate="b1.fx"), None, "gate"),
            (lambda L: L.update({"in": [L["in"][0], "b1.fx"]}) if L["op"] == "join" else None, None, "shape"),
            (nothing, {"seed": {"dtype": "f32"}}, "must be an input"),
            (nothing, {"fresh": {"shape": [21]}}, "must be an input"),
            (nothing, {"span": {"shape": [22, 2]}}, "must be an input")):
        with pytest.raises(ValueError, match=what):
            netdef.Net(broken(change, inputs))
    spec = small_packed(layers=1)
    spec["logits"] = "head2"
    spec["layers"].append({"name": "head2", "op": "linear", "in": ["b1.join2.h"], "in_features": 24,
                           "out_features": 13})
    with pytest.raises(ValueError, match="but its stream"):
        netdef.Net(spec)


def test_extra_inputs_and_the_benchmark_s_work(lib):
    spec = small_packed(batch=3, seq=40)
    e = synth.make_extra_inputs(spec)
    span, fresh = e["span"].reshape(3, 40, 3), e["fresh"].reshape(3, 40)
    assert fresh[:, 0].all() and 3 <= fresh.sum() <= 12
    for b in range(3):
        start = 0
        for t in range(40):
            start = t if fresh[b, t] else start
            assert span[b, t].tolist() == [start, t + 1, t]
    assert e["mod"][0] == 2 and len(e["mod"]) == 5 and (np.diff(e["mod"][1:]) < 0).all()
    assert e["seed"].dtype == np.int32 and e["scale"].tolist() == [1.0]
    net = netdef.Net(spec)
    table = bench.kernel_table(net, [1.0] * len(net.fn_ops), e)
    pairs = int((span[..., 1] - span[..., 0]).sum())
    assert table["span_attention_fwd"]["work"] == 4 * 4 * pairs * 6
    assert table["span_attention_bwd"]["work"] == 10 * 4 * pairs * 6
    rows = 120
    assert table["dropout"]["work"] == 4 * 8 * rows * 20 and table["join_fwd"]["work"] == 4 * 16 * rows * 24
    assert table["join_bwd"]["work"] == (3 * 24 + 20) * rows * 24
    assert table["scan_fwd"]["work"] == 12 * rows * 24 and table["scan_bwd"]["work"] == 24 * rows * 24
    assert "fp16" in bench.roofline(table["span_attention_bwd"], "span_attention_bwd")["peak_of"]
