"""Rotation, per-head norms and cross attention without a GPU: the oracle's formulas against
differences and plain loops, the product's sequence against the oracle's, and everything the
library refuses."""

import ctypes as C

import numpy as np
import pytest

import attention_util as au
import bench
from oracle import ops
from oracle import schedule as S
from oracle.lower import lower
from paper_2010_14109_amd import netdef, ooc, synth

R, W, RW = ooc.R, ooc.W, ooc.RW


def small_seq2seq(**kw):
    args = dict(batch=3, src_seq=7, seq=5, d=24, heads=4, kv_heads=2, ffn=20, layers=2, vocab=11)
    args.update(kw)
    return synth.seq2seq(**args)


def difference(f, x, direction, step=1e-6):
    return (f(x + step * direction) - f(x - step * direction)) / (2 * step)


# ---------------------------------------------------------------- the oracle's formulas
@pytest.mark.parametrize("layout", [0, 1])
def test_rotation_against_plain_loops(layout):
    a, x, pos, table = au.rope_case(1, 5, 3, 10, 6, layout, 4, True)
    y = ops.rope(x.astype(np.float64), pos, table, a)
    for r in range(5):
        for h in range(3):
            for d in range(10):
                if d >= 6:
                    assert y[r, h * 10 + d] == x[r, h * 10 + d]
                    continue
                i, second = (d // 2, d % 2) if layout == 0 else (d % 3, d // 3)
                ang = float(pos[r]) * table[i]
                p0, p1 = (2 * i, 2 * i + 1) if layout == 0 else (i, i + 3)
                x0, x1 = float(x[r, h * 10 + p0]), float(x[r, h * 10 + p1])
                want = x0 * np.sin(ang) + x1 * np.cos(ang) if second else \
                    x0 * np.cos(ang) - x1 * np.sin(ang)
                assert abs(y[r, h * 10 + d] - table[-1] * want) < 1e-9
    assert np.array_equal(y[:, 30:], x[:, 30:])
    # the backward is the transposed map: <y, g> = <x, back(g)>
    g = np.random.default_rng(2).standard_normal(y.shape)
    assert np.isclose((y * g).sum(), (x * ops.rope(g, pos, table, a, back=True)).sum(), rtol=1e-12)


@pytest.mark.parametrize("h2,rot", [(2, 6), (0, 0), (1, 10)])
def test_norm_gradients_against_differences(h2, rot):
    a, x, gain, where, dy = au.qknorm_case(3, 4, 3, h2, 10, rot, 1, 3, False)
    x, gain, dy = x.astype(np.float64), gain.astype(np.float64), dy.astype(np.float64)
    y = ops.qknorm_fwd(x, gain, *where, a=a)
    if not rot:
        h = y[:, :(3 + h2) * 10].reshape(4, -1, 10) / ops._head_gain(gain, a)
        ms = (x[:, :(3 + h2) * 10].reshape(4, -1, 10) ** 2).mean(-1)
        assert np.allclose((h ** 2).mean(-1), ms / (ms + 1e-5), rtol=1e-12)
    dx, dgain = ops.qknorm_bwd(x, gain, dy, *where, a=a)
    g = np.random.default_rng(5)
    for _ in range(4):
        vx, vg = g.standard_normal(x.shape) * np.abs(x), g.standard_normal(gain.shape)
        num = difference(lambda t: (ops.qknorm_fwd(t, gain, *where, a=a) * dy).sum(), x, vx)
        assert np.isclose(num, (dx * vx).sum(), rtol=1e-5, atol=1e-5)
        num = difference(lambda t: (ops.qknorm_fwd(x, t, *where, a=a) * dy).sum(), gain, vg)
        assert np.isclose(num, (dgain * vg).sum(), rtol=1e-6, atol=1e-6)


def test_cross_attention_against_plain_loops_and_differences():
    a, q, kv, klen, dy = au.cross_case(7, 3, 4, 5, 4, 2, 3, [5, 0, 2])
    q, kv, dy = q.astype(np.float64), kv.astype(np.float64), dy.astype(np.float64)
    y, lse = ops.cross_attention_fwd(q, kv, klen, a)
    for b in range(3):
        for h in range(4):
            for i in range(4):
                qr = q[b * 4 + i, h * 3:h * 3 + 3]
                e = [np.exp(qr @ kv[b * 5 + j, h // 2 * 3:h // 2 * 3 + 3] / np.sqrt(3))
                     for j in range(klen[b])]
                want = sum((w * kv[b * 5 + j, 6 + h // 2 * 3:9 + h // 2 * 3]
                            for j, w in enumerate(e)), np.zeros(3)) / (sum(e) or 1)
                assert np.allclose(y[b * 4 + i, h * 3:h * 3 + 3], want, rtol=1e-12, atol=1e-14)
                assert np.isclose(lse[b, h, i], np.log(sum(e)) if e else -np.inf)
    dq, dkv, delta = ops.cross_attention_bwd(q, kv, klen, dy, a)
    assert np.allclose(delta.transpose(0, 2, 1).reshape(12, 4),
                       (dy * y).reshape(12, 4, 3).sum(-1), atol=1e-13)
    assert not dkv[5:10].any() and not dkv[12:].any() and not dq[4:8].any()
    g = np.random.default_rng(8)
    for _ in range(4):
        vq, vk = g.standard_normal(q.shape), g.standard_normal(kv.shape)
        num = difference(lambda t: (ops.cross_attention_fwd(t, kv, klen, a)[0] * dy).sum(), q, vq)
        assert np.isclose(num, (dq * vq).sum(), rtol=1e-6, atol=1e-8)
        num = difference(lambda t: (ops.cross_attention_fwd(q, t, klen, a)[0] * dy).sum(), kv, vk)
        assert np.isclose(num, (dkv * vk).sum(), rtol=1e-6, atol=1e-8)


def test_the_bounds_separate_a_dropped_state():
    """Planted in the oracle: attention over one state fewer is out of every bound."""
    a, q, kv, klen, dy = au.cross_case(9, 1, 8, 60, 2, 1, 16, 60)
    f = np.float64
    y, lse = ops.cross_attention_fwd(q.astype(f), kv.astype(f), klen, a)
    ey, el, eq, ek = au.cross_bounds(q, kv, klen, dy, a)
    y1, l1 = ops.cross_attention_fwd(q.astype(f), kv.astype(f), klen - 1, a)
    assert (np.abs(y - y1) > ey).mean() > 0.9 and (np.abs(lse - l1) > el).mean() > 0.9
    dq, dkv, _ = ops.cross_attention_bwd(q.astype(f), kv.astype(f), klen, dy.astype(f), a)
    dq1, dkv1, _ = ops.cross_attention_bwd(q.astype(f), kv.astype(f), klen - 1, dy.astype(f), a)
    assert (np.abs(dq - dq1) > eq).mean() > 0.9 and (np.abs(dkv - dkv1) > ek).mean() > 0.9


def test_rotary_table():
    t = netdef.rotary_table(8)
    assert np.allclose(t, [1, 0.1, 0.01, 0.001, 1.0])
    assert np.allclose(netdef.rotary_table(8, base=100.0, scale=4.0),
                       [0.25, 0.25 * 100 ** -0.25, 0.025, 0.25 * 100 ** -0.75, 1.0])
    t = netdef.rotary_table(64, scale=16.0, trained=4096)
    plain = netdef.rotary_table(64)
    turns = 4096 * np.array(plain[:-1]) / (2 * np.pi)
    ratio = np.array(t[:-1]) / plain[:-1]
    assert np.allclose(ratio[turns >= 32], 1) and np.allclose(ratio[turns <= 1], 1 / 16)
    mid = (turns > 1) & (turns < 32)
    assert mid.any() and (ratio[mid] > 1 / 16).all() and (ratio[mid] < 1).all()
    assert np.isclose(t[-1], 1 + 0.1 * np.log(16))
    for bad in (dict(rot=0), dict(rot=3), dict(rot=4, scale=0.5), dict(rot=4, base=0.0),
                dict(rot=4, trained=0), dict(rot=4, turns=(2, 1))):
        with pytest.raises(ValueError):
            netdef.rotary_table(**bad)


# ---------------------------------------------------------------- the function sequence
@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("kw", [{}, dict(d=20, kv_heads=1, layers=1), dict(batch=1, seq=1, src_seq=300)],
                         ids=str)
def test_sequence_matches_the_oracle(lib, kw, keep):
    spec = small_seq2seq(**kw)
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
    b, k, f = mine.var_bytes, mine.var_kinds, mine.fn_vars
    chunk = 4096
    B = max(S.budget_for(0.4, S.incore_peak(b, k, f, chunk), chunk), S.working_set_max(b, f, chunk))
    ctx.set_chunk(chunk)
    ctx.set_budget(B)
    ctx.build_schedule()
    assert ctx.stats()["peak_accounted"] <= B
    ctx.close()


def test_seq2seq_oracle_gradients_by_differences(lib):
    """The wiring: the loss's change along a direction of every parameter is the gradients'."""
    from oracle.interp import run
    spec = small_seq2seq(layers=1)
    reg = lower(spec, keep_grads=True)
    x, labels = synth.make_inputs(spec, 0)
    tables = {"table": netdef.rotary_table(6), "src_table": netdef.rotary_table(2)}
    extra = synth.make_extra_inputs(spec, tables)
    g = np.random.default_rng(4)
    params = {n: v.astype(np.float64) + 0.3 * g.standard_normal(v.shape)
              for n, v in synth.make_params(spec, 1).items()}
    out = run(reg, x, labels, params, inputs=extra)
    for name in params:
        v = g.standard_normal(params[name].shape)

        def loss(t):
            return run(reg, x, labels, dict(params, **{name: params[name] + t * v}),
                       inputs=extra)["loss"][-1]
        num = (loss(1e-5) - loss(-1e-5)) / 2e-5
        assert np.isclose(num, (out["d:" + name] * v).sum(), rtol=1e-4, atol=1e-8), name


def test_wrong_descriptions_are_refused():
    def broken(change):
        spec = small_seq2seq(layers=1)
        for L in spec["layers"]:
            change(L)
        return spec
    for change, what in (
            (lambda L: L.update(pos="src_len") if L["op"] == "rope" else None, "must be an input"),
            (lambda L: L.update(table="src_table") if L["op"] == "qknorm" else None, "must be an input"),
            (lambda L: L.update(klen="src_pos") if L["op"] == "cross_attention" else None, "length"),
            (lambda L: L.update(klen="memory") if L["op"] == "cross_attention" else None, "length"),
            (lambda L: L.update(kv_heads=4) if L["op"] == "cross_attention" else None, "widths")):
        with pytest.raises(ValueError, match=what):
            netdef.Net(broken(change))


def test_lengths_that_are_not_integers_are_refused():
    spec = small_seq2seq(layers=1)
    spec["inputs"] = [dict(v, dtype="f32") if v["name"] == "src_len" else v for v in spec["inputs"]]
    with pytest.raises(ValueError, match="length"):
        netdef.Net(spec)


# ---------------------------------------------------------------- refusals of the library
def add(op, sizes, access, attrs, kinds=None):
    """add_fn on a host context; the error message, or ''."""
    ctx = ooc.Context(-1)
    try:
        ids = [ctx.add_var(max(1, s), ooc.STATE) for s in sizes]
        ctx.add_fn(op, ids, access, attrs)
    except ooc.OocError as e:
        assert e.status == ooc.E_INVALID
        return e.message
    finally:
        ctx.close()
    return ""


def rope_sizes(rows, cols, heads, dh, rot, layout):
    return [rows * cols * 4, rows * 4, (rot // 2 + 1) * 8, rows * cols * 4]


def qknorm_sizes(rows, cols, h1, h2, dh, rot, layout, slices=None):
    x, g = rows * cols * 4, (2 if h2 else 1) * dh * 4
    where = [rows * 4, (rot // 2 + 1) * 8] if rot else []
    return [x, g] + where + ([x] if slices is None else [x, x, g, slices * g])


def cross_sizes(B, Tq, Tk, H, Hkv, dh, *slices):
    q, kv, l = B * Tq * H * dh * 4, B * Tk * 2 * Hkv * dh * 4, B * H * Tq * 4
    if len(slices) == 1:
        return [q, kv, B * 4, q, l] + ([slices[0] * (q + l)] if slices[0] > 1 else [])
    part = max(slices[0] * q if slices[0] > 1 else 0, slices[1] * kv if slices[1] > 1 else 0)
    return [q, kv, B * 4, q, l, q, q, kv, l] + ([part] if part else [])


ACCESS = {
    "rope_fwd": [R, R, R, W], "rope_bwd": [R, R, R, W],
    "qknorm_fwd": [R, R, R, R, W], "qknorm_bwd": [R, R, R, R, R, W, W, W],
    "cross_attention_fwd": [R, R, R, W, W, W],
    "cross_attention_bwd": [R, R, R, R, R, R, W, W, W, W],
}
GOOD = [
    ("rope_fwd", [3, 50, 2, 20, 10, 1]), ("rope_bwd", [1, 2, 1, 2, 2, 0]),
    ("qknorm_fwd", [3, 50, 2, 1, 10, 6, 1]), ("qknorm_bwd", [9, 50, 2, 1, 10, 6, 1, 4]),
    ("cross_attention_fwd", [2, 3, 70, 4, 2, 10, 5]),
    ("cross_attention_bwd", [2, 3, 70, 4, 2, 10, 5, 2]),
]
SIZES = {"rope": rope_sizes, "qknorm": qknorm_sizes, "cross": cross_sizes}


def sizes_of(op, attrs):
    return SIZES[op.split("_")[0]](*attrs)


@pytest.mark.parametrize("op,attrs", GOOD, ids=lambda v: str(v))
def test_signatures(lib, op, attrs):
    sizes, access = sizes_of(op, attrs), ACCESS[op]
    assert add(op, sizes, access, attrs) == ""
    for j in range(len(sizes)):
        off = list(sizes)
        off[j] += 4
        assert "bytes, attributes imply" in add(op, off, access, attrs), j
        wrong = list(access)
        wrong[j] = RW
        assert "access" in add(op, sizes, wrong, attrs), j
    assert add(op, sizes[:-1], access[:-1], attrs) != ""
    assert add(op, sizes + [4], access + [W], attrs) != ""
    assert "attributes" in add(op, sizes, access, attrs[:-1])
    assert "attributes" in add(op, sizes, access, attrs + [1])
    for j in range(len(attrs)):
        for v in (-1, 1 << 41):
            bad = list(attrs)
            bad[j] = v
            assert add(op, sizes, access, bad) != "", (j, v)


@pytest.mark.parametrize("op,attrs", [
    ("rope_fwd", [3, 50, 2, 20, 9, 1]), ("rope_fwd", [3, 50, 2, 20, 0, 1]),
    ("rope_fwd", [3, 50, 2, 20, 22, 1]), ("rope_fwd", [3, 50, 2, 20, 10, 2]),
    ("rope_fwd", [3, 39, 2, 20, 10, 1]), ("rope_fwd", [0, 50, 2, 20, 10, 1]),
    ("rope_fwd", [3, 50, 0, 20, 10, 1]), ("rope_fwd", [3, 5000, 1, 5000, 1026, 1]),
    ("rope_fwd", [1 << 31, 2, 1, 2, 2, 0]), ("rope_fwd", [1, 1 << 30, 1, 2, 2, 0]),
    ("rope_fwd", [3, 50, 1 << 39, 1 << 39, 2, 0]),
    ("rope_bwd", [1 << 27, 2, 1, 2, 2, 0]), ("qknorm_fwd", [1 << 27, 2, 1, 0, 2, 0, 0]),
    ("qknorm_fwd", [3, 50, 2, -1, 10, 6, 1]), ("qknorm_fwd", [3, 50, 2, 1, 10, -2, 1]),
    ("qknorm_bwd", [9, 50, 2, 1, 10, -4, 1, 2]), ("qknorm_fwd", [3, 50, 1 << 62, 1 << 62, 10, 6, 1]),
    ("qknorm_fwd", [3, 50, 0, 1, 10, 6, 1]), ("qknorm_fwd", [3, 50, 2, 1, 10, 5, 1]),
    ("qknorm_fwd", [3, 2050, 1, 1, 1025, 6, 1]), ("qknorm_fwd", [3, 29, 2, 1, 10, 6, 1]),
    ("qknorm_fwd", [3, 50, 2, 1, 10, 12, 1]), ("qknorm_fwd", [3, 50, 2, 1, 10, 6, 3]),
    ("qknorm_bwd", [9, 50, 2, 1, 10, 6, 1, 0]), ("qknorm_bwd", [9, 50, 2, 1, 10, 6, 1, 10]),
    ("cross_attention_fwd", [2, 3, 70, 4, 3, 10, 1]), ("cross_attention_fwd", [2, 3, 70, 4, 2, 257, 1]),
    ("cross_attention_fwd", [2, 3, 70, 4, 2, 10, 0]), ("cross_attention_fwd", [2, 3, 70, 4, 2, 10, 65]),
    ("cross_attention_fwd", [2, 3, 4, 4, 2, 10, 5]), ("cross_attention_fwd", [2, 0, 70, 4, 2, 10, 1]),
    ("cross_attention_fwd", [2, 3, 0, 4, 2, 10, 1]), ("cross_attention_fwd", [0, 3, 70, 4, 2, 10, 1]),
    ("cross_attention_fwd", [1 << 25, 1, 1, 1, 1, 1, 1]),
    ("cross_attention_fwd", [1, 1, 1 << 29, 1, 1, 1, 1]),
    ("cross_attention_fwd", [1 << 12, 1 << 28, 1 << 28, 16, 16, 256, 1]),
    ("cross_attention_fwd", [1 << 16, 1 << 14, 64, 8, 8, 16, 1]),
    ("cross_attention_bwd", [1 << 16, 1, 1 << 14, 8, 8, 200, 1, 1]),
    ("cross_attention_bwd", [2, 3, 70, 4, 2, 10, 5, 7]), ("cross_attention_bwd", [2, 3, 70, 4, 2, 10, 5, 0]),
], ids=lambda v: str(v))
def test_attributes_out_of_their_ranges(lib, op, attrs):
    sizes = [min(max(1, s), 1 << 50) for s in sizes_of(op, attrs)]
    access = ACCESS[op]
    if op.startswith("qknorm") and attrs[5] == 0:
        access = access[:2] + access[4:]
    if op.startswith("cross"):
        access = access[:len(sizes)]
    msg = add(op, sizes, access, attrs)
    assert msg.startswith(op.upper()) and "imply" not in msg, msg


def test_norm_without_rotation_takes_no_positions(lib):
    attrs = [3, 50, 2, 1, 10, 0, 1]
    assert add("qknorm_fwd", qknorm_sizes(*attrs), [R, R, W], attrs) == ""
    assert "iff rot > 0" in add("qknorm_fwd", qknorm_sizes(3, 50, 2, 1, 10, 6, 1), ACCESS["qknorm_fwd"],
                                attrs)


def test_slice_counts(lib):
    assert [ooc.qknorm_slices(n) for n in (1, 8, 9, 16384, 1 << 30)] == [1, 1, 2, 2048, 2048]
    with pytest.raises(ooc.OocError):
        ooc.qknorm_slices(0)
    g = np.random.default_rng(1)
    for _ in range(300):
        hkv = int(g.integers(1, 9))
        a = [int(2 ** g.uniform(0, 6)), int(2 ** g.uniform(0, 13)), int(2 ** g.uniform(0, 15)),
             hkv * int(g.integers(1, 9)), hkv, int(g.integers(1, 257))]
        for op in ("cross_attention_fwd", "cross_attention_bwd"):
            slices, part = ooc.attention_slices(op, a)
            sizes = cross_sizes(*a, *slices)
            assert part == (sizes[-1] if any(s > 1 for s in slices) else 0)
            n = (5 if op.endswith("fwd") else 9) + (part > 0)
            assert len(sizes) == n
            access = ACCESS[op][:n]
            assert add(op, sizes, access, a + slices) == "", a
    for op, a in (("linear_fwd", [1] * 6), ("cross_attention_fwd", [1] * 5),
                  ("cross_attention_fwd", [1, 1, 1, 1, 1, 300]), ("cross_attention_bwd", [1, 1, 1, 3, 2, 8]),
                  ("cross_attention_bwd", [1 << 62, 1, 1, 1, 1, 1])):
        with pytest.raises(ooc.OocError) as e:
            ooc.attention_slices(op, a)
        assert e.value.status == ooc.E_INVALID and "ooc_attention_slices" in e.value.message


def test_run_fn_refusals_before_the_device(lib):
    """Everything that is checked before any HIP call."""
    def refused(status, what, op, ptrs, access, attrs, sizes=None, device=0):
        with pytest.raises(ooc.OocError) as e:
            ooc.run_fn(op, list(zip(ptrs, sizes or [64] * len(ptrs))), access, attrs, device=device)
        assert e.value.status == status and what in e.value.message, e.value.message
    at = 1 << 20
    refused(ooc.E_INVALID, "not aligned", "relu_fwd", [at + 4, at + 128], [R, W], [16])
    refused(ooc.E_INVALID, "NULL", "relu_fwd", [0, at], [R, W], [16])
    refused(ooc.E_INVALID, "overlaps", "relu_fwd", [at, at], [R, W], [16])
    refused(ooc.E_INVALID, "overlaps", "relu_fwd", [at, at + 48], [R, W], [16])
    refused(ooc.E_INVALID, "overlaps", "acc", [at, at], [RW, R], [16])
    refused(ooc.E_INVALID, "size", "relu_fwd", [at, at + 64], [R, W], [16], sizes=[64, 0])
    refused(ooc.E_INVALID, "imply", "relu_fwd", [at, at + 64], [R, W], [17])
    refused(ooc.E_INVALID, "access", "relu_fwd", [at, at + 64], [R, 0], [16])
    refused(ooc.E_INVALID, "wrong access", "relu_fwd", [at, at + 64], [R, RW], [16])
    refused(ooc.E_INVALID, "attributes", "relu_fwd", [at, at + 64], [R, W], [])
    refused(ooc.E_INVALID, "unknown operation", 999, [at, at + 64], [R, W], [16])
    refused(ooc.E_INVALID, "unknown operation", -3, [at, at + 64], [R, W], [16])
    refused(ooc.E_INVALID, "device", "relu_fwd", [at, at + 64], [R, W], [16], device=-1)
    refused(ooc.E_INVALID, "variables", "noop", [], [], [])
    refused(ooc.E_UNSUPPORTED, "SGD", "sgd", [at, at + 64], [RW, R], [1, 0])
    assert lib.ooc_run_fn(0, None, 4, None, None, None, 2, None, 0) == ooc.E_INVALID
    p = (C.c_void_p * 1)(at)
    b, a = (C.c_uint64 * 1)(64), (C.c_uint8 * 1)(R)
    assert lib.ooc_run_fn(0, None, 4, p, b, a, 1, None, 3) == ooc.E_INVALID
    assert lib.ooc_qknorm_slices(3, None) == ooc.E_INVALID


def test_extra_inputs_of_a_workload():
    spec = small_seq2seq(layers=1)
    a, b = synth.make_extra_inputs(spec), synth.make_extra_inputs(spec)
    assert sorted(a) == sorted(v["name"] for v in spec["inputs"])
    for v in spec["inputs"]:
        np.testing.assert_array_equal(a[v["name"]], b[v["name"]])
        assert list(a[v["name"]].shape) == list(v["shape"])
    src = a["src"]
    assert src.min() >= 0 and src.max() < spec["classes"]
    assert a["src_len"].min() >= 1 and a["src_len"].max() <= src.shape[1]
    np.testing.assert_array_equal(a["src_pos"], np.tile(np.arange(src.shape[1]), src.shape[0]))
    half = a["table"].shape[0] - 1
    np.testing.assert_allclose(a["table"], netdef.rotary_table(2 * half), rtol=1e-14)
    given = np.full(half + 1, 0.25)
    np.testing.assert_array_equal(synth.make_extra_inputs(spec, {"table": given})["table"], given)


def test_two_tensors_of_one_name_are_refused():
    spec = small_seq2seq(layers=1)
    for name in (spec["inputs"][0]["name"], spec["layers"][0]["name"], "x", "labels"):
        wrong = dict(spec, inputs=spec["inputs"] + [{"name": name, "shape": [4], "dtype": "i32"}])
        with pytest.raises(ValueError, match="two tensors"):
            netdef.Net(wrong)


def test_work_of_the_operators():
    assert bench.fn_work("rope_fwd", [6, 32, 2, 16, 8, 0]) == ("byte", 8 * 6 * 32 + 24)
    assert bench.fn_work("qknorm_bwd", [6, 32, 1, 1, 16, 0, 0, 1]) == ("byte", 12 * 6 * 32 + 24)
    assert bench.fn_work("cross_attention_fwd", [2, 3, 5, 4, 2, 8, 1]) == \
        ("flop", 2 * 2 * 2 * 4 * 3 * 5 * 8)
    assert bench.fn_work("cross_attention_bwd", [2, 3, 5, 4, 2, 8, 1, 1]) == \
        ("flop", 5 * 2 * 2 * 4 * 3 * 5 * 8)
