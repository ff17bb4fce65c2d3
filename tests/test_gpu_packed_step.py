"""Training steps of decoders over packed documents: span attention, gated recurrences, joins and dropout
together, in core against the oracle and out of core bit for bit."""

import numpy as np
import pytest

from oracle import schedule as S
from oracle.interp import run as oracle_run
from oracle.lower import lower
from paper_2010_14109_amd import netdef, synth
from test_decoder_ops_host import gated_and_carried, small_packed
from test_gpu_attention_ops import run_step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("build", [
    lambda: small_packed(), gated_and_carried, lambda: small_packed(p=0.0, cap=0.0, layers=3),
    lambda: small_packed(batch=1, seq=1), lambda: small_packed(d=128, heads=2, kv_heads=1, seq=300, ffn=70)],
    ids=["packed", "gated", "plain", "one", "wide"])
def test_packed_step(build):
    """Loss, every gradient and update of a step against the oracle; out of core, the same bits."""
    spec = build()
    x, labels = synth.make_inputs(spec, 0)
    params, extra = synth.make_params(spec, 1), synth.make_extra_inputs(spec)
    g = np.random.default_rng(5)
    for n in params:      # gains and gates of their own
        if n.endswith((".post", ".pre", ".gate")):
            params[n] = (params[n] + 0.3 * g.standard_normal(params[n].shape)).astype(np.float32)
    loss, outs = run_step(spec, x, labels, params, extra)
    net = netdef.Net(spec, keep_grads=True)
    reg = lower(spec, keep_grads=True, slices=net.slices)
    ref = oracle_run(reg, x, labels, {k: v.astype(np.float64) for k, v in params.items()}, inputs=extra)
    assert abs(loss - ref["loss"][-1]) <= 1e-5 * abs(ref["loss"][-1])
    one = spec["input"][1] == 1
    for name, v in outs.items():
        want = ref[name].reshape(v.shape)
        # the whole-step tolerance of the other networks.  With one state to see, P = 1: dq and dk are
        # differences of equal sums, zero but for their roundings, 64 u |dy| |v| |k| or less with all
        # three below 1 here, of which what they alone feed sums 24: 9e-5
        if one and ".q." in name or one and ".kv." in name:
            assert np.abs(v - want).max() <= 1e-4, name
            continue
        assert np.linalg.norm(v - want) <= 1e-4 * np.linalg.norm(want) + 1e-9, name
    b, k, f = net.var_bytes, net.var_kinds, net.fn_vars
    want2 = run_step(spec, x, labels, params, extra, steps=2)
    for frac, policy in ((0.5, "C"), (0.0, "C"), (0.4, "L")):
        budget = max(S.budget_for(frac, S.incore_peak(b, k, f, 4096), 4096) if frac else 0,
                     S.working_set_max(b, f, 4096))
        got = run_step(spec, x, labels, params, extra, budget, policy, steps=2)
        assert got[0] == want2[0]
        for name in got[1]:
            assert got[1][name].tobytes() == want2[1][name].tobytes(), (name, frac, policy)
