"""Benchmark of the out-of-core training step on one MI355X.

Prints one JSON line: samples/s of the out-of-core step at the workload's
budget (the value), the in-core step on the same data, host-link rates, the
device bytes the pool owns, the roofline of the dominant kernel and the CPU
oracle timed on a bounded sample.

    python bench.py [--steps K] [--warmup W] [--workload resnet50_b1440|cnn|mlp|resnet50_b256|...]

The default workload is ResNet-50 at batch 1440 with a budget of P_incore / 7.5, the setting of
the paper's Table 1 (Section 5.1).  Its host footprint exceeds what one process can pin on the
MI355X hosts here, so the out-of-core run retries with a 56 GiB pinned limit when the whole arena
is refused (TEMPs beyond it move through pinned staging slots).

Inputs and parameters are seeded and synthetic (shapes of the workload).  In
the out-of-core step the pinned host arena is the variables' home: the step
swaps them in and out itself, and that traffic is the method's work, so it is
inside the timed region.  The in-core step keeps everything in HBM.
"""

from __future__ import annotations

import argparse
import json
import os
import platform
import sys
import time

import numpy as np

from paper_2010_14109_amd import netdef, ooc, synth

PEAK_BF16_TFLOPS = 2500.0      # MI355X dense bf16 matrix instructions, and fp16
PRODUCTS = 6                   # of bf16 pieces for each fp32 product (gemm.hip)
FP16_PRODUCTS = 3              # of fp16 pieces for each fp32 product (attend.hip)
PEAK_HBM_GBS = 8000.0          # MI355X HBM3E
PCIE5_X16_GBS = 63.0           # theoretical, per direction


def fn_work(op, attrs, states=None):
    """Algorithmic work of one function: ('flop', n) for GEMM-shaped ops, ('byte', n) for
    memory-bound ones (compulsory HBM bytes: every operand read once, every result
    written once).  ``states``: of all sequences together, for a cross attention whose sequences
    are padded."""
    a = attrs
    if op in ("linear_fwd", "linear_bwd_w", "linear_bwd_x"):
        return "flop", 2 * a[0] * a[1] * a[2]
    if op in ("conv_fwd", "conv_bwd_x", "conv_bwd_w"):
        N, H, W, C, K, R, S, st, pd, P, Q = a[:11]
        return "flop", 2 * N * P * Q * K * R * S * C
    if op == "relu_fwd":
        return "byte", 8 * a[0]
    if op in ("relu_bwd", "add", "acc"):
        return "byte", 12 * a[0]
    if op == "bn_fwd":
        return "byte", 8 * a[0] * a[1]
    if op == "bn_bwd":
        return "byte", 12 * a[0] * a[1]
    if op == "maxpool_fwd":
        N, H, W, C, k, st, pd, P, Q = a
        return "byte", 4 * N * H * W * C + 5 * N * P * Q * C
    if op == "maxpool_bwd":
        N, H, W, C, k, st, pd, P, Q = a
        return "byte", 5 * N * P * Q * C + 4 * N * H * W * C
    if op in ("avgpool_fwd", "avgpool_bwd"):
        N, H, W, C = a
        return "byte", 4 * N * H * W * C + 4 * N * C
    if op == "softmax_ce":
        return "byte", 8 * a[0] * a[1]
    if op == "embed_fwd":
        B, T, V, d = a
        return "byte", 8 * B * T * d + 4 * B * T + 4 * T * d
    if op == "embed_bwd":
        B, T, V, d = a
        return "byte", 4 * B * T * d + 4 * B * T + 4 * V * d + 4 * T * d
    if op == "layernorm_fwd":
        return "byte", 8 * a[0] * a[1] + 8 * a[0]
    if op == "layernorm_bwd":
        return "byte", 12 * a[0] * a[1] + 8 * a[0]
    if op == "gelu_fwd":
        return "byte", 8 * a[0]
    if op == "gelu_bwd":
        return "byte", 12 * a[0]
    if op in ("concat_fwd", "concat_bwd"):
        return "byte", 8 * a[0] * sum(a[1:])
    if op in ("upsample_fwd", "upsample_bwd"):
        N, H, W, C = a
        return "byte", 20 * N * H * W * C
    if op in ("attention_fwd", "attention_bwd"):
        # q k^T and P v forward; backward, q k^T again (P is recomputed) and four products
        # of the same size; causal attention needs only the T (T + 1) / 2 entries on and
        # below the diagonal
        B, T, H, dh, causal = a[:5]
        pairs = T * (T + 1) // 2 if causal else T * T
        return "flop", (2 if op == "attention_fwd" else 5) * 2 * B * H * pairs * dh
    if op in ("rope_fwd", "rope_bwd", "qknorm_fwd"):
        return "byte", 8 * a[0] * a[1] + 4 * a[0]
    if op == "qknorm_bwd":
        return "byte", 12 * a[0] * a[1] + 4 * a[0]
    if op in ("cross_attention_fwd", "cross_attention_bwd"):
        # two products of every query and state of its sequence forward, five backward
        B, Tq, Tk, H, Hkv, dh = a[:6]
        pairs = Tq * (B * Tk if states is None else states)
        return "flop", (2 if op.endswith("fwd") else 5) * 2 * H * pairs * dh
    return "byte", 0


def sgd_bytes(net, j):
    mom = net.fn_attrs[j][1]
    total = 0
    for v, acc in net.fn_vars[j]:
        total += net.var_bytes[v] * (2 if acc == ooc.RW else 1)
    return total if mom in (0, 1) else 0


def algorithmic_bytes(net, op):
    """Mean compulsory bytes per launch of ``op``: every operand read once and every result
    written once (an input gradient reads the filter and the output gradient and writes the
    input gradient).  Partial sums (``.part``, ``.bpart``) are not compulsory and are left out."""
    tot, n = 0, 0
    for j, o in enumerate(net.fn_ops):
        if o == op:
            tot += sum(net.var_bytes[v] for v, _ in net.fn_vars[j]
                       if not net.names[v].endswith((".part", ".bpart")))
            n += 1
    return round(tot / n) if n else None


def roofline(dom, op=None):
    """Rate of the dominant function (``op``) against what bounds it: products against the matrix
    instructions that carry them, everything else against HBM."""
    if dom["unit"] == "flop":
        fp16 = op in ("cross_attention_fwd", "cross_attention_bwd")
        products = FP16_PRODUCTS if fp16 else PRODUCTS
        peak = PEAK_BF16_TFLOPS / products
        return {"bound": "mfma", "achieved": round(dom["rate"], 3), "peak": round(peak, 1),
                "peak_of": f"fp32 products as {products} {'fp16' if fp16 else 'bf16'} products of "
                           f"split operands, "
                           f"{PEAK_BF16_TFLOPS:g} TFLOP/s dense",
                "unit": "TFLOP/s", "frac": round(dom["rate"] / peak, 4), "traffic": None}
    return {"bound": "hbm", "achieved": round(dom["rate"], 1), "peak": PEAK_HBM_GBS,
            "unit": "GB/s", "frac": round(dom["rate"] / PEAK_HBM_GBS, 4), "traffic": None}


def measured_traffic(net, op):
    """Mean HBM bytes per launch of ``op`` in this network, from the rocprofv3 FETCH_SIZE /
    WRITE_SIZE measurements recorded under profiles/ (lines ``traffic: op=... key=<attrs>
    bytes=... source=<file> sha256=...``).  None unless every launch's attribute list has a
    measurement whose kernel source is unchanged since it was taken."""
    import glob
    import hashlib
    here = os.path.dirname(os.path.abspath(__file__))
    table = {}
    for f in glob.glob(os.path.join(here, "profiles", "traffic_*.md")):
        with open(f) as fh:
            for line in fh:
                if not line.startswith("traffic: "):
                    continue
                kv = dict(t.split("=", 1) for t in line.split()[1:])
                src = os.path.join(here, kv["source"])
                if not os.path.exists(src):
                    continue
                with open(src, "rb") as sf:
                    if hashlib.sha256(sf.read()).hexdigest() != kv["sha256"]:
                        continue
                table[(kv["op"], kv["key"])] = int(kv["bytes"])
    got = []
    for o, attrs in zip(net.fn_ops, net.fn_attrs):
        if o == op:
            b = table.get((op, ",".join(str(a) for a in attrs)))
            if b is None:
                return None
            got.append(b)
    return round(sum(got) / len(got)) if got else None


# schedule-window W as a fraction of the budget.  The paper leaves W to the user and the library's
# default is B/2; a sweep on one MI355X (0.1 to 0.5 of B) found B/4 best or level on every workload
# but the MLP: a narrower window admits swap-ins later, so fewer variables are swapped out early to
# make room, and the host link carries fewer bytes.  The MLP's swap-ins are weights needed in both
# passes, which want the wider window.
DEFAULT_WINDOW_FRAC = 0.25
WINDOW_FRAC = {"mlp": 0.5}


def window_fraction(workload):
    return WINDOW_FRAC.get(workload, DEFAULT_WINDOW_FRAC)

# pinned host memory asked for when the whole arena cannot be pinned (on the MI355X hosts measured
# one process pins at most 64 GiB)
DEFAULT_HOST_LIMIT = 56 << 30

# The paper's own throughput for the one setting measured here exactly as it states it (Table 1,
# Schedule + VA): ResNet-50 at batch 1440 on a 16 GB V100, i.e. a budget of about P_incore / 7.5,
# 321 images/s.  Another machine's figure: it gives ``vs_baseline`` as context, not a target.
PAPER_TABLE1_B1440_IPS = 321.0


def paper_figure(workload, batch, frac, scheduler, layout, wait_order):
    """The paper's samples/s for this run's exact setting, or None where it prints none."""
    exact = (workload == "resnet50_b1440" and batch == 1440
             and abs(frac - synth.budget_fraction("resnet50_b1440")) < 1e-9
             and scheduler == "adaptive" and layout == "pool" and wait_order == "oldest")
    return PAPER_TABLE1_B1440_IPS if exact else None
MAP_ENTRY_LIMIT = 40000   # chunks + mappings per plan; the process table holds ~65530


def plan_for(net, frac, window_frac, chunk, policy="C", fixed=None, wait="oldest",
             budget_bytes=None):
    """Budget, window and (chunks, mappings) of the out-of-core and in-core plans.  The budget
    is frac * P_incore (P_incore at this chunk size), or budget_bytes when given, rounded down
    to whole chunks and never below WS_max."""
    ctx = ooc.Context(-1)
    try:
        net.register(ctx)
        ctx.set_chunk(chunk)
        p_incore, ws_max = ctx.incore_peak(), ctx.working_set_max()
    finally:
        ctx.close()
    want = int(p_incore * frac) if budget_bytes is None else budget_bytes
    budget = want // chunk * chunk
    if budget < ws_max:
        if budget_bytes is not None:
            raise ooc.OocError(ooc.E_INFEASIBLE, f"budget {budget} B is below WS_max {ws_max} B "
                                                 f"at chunk {chunk} B")
        budget = ws_max
    window = int(budget * window_frac)
    counts = []
    build_ms = None
    for b, w in ((budget, window), (ooc.UNLIMITED, None)):
        ctx = ooc.Context(-1)
        try:
            net.register(ctx)
            ctx.set_chunk(chunk)
            ctx.set_budget(b)
            if w is not None:
                ctx.set_window(w)
                ctx.set_policy(policy)
                ctx.set_wait_order(wait)
                if fixed is not None:
                    ctx.set_fixed_distance(*fixed)
            t0 = time.perf_counter()
            ctx.build_schedule()
            if build_ms is None:
                build_ms = (time.perf_counter() - t0) * 1e3
            counts.append(sum(ctx.plan_counts()))
        finally:
            ctx.close()
    return {"p_incore": p_incore, "ws_max": ws_max, "budget": budget, "window": window,
            "map_entries": max(counts), "build_ms": build_ms}


def choose_chunk(net, frac, window_frac, policy="C", fixed=None, wait="oldest"):
    """Smallest chunk (2 MiB .. 256 MiB) whose plans fit the memory-map table: the
    trade-off of Section 4 between mapping overhead and internal fragmentation."""
    for mib in (2, 4, 8, 16, 32, 64, 128, 256):
        plan = plan_for(net, frac, window_frac, mib << 20, policy, fixed, wait)
        if plan["map_entries"] <= MAP_ENTRY_LIMIT:
            return mib << 20, plan
    return 256 << 20, plan


def run_mode(net, spec, x, labels, params, budget, window, chunk, steps, warmup, depth=None,
             policy="C", fixed=None, wait="oldest", host_limit=None, layout="pool"):
    ctx = ooc.Context(0)
    try:
        net.register(ctx)
        if budget != ooc.UNLIMITED:
            ctx.set_layout(layout)
        if host_limit is not None and budget != ooc.UNLIMITED:
            ctx.set_host_limit(host_limit)
        ctx.set_policy(policy)
        ctx.set_wait_order(wait)
        if fixed is not None and budget != ooc.UNLIMITED:
            ctx.set_fixed_distance(*fixed)
        if depth is not None:
            ctx.set_swapout_depth(depth)
        ctx.set_chunk(chunk)
        ctx.set_budget(budget)
        if window is not None:
            ctx.set_window(window)
        ctx.build_schedule()
        ctx.prepare()
        net.view(ctx, "x")[...] = x
        net.view(ctx, "labels")[...] = labels
        for name, value in synth.make_extra_inputs(spec).items():
            net.view(ctx, name)[...] = value
        for name in net.param_names():
            net.view(ctx, name)[...] = params[name]
        for name in net.names:
            if name.startswith("m:"):
                net.view(ctx, name)[...] = 0
        ctx.upload()
        lr, mu = spec["optimizer"]["lr"], spec["optimizer"]["momentum"]
        mode = "in-core" if budget == ooc.UNLIMITED else "out-of-core"
        for i in range(warmup):
            s0 = time.perf_counter()
            ctx.step(lr, mu)
            print(f"{mode} warm-up step {i}: {(time.perf_counter() - s0) * 1e3:.1f} ms",
                  file=sys.stderr, flush=True)
        # ooc_step returns after all three streams are synchronized
        t0 = time.perf_counter()
        loss = None
        step_ms = []
        for _ in range(steps):
            s0 = time.perf_counter()
            loss = ctx.step(lr, mu)
            step_ms.append((time.perf_counter() - s0) * 1e3)
            if step_ms[-1] > 1000:   # long steps report as they go
                print(f"{mode} step: {step_ms[-1]:.1f} ms", file=sys.stderr, flush=True)
        elapsed = time.perf_counter() - t0
        return {"elapsed": elapsed, "loss": loss, "stats": ctx.stats(), "fn_ms": ctx.fn_times(),
                "step_ms": step_ms, "timeline": ctx.timeline()}
    finally:
        ctx.close()


def kernel_table(net, fn_ms, inputs=None):
    """Time and work of each operation; ``inputs``: {name: array} of the network's further inputs,
    whose lengths say how many states a cross attention has."""
    table = {}
    for j, (op, attrs) in enumerate(zip(net.fn_ops, net.fn_attrs)):
        states = None
        if op.startswith("cross_attention") and inputs:
            states = int(inputs[net.names[net.fn_vars[j][2][0]]].sum())
        kind, work = fn_work(op, attrs, states)
        if op == "sgd":
            kind, work = "byte", sgd_bytes(net, j)
        e = table.setdefault(op, {"ms": 0.0, "launches": 0, "unit": kind, "work": 0})
        e["ms"] += fn_ms[j]
        e["launches"] += 1
        e["work"] += work
    for op, e in table.items():
        sec = e["ms"] / 1e3
        if e["unit"] == "flop":
            e["rate"] = e["work"] / sec / 1e12 if sec > 0 else 0.0
            e["rate_unit"] = "TFLOP/s"
        else:
            e["rate"] = e["work"] / sec / 1e9 if sec > 0 else 0.0
            e["rate_unit"] = "GB/s"
    return table


def _cpu_model():
    try:
        with open("/proc/cpuinfo") as fh:
            for line in fh:
                if line.startswith("model name"):
                    return line.split(":", 1)[1].strip()
    except OSError:
        pass
    return platform.processor() or "unknown"


def _blas():
    try:
        from threadpoolctl import threadpool_info
        libs = [f"{p.get('internal_api')} {p.get('version')}" for p in threadpool_info()
                if p.get("user_api") == "blas"]
        return ", ".join(libs) or "unknown"
    except Exception:  # noqa: BLE001 - informational only
        return "unknown"


def oracle_schedule_ms(spec, slices, budget, window, chunk, policy, fixed, wait="oldest"):
    """Wall time of the oracle's scheduler on the full-size function sequence (median of 3);
    ``slices``: the split-K counts of the weight gradients, as registered."""
    from oracle import schedule as S
    from oracle.lower import as_schedule_input, lower
    b, k, f = as_schedule_input(lower(spec, slices=slices))
    ahead, thr = fixed if fixed is not None else (None, None)
    times = []
    for _ in range(3):
        t0 = time.perf_counter()
        S.build(b, k, f, budget, window, chunk, policy, ahead, thr, wait=wait)
        times.append((time.perf_counter() - t0) * 1e3)
    return sorted(times)[1]


def cpu_baseline(name, budget_seconds=15.0):
    """The float32 oracle step (``oracle.interp``) on a reduced batch of the same network."""
    from oracle.interp import run as oracle_run
    from oracle.lower import lower
    small = {"mlp": 256, "cnn": 8, "resnet50_b256": 2, "resnet50_b1440": 2,
             "transformer": 1, "seq2seq": 1, "densenet": 2, "unet": 1}[name]
    spec = synth.workload(name, batch=small)
    reg = lower(spec)
    x, labels = synth.make_inputs(spec, 0)
    params = synth.make_params(spec, 1)
    extra = synth.make_extra_inputs(spec)
    try:
        from threadpoolctl import threadpool_info
        threads = max([p.get("num_threads", 1) for p in threadpool_info()] or [1])
    except Exception:  # noqa: BLE001 - informational only
        threads = len(os.sched_getaffinity(0))
    oracle_run(reg, x, labels, params, dtype=np.float32, inputs=extra)     # warm-up
    n = 0
    t0 = time.perf_counter()
    while True:
        oracle_run(reg, x, labels, params, dtype=np.float32, inputs=extra)
        n += 1
        el = time.perf_counter() - t0
        if el >= budget_seconds or n >= 1000:
            break
    return {"value": n * small / el, "unit": "samples/s", "cores": threads, "kind": "oracle",
            "sample": f"{n} float32 oracle steps of {spec['name']} (batch {small}) in "
                      f"{el:.1f} s",
            "cpu_model": _cpu_model(), "blas": _blas()}


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--gpus", type=int, default=1)
    ap.add_argument("--steps", type=int, default=10)
    ap.add_argument("--warmup", type=int, default=2)
    ap.add_argument("--workload", default="resnet50_b1440", choices=sorted(synth.WORKLOADS))
    ap.add_argument("--batch", type=int, default=0, help="override the workload's batch")
    ap.add_argument("--budget-frac", type=float, default=None)
    ap.add_argument("--budget-bytes", type=int, default=None,
                    help="budget in bytes instead of a fraction of P_incore (the chunk-size sweep "
                         "keeps it fixed while m_c changes)")
    ap.add_argument("--window-frac", type=float, default=None,
                    help="W / B (default: B/4, the MLP B/2)")
    ap.add_argument("--chunk", type=int, default=0, help="bytes; 0 = smallest that fits")
    ap.add_argument("--no-cpu-baseline", action="store_true")
    ap.add_argument("--no-incore", action="store_true")
    ap.add_argument("--swapout-depth", type=int, default=None,
                    help="swap-outs in flight (library default when omitted; 0 = unbounded)")
    ap.add_argument("--scheduler", default="adaptive", choices=("adaptive", "naive", "lms"),
                    help="adaptive: the schedule-window algorithm with W = window-frac * B and "
                         "cancelled swap-outs; naive: swap every variable in right before and "
                         "out right after each use (W = 0, literal policy); lms: the "
                         "fixed-distance rule with --swapin-ahead / --swapout-threshold")
    ap.add_argument("--wait-order", default="oldest", choices=("oldest", "furthest"),
                    help="which pending swap-out a budget wait completes: the oldest (the "
                         "paper's procedure) or the one whose variable is used again furthest "
                         "ahead")
    ap.add_argument("--swapin-ahead", type=int, default=1, help="functions (lms)")
    ap.add_argument("--swapout-threshold", type=int, default=1, help="functions (lms)")
    ap.add_argument("--host-limit-gib", type=float, default=None,
                    help="most pinned host memory for the arena (GiB); TEMPs beyond it get "
                         "pageable homes copied through pinned staging slots")
    ap.add_argument("--layout", default="pool", choices=("pool", "bestfit"),
                    help="device memory of the out-of-core run: the chunk pool (Section 4), or "
                         "one contiguous best-fit heap holding each allocation at its replayed "
                         "offset (the allocator the pool is compared with, Fig. 3)")
    ap.add_argument("--timeline", default="",
                    help="write the last out-of-core step's kernel and copy spans (JSON) here")
    args = ap.parse_args()
    if args.gpus != 1:
        print(json.dumps({"error": "this build runs on one GPU; --gpus must be 1 "
                                   "(multi-GPU sharding is described, not built)"}))
        sys.exit(2)

    spec = synth.workload(args.workload, **({"batch": args.batch} if args.batch else {}))
    net = netdef.Net(spec)
    frac = args.budget_frac if args.budget_frac is not None else synth.budget_fraction(args.workload)
    policy = "L" if args.scheduler == "naive" else "C"
    if args.window_frac is None:
        args.window_frac = window_fraction(args.workload)
    window_frac = args.window_frac if args.scheduler == "adaptive" else 0.0
    fixed = (args.swapin_ahead, args.swapout_threshold) if args.scheduler == "lms" else None
    try:
        if args.chunk:
            chunk, plan = args.chunk, plan_for(net, frac, window_frac, args.chunk, policy, fixed,
                                               args.wait_order, args.budget_bytes)
        else:
            chunk, plan = choose_chunk(net, frac, window_frac, policy, fixed, args.wait_order)
    except ooc.OocError as e:
        if e.status != ooc.E_INFEASIBLE:
            raise
        print(json.dumps({"error": "infeasible", "scheduler": args.scheduler,
                          "detail": str(e)}))
        sys.exit(3)
    p_incore, budget, window = plan["p_incore"], plan["budget"], plan["window"]
    x, labels = synth.make_inputs(spec, 0)
    params = synth.make_params(spec, 1)
    batch = spec["input"][0]

    link = ooc.link_probe(0, 1 << 30, 3)
    inc = None
    if not args.no_incore:
        inc = run_mode(net, spec, x, labels, params, ooc.UNLIMITED, None, chunk, args.steps,
                       args.warmup)
    host_limit = None if args.host_limit_gib is None else int(args.host_limit_gib * (1 << 30))
    try:
        out = run_mode(net, spec, x, labels, params, budget, window, chunk, args.steps,
                       args.warmup, args.swapout_depth, policy, fixed, args.wait_order, host_limit,
                       args.layout)
    except ooc.OocError as e:
        # the host could not pin the whole arena: give the TEMPs beyond a limit pageable homes
        if e.status != ooc.E_HOST_OOM or host_limit is not None:
            raise
        host_limit = DEFAULT_HOST_LIMIT
        print(f"pinned arena refused ({e}); retrying with --host-limit-gib "
              f"{host_limit / (1 << 30):g}", file=sys.stderr, flush=True)
        out = run_mode(net, spec, x, labels, params, budget, window, chunk, args.steps,
                       args.warmup, args.swapout_depth, policy, fixed, args.wait_order, host_limit,
                       args.layout)
    if args.timeline:
        with open(args.timeline, "w") as fh:
            json.dump({"fns": net.fn_ops, "vars": net.names,
                       "spans": [list(t) for t in out["timeline"]]}, fh)
    st = out["stats"]
    ms = out["elapsed"] / args.steps * 1e3
    value = batch * args.steps / out["elapsed"]
    table = kernel_table(net, out["fn_ms"], synth.make_extra_inputs(spec))
    dom_op = max(table, key=lambda o: table[o]["ms"])
    dom = table[dom_op]
    roof = roofline(dom, dom_op)
    roof["traffic"] = measured_traffic(net, dom_op)
    roof["traffic_unit"] = ("bytes per launch fetched and written back by the L2 caches (rocprofv3 "
                            "FETCH_SIZE + WRITE_SIZE, calibrated; last-level-cache hits included)")
    roof["algorithmic_bytes"] = algorithmic_bytes(net, dom_op)
    roof["kernel"] = dom_op
    roof["launches_per_step"] = dom["launches"]
    roof["avg_launch_ms"] = round(dom["ms"] / max(1, dom["launches"]), 4)

    step_s = out["elapsed"] / args.steps
    moved = st["h2d_bytes"] + st["d2h_bytes"]
    # link ceiling: forward compute overlapped with the swap-outs, backward compute with the
    # swap-ins, each direction at its probed rate (the forward only swaps out, the backward
    # mostly swaps in, so the two directions do not overlap each other)
    ceiling = None
    if inc is not None:
        split = max(j for j, op in enumerate(net.fn_ops) if op == "softmax_ce") + 1
        t_fwd, t_bwd = sum(inc["fn_ms"][:split]), sum(inc["fn_ms"][split:])
        t_inc = inc["elapsed"] / args.steps * 1e3
        bound = (max(t_fwd, st["d2h_bytes"] / link["d2h"] / 1e6)
                 + max(t_bwd, st["h2d_bytes"] / link["h2d"] / 1e6))
        ceiling = {"bound_ms": round(bound, 2), "pct_of_incore": round(100 * t_inc / bound, 2),
                   "measured_pct_of_ceiling": round(100 * bound / ms, 2)}
    paper = paper_figure(args.workload, batch, frac, args.scheduler, args.layout, args.wait_order)
    res = {
        "metric": "samples/s at budget B as % of in-core; host-link GB/s; peak device bytes",
        "value": round(value, 3),
        "unit": "samples/s",
        "n_gpus": 1,
        "steps": args.steps,
        "warmup": args.warmup,
        "ms_per_step": round(ms, 3),
        "median_ms_per_step": round(float(np.median(out["step_ms"])), 3),
        "higher_is_better": True,
        "scaling": "weak",
        "vs_baseline": None if paper is None else round(value / paper, 4),
        "vs_baseline_basis": None if paper is None else {
            "value": paper, "unit": "images/s",
            "source": "paper Table 1, Schedule + VA, ResNet-50 batch 1440, one 16 GB V100 "
                      "(other hardware: context, not a target)"},
        "dtype": "f32",
        "data": "synthetic (seeded N(0,1) inputs, uniform labels, He-normal weights)",
        "config": {"workload": spec["name"], "batch": batch, "budget_bytes": budget,
                   "budget_frac_of_incore_peak": round(budget / p_incore, 4),
                   "incore_peak_bytes": p_incore, "window_bytes": window, "chunk_bytes": chunk,
                   "map_entries": plan["map_entries"],
                   "scheduler": args.scheduler,
                   **({"swapin_ahead": fixed[0], "swapout_threshold": fixed[1]} if fixed else {}),
                   "policy": "cancel" if policy == "C" else "literal",
                   "wait_order": args.wait_order, "layout": args.layout,
                   "swapout_depth": "library default" if args.swapout_depth is None
                   else args.swapout_depth},
        "roofline": roof,
        "incore": None if inc is None else {
            "samples_per_s": round(batch * args.steps / inc["elapsed"], 3),
            "ms_per_step": round(inc["elapsed"] / args.steps * 1e3, 3),
            "pool_bytes": inc["stats"]["pool_bytes"]},
        "pct_of_incore": None if inc is None else round(100 * inc["elapsed"] / out["elapsed"], 2),
        "host_link": {
            "h2d_bytes_per_step": st["h2d_bytes"], "d2h_bytes_per_step": st["d2h_bytes"],
            "sched_d2h_bytes_per_step": st["sched_d2h_bytes"],
            "achieved_GBps": round(moved / step_s / 1e9, 2),
            "h2d_busy_GBps": round(st["h2d_bytes"] / (st["h2d_busy_ms"] / 1e3) / 1e9, 2)
            if st["h2d_busy_ms"] > 0 else None,
            "d2h_busy_GBps": round(st["d2h_bytes"] / (st["d2h_busy_ms"] / 1e3) / 1e9, 2)
            if st["d2h_busy_ms"] > 0 else None,
            "h2d_busy_ms": round(st["h2d_busy_ms"], 2), "d2h_busy_ms": round(st["d2h_busy_ms"], 2),
            "probe_GBps": {k: round(v, 2) for k, v in link.items()},
            "pcie5_x16_theoretical_GBps_per_dir": PCIE5_X16_GBS,
            "full_duplex_bound_ms": round(max(st["h2d_bytes"] / link["h2d"],
                                              st["d2h_bytes"] / link["d2h"],
                                              moved / link["both"]) / 1e6, 2),
            "ceiling": ceiling,
            "pinned_arena_bytes": st["host_bytes"],
            "host_limit_bytes": host_limit,
            "pageable_overflow_bytes": st["spill_bytes"],
            "staged_h2d_bytes_per_step": st["staged_h2d_bytes"],
            "staged_d2h_bytes_per_step": st["staged_d2h_bytes"],
        },
        "peak_device_bytes": {"pool": st["pool_bytes"], "prepare_ms": round(st["prepare_ms"], 1),
                              "mappings": st["n_mappings"], "max_chunks_in_use_bytes":
                              st["max_chunks_used"] * chunk, "peak_accounted": st["peak_accounted"],
                              "hipMemGetInfo_delta": st["device_bytes_delta"],
                              "runtime_overhead": st["device_bytes_delta"] - st["pool_bytes"],
                              "budget": budget},
        "schedule_build_ms": {"library": round(plan["build_ms"], 3), "oracle": None},
        "compute_busy_ms_per_step": round(st["compute_busy_ms"], 2),
        "loss": out["loss"],
        "kernels": {op: {"ms": round(e["ms"], 3), "launches": e["launches"],
                         "rate": round(e["rate"], 3), "unit": e["rate_unit"]}
                    for op, e in sorted(table.items(), key=lambda kv: -kv[1]["ms"])},
        "cpu_baseline": None,
    }
    if not args.no_cpu_baseline:
        res["cpu_baseline"] = cpu_baseline(args.workload)
        res["schedule_build_ms"]["oracle"] = round(
            oracle_schedule_ms(spec, net.slices, budget, window, chunk, policy, fixed,
                               args.wait_order), 3)
    print(json.dumps(res), flush=True)


if __name__ == "__main__":
    main()
