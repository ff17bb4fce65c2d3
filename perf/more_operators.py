"""Timed calls of the operators of a decoder over packed documents: attention to a span of states with
capped scores and a distance bias, dropout whose mask is drawn again in the backward, the norms
around a block with its gate and residual scale, and a gated linear recurrence.

A case is one call as a program with tensors on the device makes it, forward ("fwd") or forward and
backward ("train").  Tensors are float32, as everywhere in the library.

* ``span``: ``Tq`` queries of each sequence against ``Tk`` states, ``H / Hkv`` query heads for each
  key head; query i sees the states lo <= j < hi of its own row of ``span`` = (lo, hi, at).  With
  ``cap`` scores become cap tanh(score / cap), with ``bias`` a head's slope times |at - j| is taken off.
  ``mask``: "causal"; "docs" (``docs`` documents a sequence, causal in each, a padded tail that sees
  nothing); "window" (those with the last ``window`` states only); "prefix" (a prefix that all see,
  causal behind it); "token" (one query behind a cache of another length in each sequence).
* ``dropout``: n values, each kept with probability 1 - drop / 2^32, by Philox 4x32-10 of its index.
* ``join``: h = scale x + gate drop(post rms(f)), n = pre rms(h); a gate row per sequence or one.
* ``scan``: h_t = a_t h_(t-1) + (1 - a_t) x_t with a = sigmoid(f), rows of f then x; ``carry``: from
  a state handed in; ``fresh``: from zero where a document starts.
"""

import math

import numpy as np
import torch

own = False

EPS = 1e-5
KINDS = {"span": ("B", "Tq", "Tk", "H", "Hkv", "dh"), "scan": ("B", "T", "C")}


def listed():
    return [
        # a new token of each of 8 sequences behind a cache, a sliding window, capped scores
        dict(name="span_token", op="span", dir="fwd", B=8, Tq=1, Tk=4096, H=16, Hkv=4, dh=64,
             mask="token", window=2048, docs=1, cap=30.0, bias=False),
        # a training batch of short documents packed into sequences of 512
        dict(name="span_docs", op="span", dir="train", B=24, Tq=512, Tk=512, H=16, Hkv=16, dh=64,
             mask="docs", window=0, docs=4, cap=0.0, bias=False),
        # a prefix read both ways, distances instead of positions, odd lengths and head width
        dict(name="span_prefix_odd", op="span", dir="train", B=3, Tq=1111, Tk=1111, H=12, Hkv=12,
             dh=85, mask="prefix", window=0, docs=1, cap=0.0, bias=True),
        # local attention over long documents, shared key heads, capped scores
        dict(name="span_window", op="span", dir="train", B=2, Tq=4096, Tk=4096, H=16, Hkv=4, dh=128,
             mask="window", window=1024, docs=3, cap=50.0, bias=False),
        # a long prompt, everything before each token
        dict(name="span_prompt", op="span", dir="fwd", B=1, Tq=8192, Tk=8192, H=8, Hkv=2, dh=64,
             mask="causal", window=0, docs=1, cap=0.0, bias=True),
        # the hidden row of a few tokens
        dict(name="dropout_small", op="dropout", dir="fwd", n=77 * 1024, drop=0.1),
        # the feed-forward's hidden values of a training batch
        dict(name="dropout_batch", op="dropout", dir="train", n=12288 * 4096, drop=0.1),
        # one token of 8 sequences, no dropout
        dict(name="join_tokens", op="join", dir="fwd", rows=8, d=1024, groups=1, drop=0.0),
        # a training batch, a gate for each of its 24 sequences
        dict(name="join_batch", op="join", dir="train", rows=12288, d=1024, groups=24, drop=0.1),
        # one token of 8 sequences with the states kept from before
        dict(name="scan_token", op="scan", dir="fwd", B=8, T=1, C=1024, carry=True, fresh=False),
        # a training batch
        dict(name="scan_batch", op="scan", dir="train", B=24, T=512, C=1024, carry=False, fresh=False),
        # one long sequence of documents, odd sizes
        dict(name="scan_long", op="scan", dir="train", B=1, T=32765, C=1365, carry=True, fresh=True),
    ]


def _log(rng, lo, hi):
    """An integer of lo .. hi, spread over its logarithm."""
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    """One more case of the same ranges."""
    most = {"span": 3.2e11, "dropout": 8.1e8, "join": 5.2e8, "scan": 1.7e9}
    while True:
        op = rng.choice(["span", "span", "span", "dropout", "join", "scan", "scan"])
        c = dict(op=op, dir=rng.choice(["fwd", "train"]))
        if op == "span":
            hkv = rng.choice([1, 2, 4, 5, 8, 12, 16])
            mask = rng.choice(["causal", "docs", "window", "prefix", "token"])
            T = _log(rng, 1, 8192)
            c.update(B=_log(rng, 1, 32), Tq=1 if mask == "token" else T, Tk=T,
                     H=hkv * rng.choice([1, 1, 2, 4]), Hkv=hkv,
                     dh=rng.choice([32, 48, 64, 64, 64, 80, 96, 128, 128, rng.randint(17, 128)]),
                     mask=mask, window=_log(rng, 1, max(1, T)) if mask in ("window", "token") else 0,
                     docs=_log(rng, 1, 16) if mask in ("docs", "window") else 1,
                     cap=rng.choice([0.0, 0.0, 20.0, 30.0, 50.0]), bias=rng.random() < 0.4)
            if mask == "token":
                c["dir"] = "fwd"
            if c["B"] * c["H"] * c["Tq"] * c["Tk"] > 6e8:
                continue
        elif op == "dropout":
            c.update(n=_log(rng, 1, 6e7), drop=rng.choice([0.0, 0.05, 0.1, 0.5, rng.random()]))
        elif op == "join":
            groups = _log(rng, 1, 32)
            c.update(rows=groups * _log(rng, 1, 16384), d=_log(rng, 1, 8192), groups=groups,
                     drop=rng.choice([0.0, 0.1, 0.1, rng.random()]))
        else:
            c.update(B=_log(rng, 1, 64), T=_log(rng, 1, 32768), C=_log(rng, 1, 8192),
                     carry=rng.random() < 0.5, fresh=rng.random() < 0.5)
        w = work(c)
        if (w["flops"] if op == "span" else w["bytes"]) <= most[op]:
            return c


# ---------------------------------------------------------------- inputs

def _spans(case, g):
    """(lo, hi, at) of every query, int32 [B Tq, 3]."""
    B, Tq, Tk, mask, dev = case["B"], case["Tq"], case["Tk"], case["mask"], g.device
    i = torch.arange(Tq, device=dev).expand(B, Tq)
    lo, hi, at = torch.zeros_like(i), i + 1, i

    def uniform(n, most):
        return torch.randint(0, most, (B, n), generator=g, device=dev)

    if mask == "token":
        n = 1 + uniform(1, Tk)
        n[0] = Tk
        lo, hi, at = (n - case["window"]).clamp(min=0), n, n - 1
        if B > 2:              # a sequence that has ended
            hi = hi.clone()
            hi[1] = lo[1]
    if mask in ("docs", "window"):
        starts = torch.zeros(B, Tq, dtype=torch.int64, device=dev)
        if case["docs"] > 1:
            where = uniform(case["docs"] - 1, Tq)
            starts.scatter_(1, where, where)
        lo = starts.cummax(1).values
    if mask == "window":
        lo = torch.maximum(lo, hi - case["window"])
    if mask == "docs":         # a padded tail
        end = Tq - uniform(1, Tq // 8 + 1)
        lo, hi = (torch.where(i < end, t, torch.zeros_like(t)) for t in (lo, hi))
    if mask == "prefix":
        hi = torch.maximum(hi, uniform(1, Tk) + 1)
    return torch.stack((lo, hi, at), -1).view(B * Tq, 3).to(torch.int32).contiguous()


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator(device=dev)
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.float32)

    s = dict(case)
    train = case["dir"] == "train"
    if case["op"] in ("dropout", "join"):
        s["drop"] = int(case["drop"] * 2.0 ** 32)
        s["salt"] = 7
        s["seed"] = torch.randint(-2 ** 31, 2 ** 31, (2,), generator=g, device=dev).to(torch.int32)
    if case["op"] == "span":
        B, Tq, Tk, H, Hkv, dh = (case[k] for k in KINDS["span"])
        s["q"] = normal(B * Tq, H * dh) * (3.0 if case["cap"] else 1.0)   # scores that meet the cap
        s["kv"] = normal(B * Tk, 2 * Hkv * dh)
        s["span"] = _spans(case, g)
        mod = [case["cap"]] if case["cap"] else []
        if case["bias"]:
            mod += [2.0 ** (-8.0 * (h + 1) / H) for h in range(H)]
        s["mod"] = torch.tensor(mod, dtype=torch.float32, device=dev)
        if train:
            s["dy"] = normal(B * Tq, H * dh)
    elif case["op"] == "dropout":
        s["x"] = normal(case["n"])
        if train:
            s["dy"] = normal(case["n"])
    elif case["op"] == "join":
        rows, d = case["rows"], case["d"]
        s["x"], s["f"] = normal(rows, d), normal(rows, d) * 0.5
        s["post"], s["pre"] = 1.0 + 0.1 * normal(d), 1.0 + 0.1 * normal(d)
        s["gate"] = 0.3 * normal(case["groups"], d)
        s["scale"] = torch.full((1,), 0.9, device=dev)
        if train:
            s["dh"], s["dn"] = normal(rows, d), normal(rows, d)
    else:
        B, T, C = (case[k] for k in KINDS["scan"])
        s["fx"] = normal(B * T, 2 * C)
        s["fx"][:, :C] += 3.0          # states that last for some twenty rows
        if case["carry"]:
            s["h0"] = normal(B, C)
        if case["fresh"]:              # documents of some 500 rows
            s["fresh_rows"] = (torch.rand(B * T, generator=g, device=dev) < 1 / 500).to(torch.int32)
        if train:
            s["dh"] = normal(B * T, C)
    return s


# ---------------------------------------------------------------- plain forms, in 32 bits

def _product(a, b):
    """High and low 32 bits of a constant times values below 2^32, in int64."""
    t = a * (b & 0xffff)
    u = a * (b >> 16) + (t >> 16)
    return u >> 16, ((u & 0xffff) << 16) | (t & 0xffff)


def _keep(s, n):
    """Which of n values are kept: word i % 4 of Philox 4x32-10 at counter (i / 4, salt)."""
    i = torch.arange((n + 3) // 4, device=s["seed"].device)
    c = [i & 0xffffffff, i >> 32, torch.full_like(i, s["salt"] & 0xffffffff),
         torch.full_like(i, s["salt"] >> 32)]
    key = s["seed"].long() & 0xffffffff
    for r in range(10):
        k0 = (key[0] + r * 0x9E3779B9) & 0xffffffff
        k1 = (key[1] + r * 0xBB67AE85) & 0xffffffff
        h0, l0 = _product(0xD2511F53, c[0])
        h1, l1 = _product(0xCD9E8D57, c[2])
        c = [h1 ^ c[1] ^ k0, l1, h0 ^ c[3] ^ k1, l0]
    return torch.stack(c, -1).view(-1)[:n] >= s["drop"]


def _drop(s, x):
    if not s["drop"]:
        return x
    keep = _keep(s, x.numel()).view(x.shape)
    return torch.where(keep, x * (2.0 ** 32 / (2 ** 32 - s["drop"])), torch.zeros_like(x))


def _split(s):
    """q, dy rows [B, Hkv, G Tq, dh] and k, v [B, Hkv, Tk, dh]: the query heads of a key head as rows."""
    B, Tq, Tk, H, Hkv, dh = (s[k] for k in KINDS["span"])

    def q_rows(t):
        return t.view(B, Tq, Hkv, H // Hkv, dh).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, dh)

    k, v = s["kv"].view(B, Tk, 2, Hkv, dh).permute(2, 0, 3, 1, 4)
    return q_rows, k.contiguous(), v.contiguous()


def _join_heads(s, t):
    """The rows of ``q_rows`` back in their layout."""
    B, Tq, _, H, Hkv, dh = (s[k] for k in KINDS["span"])
    return t.view(B, Hkv, H // Hkv, Tq, dh).permute(0, 3, 1, 2, 4).reshape(B * Tq, H * dh)


def _probs(s, q, k):
    """Probabilities, row logarithms, and what the cap multiplies gradients by (or None)."""
    B, Tq, Tk, H, Hkv, dh = (s[n] for n in KINDS["span"])
    S = q @ k.transpose(-1, -2).contiguous() * dh ** -0.5
    slope = None
    if s["cap"]:
        t = torch.tanh(S / s["cap"])
        S = s["cap"] * t
        slope = 1 - t * t
    S = S.view(B, H, Tq, Tk)
    lo, hi, at = s["span"].view(B, 1, Tq, 1, 3).unbind(-1)
    j = torch.arange(Tk, device=q.device, dtype=torch.int32)
    if s["bias"]:
        S = S - s["mod"][-H:].view(H, 1, 1) * (at - j).abs().float()
    S = S.masked_fill((j < lo) | (j >= hi), -math.inf)
    top = S.amax(-1, keepdim=True)
    P = torch.exp(S - top.clamp(min=-3e38))
    total = P.sum(-1, keepdim=True)      # a row that sees nothing: P = 0, lse = -inf
    P = (P / total.clamp(min=1e-38)).view(B, Hkv, -1, Tk)
    return P, (top + torch.log(total)).view(-1), slope


def _span(s):
    q_rows, k, v = _split(s)
    q = q_rows(s["q"])
    P, lse, slope = _probs(s, q, k)
    y = P @ v
    if s["dir"] == "fwd":
        return {"y": _join_heads(s, y), "lse": lse}
    dy = q_rows(s["dy"])
    dv = P.transpose(-1, -2).contiguous() @ dy
    dP = dy @ v.transpose(-1, -2).contiguous()
    dS = P * (dP - (dy * y).sum(-1, keepdim=True)) * s["dh"] ** -0.5
    if slope is not None:
        dS = dS * slope
    dq = dS @ k
    dk = dS.transpose(-1, -2).contiguous() @ q
    dkv = torch.stack((dk, dv)).permute(1, 3, 0, 2, 4).reshape(s["kv"].shape)
    return {"y": _join_heads(s, y), "lse": lse, "dq": _join_heads(s, dq), "dkv": dkv}


def _rms(x):
    return (x.square().mean(-1, keepdim=True) + EPS).rsqrt()


def _by_group(s, x):
    """x [rows, d] summed over the rows of each gate."""
    return x.view(s["groups"], -1, s["d"]).sum(1)


def _join(s):
    f, gate = s["f"], s["gate"].repeat_interleave(s["rows"] // s["groups"], 0)
    v = f * _rms(f)
    w = _drop(s, s["post"] * v)
    h = s["scale"] * s["x"] + gate * w
    r = _rms(h)
    t = h * r
    out = {"h": h, "n": s["pre"] * t}
    if s["dir"] == "fwd":
        return out
    dt = s["pre"] * s["dn"]
    dh = s["dh"] + r * (dt - t * (dt * t).mean(-1, keepdim=True))
    du = _drop(s, gate * dh)
    dv = s["post"] * du
    df = _rms(f) * (dv - v * (dv * v).mean(-1, keepdim=True))
    return dict(out, dx=s["scale"] * dh, df=df, dpost=(du * v).sum(0), dgate=_by_group(s, dh * w),
                dpre=(s["dn"] * t).sum(0))


def _doubling(A, b, back):
    """h_t = A_t h_(t-1) + b_t along axis 1 (back: h_t = A_t h_(t+1) + b_t), the reach doubled in
    each step."""
    n, T = 1, A.shape[1]
    A, b = A.clone(), b.clone()
    while n < T:
        near, far = (slice(0, T - n), slice(n, T)) if back else (slice(n, T), slice(0, T - n))
        b2, A2 = b.clone(), A.clone()
        b2[:, near] += A[:, near] * b[:, far]
        A2[:, near] *= A[:, far]
        A, b, n = A2, b2, 2 * n
    return b


def _scan(s):
    B, T, C = (s[k] for k in KINDS["scan"])
    f, x = s["fx"].view(B, T, 2, C).unbind(2)
    e = torch.exp(-f.abs())
    big, small = 1 / (1 + e), e / (1 + e)
    a, rest = torch.where(f >= 0, big, small), torch.where(f >= 0, small, big)
    A = a
    if s["fresh"]:
        A = a.masked_fill((s["fresh_rows"] != 0).view(B, T, 1), 0.0)
    b = rest * x
    if s["carry"]:
        b = b.clone()
        b[:, 0] += A[:, 0] * s["h0"]
    h = _doubling(A, b, False)
    if s["dir"] == "fwd":
        return {"h": h.view(B * T, C)}
    g = _doubling(torch.cat((A[:, 1:], torch.zeros_like(A[:, :1])), 1), s["dh"].view(B, T, C), True)
    first = s["h0"].view(B, 1, C) if s["carry"] else torch.zeros_like(h[:, :1])
    before = torch.cat((first, h[:, :-1]), 1)
    if s["fresh"]:
        before = before.masked_fill((s["fresh_rows"] != 0).view(B, T, 1), 0.0)
    df = g * (before - x) * a * rest
    out = {"h": h.view(B * T, C), "dfx": torch.stack((df, rest * g), 2).view(B * T, 2 * C)}
    if s["carry"]:
        out["dh0"] = A[:, 0] * g[:, 0]
    return out


# ---------------------------------------------------------------- the library's calls

def _call(op, reads, writes, attrs):
    from paper_2010_14109_amd import ooc
    tensors = reads + writes
    ooc.run_fn(op, [(t.data_ptr(), t.numel() * t.element_size()) for t in tensors],
               [ooc.R] * len(reads) + [ooc.W] * len(writes), attrs,
               device=tensors[0].device.index,
               stream=torch.cuda.current_stream(tensors[0].device).cuda_stream)


def _floats(t, nbytes):
    return [torch.empty(nbytes // 4, device=t.device)] if nbytes else []


def _own_span(s):
    from paper_2010_14109_amd import ooc
    shape = [s[k] for k in KINDS["span"]]
    attrs = shape + [int(s["cap"] > 0), int(s["bias"])]
    ins = [s["q"], s["kv"], s["span"]] + ([s["mod"]] if s["mod"].numel() else [])
    y = torch.empty_like(s["q"])
    lse = torch.empty(s["B"] * s["H"] * s["Tq"], device=y.device)
    slices, part = ooc.attention_slices("span_attention_fwd", shape)
    _call("span_attention_fwd", ins, [y, lse] + _floats(y, part), attrs + slices)
    if s["dir"] == "fwd":
        return {"y": y, "lse": lse}
    dq, dkv, delta = torch.empty_like(y), torch.empty_like(s["kv"]), torch.empty_like(lse)
    bounds = torch.empty(s["B"], -(-s["Tq"] // 32), 2, dtype=torch.int32, device=y.device)
    slices, part = ooc.attention_slices("span_attention_bwd", shape)
    _call("span_attention_bwd", ins + [y, lse, s["dy"]],
          [dq, dkv, delta, bounds] + _floats(y, part), attrs + slices)
    return {"y": y, "lse": lse, "dq": dq, "dkv": dkv}


def _own_dropout(s):
    attrs = [s["n"], s["drop"], s["salt"]]
    y = torch.empty_like(s["x"])
    _call("dropout", [s["x"], s["seed"]], [y], attrs)
    if s["dir"] == "fwd":
        return y
    dx = torch.empty_like(y)
    _call("dropout", [s["dy"], s["seed"]], [dx], attrs)
    return {"y": y, "dx": dx}


def _own_join(s):
    from paper_2010_14109_amd import ooc
    attrs = [s["rows"], s["d"], s["groups"], s["drop"], s["salt"]]
    gains = [s["post"], s["gate"], s["pre"], s["scale"]] + ([s["seed"]] if s["drop"] else [])
    h, n = torch.empty_like(s["x"]), torch.empty_like(s["x"])
    stats = torch.empty(s["rows"], 2, device=h.device)
    _call("join_fwd", [s["x"], s["f"]] + gains, [h, n, stats], attrs)
    if s["dir"] == "fwd":
        return {"h": h, "n": n}
    slices, part = ooc.join_slices(s["rows"], s["d"], s["groups"])
    dx, df = torch.empty_like(h), torch.empty_like(h)
    dpost, dgate, dpre = (torch.empty_like(s[k]) for k in ("post", "gate", "pre"))
    _call("join_bwd", [s["f"], h, stats] + gains + [s["dh"], s["dn"]],
          [dx, df, dpost, dgate, dpre] + _floats(h, part), attrs + [1, slices])
    return {"h": h, "n": n, "dx": dx, "df": df, "dpost": dpost, "dgate": dgate, "dpre": dpre}


def _own_scan(s):
    from paper_2010_14109_amd import ooc
    shape = [s[k] for k in KINDS["scan"]]
    attrs = shape + [int(s["carry"]), int(s["fresh"])]
    ins = [s["fx"]] + ([s["h0"]] if s["carry"] else []) + ([s["fresh_rows"]] if s["fresh"] else [])
    h = torch.empty(s["B"] * s["T"], s["C"], device=s["fx"].device)
    slices, part = ooc.scan_slices("scan_fwd", shape)
    _call("scan_fwd", ins, [h] + _floats(h, part), attrs + [slices])
    if s["dir"] == "fwd":
        return {"h": h}
    dfx = torch.empty_like(s["fx"])
    dh0 = [torch.empty_like(s["h0"])] if s["carry"] else []
    slices, part = ooc.scan_slices("scan_bwd", shape)
    _call("scan_bwd", ins + [h, s["dh"]], [dfx] + dh0 + _floats(h, part), attrs + [slices])
    return dict({"h": h, "dfx": dfx}, **({"dh0": dh0[0]} if dh0 else {}))


def run(state):
    if own:
        return {"span": _own_span, "dropout": _own_dropout, "join": _own_join,
                "scan": _own_scan}[state["op"]](state)
    if state["op"] == "dropout":
        y = _drop(state, state["x"])
        return y if state["dir"] == "fwd" else {"y": y, "dx": _drop(state, state["dy"])}
    return {"span": _span, "join": _join, "scan": _scan}[state["op"]](state)


def _pairs(case):
    """Pairs of a query and a state that it sees, in one sequence (the mean of what is drawn)."""
    T, mask, w = case["Tk"], case["mask"], case["window"]
    if mask == "token":
        return min(w, (T + 1) / 2)
    if mask == "prefix":
        return T * T * 2 / 3
    causal = T * T / (case["docs"] + 1) + T / 2
    return min(causal, T * w) if mask == "window" else causal


def work(case):
    """Bytes: inputs once, outputs once.  Flops: of attention, four per visible pair and head column
    forward, ten backward; elsewhere a few per value."""
    train = case["dir"] == "train"
    if case["op"] == "span":
        B, Tq, Tk, H, Hkv, dh = (case[k] for k in KINDS["span"])
        seen = B * (_pairs(case) if case["mask"] == "token" else Tk)
        q, kv, lse = 4 * B * Tq * H * dh, 8 * seen * Hkv * dh, 4 * B * H * Tq
        # backward: q, y, dy, kv, lse read, dq and dkv written
        back = 4 * q + 2 * kv + lse if train else 0
        return {"bytes": 2 * q + kv + 12 * B * Tq + lse + back,
                "flops": (14 if train else 4) * B * _pairs(case) * H * dh}
    if case["op"] == "dropout":
        return {"bytes": (16 if train else 8) * case["n"], "flops": (2 if train else 1) * case["n"]}
    if case["op"] == "join":
        values = case["rows"] * case["d"]
        return {"bytes": (40 if train else 16) * values, "flops": (40 if train else 12) * values}
    values = case["B"] * case["T"] * case["C"]
    return {"bytes": (36 if train else 12) * values, "flops": (20 if train else 8) * values}


# ---------------------------------------------------------------- 64 bits

def _exact_keep(s, n):
    """Truth values as 1.0 and 0.0, the generator in unsigned 64-bit arithmetic of the host."""
    word = np.uint64(0xffffffff)
    i = np.arange((n + 3) // 4, dtype=np.uint64)
    a, b = i & word, i >> np.uint64(32)
    c = np.full_like(i, s["salt"] & 0xffffffff)
    d = np.full_like(i, s["salt"] >> 32)
    k0, k1 = (int(k) & 0xffffffff for k in s["seed"].tolist())
    for _ in range(10):
        p, q = a * np.uint64(0xD2511F53), c * np.uint64(0xCD9E8D57)
        a, c = (q >> np.uint64(32)) ^ b ^ np.uint64(k0), (p >> np.uint64(32)) ^ d ^ np.uint64(k1)
        b, d = q & word, p & word
        k0, k1 = (k0 + 0x9E3779B9) & 0xffffffff, (k1 + 0xBB67AE85) & 0xffffffff
    kept = np.stack((a, b, c, d), 1).reshape(-1)[:n] >= np.uint64(s["drop"])
    return torch.from_numpy(kept).to(s["seed"].device).double()


def _exact_factor(s, n):
    if not s["drop"]:
        return torch.ones(n, dtype=torch.float64, device=s["seed"].device)
    return _exact_keep(s, n) / (1.0 - s["drop"] / 2.0 ** 32)


def _exact_join(case, s):
    d, groups = case["d"], case["groups"]
    x, f, post, pre, gate = (s[k].double() for k in ("x", "f", "post", "pre", "gate"))
    rows = torch.arange(case["rows"], device=x.device) // (case["rows"] // groups)
    m, rho = _exact_factor(s, x.numel()).view(x.shape), float(s["scale"])
    size_f = torch.sqrt((f * f).sum(1, keepdim=True) / d + EPS)
    w = post * f / size_f * m
    h = rho * x + gate[rows] * w
    size_h = torch.sqrt((h * h).sum(1, keepdim=True) / d + EPS)
    out = {"h": h, "n": pre * h / size_h}
    if case["dir"] == "fwd":
        return out
    dn = s["dn"].double()
    z = dn * pre
    dh = s["dh"].double() + z / size_h - h * (z * h).sum(1, keepdim=True) / (d * size_h ** 3)
    du = dh * gate[rows] * m
    z = du * post
    df = z / size_f - f * (z * f).sum(1, keepdim=True) / (d * size_f ** 3)
    dgate = torch.zeros_like(gate).index_add_(0, rows, dh * w)
    return dict(out, dx=rho * dh, df=df, dpost=(du * f / size_f).sum(0), dgate=dgate,
                dpre=(dn * h / size_h).sum(0))


def _exact_scan(case, s):
    B, T, C = (case[k] for k in KINDS["scan"])
    fx = s["fx"].double().view(B, T, 2 * C)
    a, x = torch.sigmoid(fx[..., :C]), fx[..., C:]
    rest = torch.sigmoid(-fx[..., :C])
    live = torch.ones(B, T, 1, dtype=torch.float64, device=fx.device)
    if case["fresh"]:
        live = (s["fresh_rows"] == 0).double().view(B, T, 1)
    h, state = torch.zeros_like(x), torch.zeros_like(x[:, 0])
    if case["carry"]:
        state = s["h0"].double()
    before = torch.zeros_like(x)
    for t in range(T):
        before[:, t] = state * live[:, t]
        state = a[:, t] * before[:, t] + rest[:, t] * x[:, t]
        h[:, t] = state
    if case["dir"] == "fwd":
        return {"h": h.view(B * T, C)}
    dh = s["dh"].double().view(B, T, C)
    g, later = torch.zeros_like(x), torch.zeros_like(x[:, 0])
    for t in range(T - 1, -1, -1):
        g[:, t] = dh[:, t] + later
        later = g[:, t] * a[:, t] * live[:, t]
    dfx = torch.cat((g * (before - x) * a * rest, g * rest), -1)
    out = {"h": h.view(B * T, C), "dfx": dfx.view(B * T, 2 * C)}
    return dict(out, dh0=later) if case["carry"] else out


def _exact_span(case, s):
    B, Tq, Tk, H, Hkv, dh = (case[k] for k in KINDS["span"])
    q = s["q"].double().view(B, Tq, H, dh)
    kv = s["kv"].double().view(B, Tk, 2, Hkv, dh)
    y, dq, dkv = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(kv)
    lse = torch.full((B, H, Tq), -math.inf, dtype=torch.float64, device=q.device)
    dy = s["dy"].double().view(B, Tq, H, dh) if "dy" in s else None
    span = s["span"].view(B, Tq, 3).double()
    j = torch.arange(Tk, device=q.device).double()
    for b in range(B):
        lo, hi, at = (span[b, :, c:c + 1] for c in range(3))
        seen = (j >= lo) & (j < hi)
        some = seen.any(1)
        for h in range(H):
            n = h * Hkv // H
            k, v = kv[b, :, 0, n], kv[b, :, 1, n]
            S = q[b, :, h] @ k.t() / math.sqrt(dh)
            turn = None
            if case["cap"]:
                turn = torch.cosh(S / case["cap"]) ** -2
                S = case["cap"] * torch.tanh(S / case["cap"])
            if case["bias"]:
                S = S - float(s["mod"][h - H]) * (at - j).abs()
            S = S.masked_fill(~seen, -math.inf)
            lse[b, h] = torch.logsumexp(S, 1)
            P = torch.where(some[:, None], torch.softmax(S, 1), torch.zeros_like(S))
            y[b, :, h] = P @ v
            if dy is None:
                continue
            g = dy[b, :, h]
            dP = g @ v.t()
            dS = P * (dP - (P * dP).sum(1, keepdim=True)) / math.sqrt(dh)
            if turn is not None:
                dS = dS * turn
            dq[b, :, h] = dS @ k
            dkv[b, :, 0, n] += dS.t() @ q[b, :, h]
            dkv[b, :, 1, n] += P.t() @ g
    out = {"y": y.view(B * Tq, H * dh), "lse": lse.view(-1)}
    return out if dy is None else dict(out, dq=dq.view(B * Tq, -1), dkv=dkv.view(B * Tk, -1))


def exact(case, seed):
    if case["op"] == "span":
        B, Tq, Tk, H, _, dh = (case[k] for k in KINDS["span"])
        if B * H * Tq * Tk * dh > 2e11:
            return None
        return _exact_span(case, prepare(case, seed))
    s = prepare(case, seed)
    if case["op"] == "join":
        return _exact_join(case, s)
    if case["op"] == "scan":
        return _exact_scan(case, s)
    m = _exact_factor(s, case["n"])
    y = s["x"].double() * m
    return y if case["dir"] == "fwd" else {"y": y, "dx": s["dy"].double() * m}
