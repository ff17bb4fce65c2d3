"""Seeded synthetic workloads: network descriptions and input/parameter bytes.

This module is shared by the product path and by the CPU oracle, so it holds
no part of the out-of-core method: no function sequence, no byte accounting,
no scheduling, no layer arithmetic.  It only states *which* network is trained
(layer kinds and their hyper-parameters, in topological order) and draws the
random bytes fed to both sides:

* data    -- ``numpy.random.Generator(PCG64(0))``: ``x`` as standard normal
             float32, then the labels as ``integers(0, classes)`` (int32);
* weights -- ``numpy.random.Generator(PCG64(1))``: He-normal fan-in for conv
             and dense weights, zero biases, BatchNorm gamma = 1, beta = 0.

Layouts are those of the library boundary: images are NHWC, conv weights are
``[K, R, S, C]`` (output channel, filter row, filter column, input channel),
dense weights are ``[out, in]``; token batches are ``[B, T]`` int32 and the
transformer's activations are ``[B T, features]``.  Transformer weights are
drawn N(0, 0.02).

The workloads stand in for the ones the paper trains (ResNet-50 on 224x224
ImageNet batches, Section 5.1 and Table 1) plus smaller networks of the same
layer kinds; ImageNet itself is not used.
"""

from __future__ import annotations

import numpy as np

# --------------------------------------------------------------------------
# network descriptions (plain data)
# --------------------------------------------------------------------------


def mlp(batch=256, width=1024, depth=8, classes=10, lr=0.01, momentum=0.0):
    """``depth`` dense layers of ``width`` with ReLU between them, last one to ``classes``."""
    layers = []
    prev = "x"
    for i in range(depth):
        out = classes if i == depth - 1 else width
        layers.append({"name": f"fc{i + 1}", "op": "linear", "in": [prev],
                       "in_features": width, "out_features": out})
        prev = f"fc{i + 1}"
        if i != depth - 1:
            layers.append({"name": f"relu{i + 1}", "op": "relu", "in": [prev]})
            prev = f"relu{i + 1}"
    return {"name": f"mlp{depth}_w{width}_b{batch}", "input": [batch, width],
            "classes": classes, "layers": layers, "logits": prev,
            "optimizer": {"lr": lr, "momentum": momentum}}


def plain_cnn(batch=128, channels=64, depth=10, hw=32, in_ch=3, classes=10,
              lr=0.01, momentum=0.0):
    """``depth`` x [conv3x3 s1 p1 + BatchNorm + ReLU], global average pool, dense head."""
    layers = []
    prev = "x"
    cin = in_ch
    for i in range(depth):
        layers.append({"name": f"conv{i + 1}", "op": "conv", "in": [prev], "cin": cin,
                       "cout": channels, "k": 3, "stride": 1, "pad": 1})
        layers.append({"name": f"bn{i + 1}", "op": "bn", "in": [f"conv{i + 1}"], "c": channels})
        layers.append({"name": f"relu{i + 1}", "op": "relu", "in": [f"bn{i + 1}"]})
        prev = f"relu{i + 1}"
        cin = channels
    layers.append({"name": "gap", "op": "avgpool", "in": [prev]})
    layers.append({"name": "fc", "op": "linear", "in": ["gap"], "in_features": channels,
                   "out_features": classes})
    return {"name": f"cnn{depth}_c{channels}_b{batch}", "input": [batch, hw, hw, in_ch],
            "classes": classes, "layers": layers, "logits": "fc",
            "optimizer": {"lr": lr, "momentum": momentum}}


def resnet(batch=256, hw=224, classes=1000, blocks=(3, 4, 6, 3), width=64,
           lr=0.01, momentum=0.9):
    """Bottleneck ResNet (ResNet-50 for blocks (3,4,6,3)); stride on the 3x3 conv."""
    layers = []

    def conv_bn(name, src, cin, cout, k, stride, pad, relu=True):
        layers.append({"name": f"{name}.conv", "op": "conv", "in": [src], "cin": cin,
                       "cout": cout, "k": k, "stride": stride, "pad": pad})
        layers.append({"name": f"{name}.bn", "op": "bn", "in": [f"{name}.conv"], "c": cout})
        if relu:
            layers.append({"name": f"{name}.relu", "op": "relu", "in": [f"{name}.bn"]})
            return f"{name}.relu"
        return f"{name}.bn"

    prev = conv_bn("stem", "x", 3, width, 7, 2, 3)
    layers.append({"name": "stem.pool", "op": "maxpool", "in": [prev], "k": 3, "stride": 2,
                   "pad": 1})
    prev = "stem.pool"
    cin = width
    for stage, nblocks in enumerate(blocks):
        mid = width * (2 ** stage)
        cout = mid * 4
        for b in range(nblocks):
            stride = 2 if (b == 0 and stage > 0) else 1
            base = f"s{stage + 1}b{b + 1}"
            h = conv_bn(f"{base}.a", prev, cin, mid, 1, 1, 0)
            h = conv_bn(f"{base}.b", h, mid, mid, 3, stride, 1)
            h = conv_bn(f"{base}.c", h, mid, cout, 1, 1, 0, relu=False)
            if b == 0:
                sc = conv_bn(f"{base}.down", prev, cin, cout, 1, stride, 0, relu=False)
            else:
                sc = prev
            layers.append({"name": f"{base}.add", "op": "add", "in": [h, sc]})
            layers.append({"name": f"{base}.out", "op": "relu", "in": [f"{base}.add"]})
            prev = f"{base}.out"
            cin = cout
    layers.append({"name": "gap", "op": "avgpool", "in": [prev]})
    layers.append({"name": "fc", "op": "linear", "in": ["gap"], "in_features": cin,
                   "out_features": classes})
    depth = 2 + 3 * sum(blocks)
    return {"name": f"resnet{depth}_b{batch}_{hw}", "input": [batch, hw, hw, 3],
            "classes": classes, "layers": layers, "logits": "fc",
            "optimizer": {"lr": lr, "momentum": momentum}}


def transformer(batch=64, seq=512, d=1024, heads=16, ffn=4096, layers=48, vocab=32000,
                lr=0.01, momentum=0.0):
    """Pre-LN causal transformer encoder with learned positions and an untied LM head,
    trained on next-token cross-entropy."""
    L = [{"name": "embed", "op": "embed", "in": ["x"], "vocab": vocab, "d": d}]
    prev = "embed"
    for i in range(layers):
        b = f"l{i + 1}"
        L += [
            {"name": f"{b}.ln1", "op": "layernorm", "in": [prev]},
            {"name": f"{b}.qkv", "op": "linear", "in": [f"{b}.ln1"], "in_features": d,
             "out_features": 3 * d},
            {"name": f"{b}.attn", "op": "attention", "in": [f"{b}.qkv"], "heads": heads,
             "causal": True},
            {"name": f"{b}.proj", "op": "linear", "in": [f"{b}.attn"], "in_features": d,
             "out_features": d},
            {"name": f"{b}.res1", "op": "add", "in": [f"{b}.proj", prev]},
            {"name": f"{b}.ln2", "op": "layernorm", "in": [f"{b}.res1"]},
            {"name": f"{b}.fc1", "op": "linear", "in": [f"{b}.ln2"], "in_features": d,
             "out_features": ffn},
            {"name": f"{b}.gelu", "op": "gelu", "in": [f"{b}.fc1"]},
            {"name": f"{b}.fc2", "op": "linear", "in": [f"{b}.gelu"], "in_features": ffn,
             "out_features": d},
            {"name": f"{b}.res2", "op": "add", "in": [f"{b}.fc2", f"{b}.res1"]},
        ]
        prev = f"{b}.res2"
    L += [{"name": "lnf", "op": "layernorm", "in": [prev]},
          {"name": "head", "op": "linear", "in": ["lnf"], "in_features": d, "out_features": vocab}]
    return {"name": f"transformer{layers}_d{d}_b{batch}_t{seq}", "input": [batch, seq],
            "tokens": True, "classes": vocab, "layers": L, "logits": "head", "init": "normal",
            "optimizer": {"lr": lr, "momentum": momentum}}


def seq2seq(batch=24, src_seq=512, seq=512, d=1024, heads=16, kv_heads=4, ffn=4096, layers=6,
            vocab=32000, lr=0.01, momentum=0.9):
    """Encoder-decoder transformer: every self-attention reads rotated queries and keys (in the
    encoder adjacent pairs of half of each head, in the decoder, after per-head norms, pairs half
    a head apart), and each decoder layer attends to the encoder's states, padded to ``src_seq``
    and of ``src_len`` tokens each, with ``kv_heads`` shared key heads and normalised queries and
    keys.  Trained on next-token cross-entropy of the decoder."""
    dh = d // heads
    L = []

    def lin(name, src, fin, fout):
        L.append({"name": name, "op": "linear", "in": [src], "in_features": fin,
                  "out_features": fout})
        return name

    def norm(name, src):
        L.append({"name": name, "op": "layernorm", "in": [src]})
        return name

    def join(name, a, b):
        L.append({"name": name, "op": "add", "in": [a, b]})
        return name

    def qknorm(name, src, h1, h2, turn):
        L.append({"name": name, "op": "qknorm", "in": [src], "h1": h1, "h2": h2, "dh": dh,
                  "rot": dh // 2 * 2 if turn else 0, "layout": 1, "pos": "pos", "table": "table"})
        return name

    def attend(b, qkv, src, causal):
        L.append({"name": f"{b}.attn", "op": "attention", "in": [qkv], "heads": heads,
                  "causal": causal})
        return join(f"{b}.res1", lin(f"{b}.proj", f"{b}.attn", d, d), src)

    def feed(b, src):
        lin(f"{b}.fc1", norm(f"{b}.lnf", src), d, ffn)
        L.append({"name": f"{b}.gelu", "op": "gelu", "in": [f"{b}.fc1"]})
        return join(f"{b}.res3", lin(f"{b}.fc2", f"{b}.gelu", ffn, d), src)

    L.append({"name": "src_embed", "op": "embed", "in": ["src"], "vocab": vocab, "d": d})
    prev = "src_embed"
    rot = max(2, dh // 4 * 2)
    for i in range(layers):
        b = f"e{i + 1}"
        lin(f"{b}.qkv", norm(f"{b}.ln1", prev), d, 3 * d)
        L.append({"name": f"{b}.rope", "op": "rope", "in": [f"{b}.qkv"], "heads": 2 * heads,
                  "dh": dh, "rot": rot, "layout": 0, "pos": "src_pos", "table": "src_table"})
        prev = feed(b, attend(b, f"{b}.rope", prev, False))
    memory = norm("memory", prev)
    L.append({"name": "embed", "op": "embed", "in": ["x"], "vocab": vocab, "d": d})
    prev = "embed"
    for i in range(layers):
        b = f"d{i + 1}"
        lin(f"{b}.qkv", norm(f"{b}.ln1", prev), d, 3 * d)
        prev = attend(b, qknorm(f"{b}.qk", f"{b}.qkv", heads, heads, True), prev, True)
        q = qknorm(f"{b}.qn", lin(f"{b}.q", norm(f"{b}.ln2", prev), d, d), heads, 0, False)
        kv = qknorm(f"{b}.kn", lin(f"{b}.kv", memory, d, 2 * kv_heads * dh), kv_heads, 0, False)
        L.append({"name": f"{b}.cross", "op": "cross_attention", "in": [q, kv], "heads": heads,
                  "kv_heads": kv_heads, "klen": "src_len"})
        prev = feed(b, join(f"{b}.res2", lin(f"{b}.cproj", f"{b}.cross", d, d), prev))
    lin("head", norm("lnf", prev), d, vocab)
    inputs = [{"name": "src", "shape": [batch, src_seq], "dtype": "i32"},
              {"name": "src_len", "shape": [batch], "dtype": "i32"},
              {"name": "src_pos", "shape": [batch * src_seq], "dtype": "i32"},
              {"name": "src_table", "shape": [rot // 2 + 1], "dtype": "f64"},
              {"name": "pos", "shape": [batch * seq], "dtype": "i32"},
              {"name": "table", "shape": [dh // 2 + 1], "dtype": "f64"}]
    return {"name": f"seq2seq{layers}_d{d}_b{batch}_t{src_seq}_{seq}", "input": [batch, seq],
            "inputs": inputs, "tokens": True, "classes": vocab, "layers": L, "logits": "head",
            "init": "normal", "optimizer": {"lr": lr, "momentum": momentum}}


def packed(batch=24, seq=512, d=1024, heads=16, kv_heads=4, ffn=4096, layers=8, vocab=8192, p=0.1,
           cap=30.0, lr=0.01, momentum=0.9):
    """Decoder over documents packed into its sequences: blocks of a gated recurrence and of attention
    in turn, each with a feed-forward block behind it.  The recurrence starts afresh where a document
    does; attention sees a token's own document up to it, its scores capped and falling with distance
    (no positions are added to them).  Each block's output joins the residual stream through a norm, a
    gate and dropout, and the next norm's output is the next block's input; the feed-forward's hidden
    values are dropped too.  Inputs beside the tokens: spans, fresh rows, mod, a seed and a scale."""
    dh = d // heads
    L = [{"name": "embed", "op": "embed", "in": ["x"], "vocab": vocab, "d": d},
         {"name": "norm", "op": "layernorm", "in": ["embed"]}]
    stream, prev, salt = "embed", "norm", 0

    def lin(name, src, fin, fout):
        L.append({"name": name, "op": "linear", "in": [src], "in_features": fin,
                  "out_features": fout})
        return name

    def join(name, out):
        nonlocal stream, prev, salt
        salt += 1
        L.append({"name": name, "op": "join", "in": [stream, out], "d": d, "p": p, "salt": salt,
                  "seed": "seed", "scale": "scale"})
        stream, prev = name + ".h", name

    for i in range(layers):
        b = f"b{i + 1}"
        if i % 2 == 0:
            L.append({"name": f"{b}.scan", "op": "scan", "in": [lin(f"{b}.fx", prev, d, 2 * d)],
                      "fresh": "fresh"})
            mixed = f"{b}.scan"
        else:
            q, kv = lin(f"{b}.q", prev, d, d), lin(f"{b}.kv", prev, d, 2 * kv_heads * dh)
            L.append({"name": f"{b}.attn", "op": "span_attention", "in": [q, kv], "heads": heads,
                      "kv_heads": kv_heads, "span": "span", "cap": cap > 0, "bias": True, "mod": "mod"})
            mixed = f"{b}.attn"
        join(f"{b}.join1", lin(f"{b}.out", mixed, d, d))
        L.append({"name": f"{b}.gelu", "op": "gelu", "in": [lin(f"{b}.fc1", prev, d, ffn)]})
        hidden = f"{b}.gelu"
        if p:
            salt += 1
            L.append({"name": f"{b}.drop", "op": "dropout", "in": [hidden], "p": p, "salt": salt,
                      "seed": "seed"})
            hidden = f"{b}.drop"
        join(f"{b}.join2", lin(f"{b}.fc2", hidden, ffn, d))
    lin("head", prev, d, vocab)
    inputs = [{"name": "span", "shape": [batch * seq, 3], "dtype": "i32"},
              {"name": "fresh", "shape": [batch * seq], "dtype": "i32"},
              {"name": "mod", "shape": [(cap > 0) + heads], "dtype": "f32"},
              {"name": "seed", "shape": [2], "dtype": "i32"},
              {"name": "scale", "shape": [1], "dtype": "f32"}]
    return {"name": f"packed{layers}_d{d}_b{batch}_t{seq}", "input": [batch, seq], "inputs": inputs,
            "tokens": True, "classes": vocab, "layers": L, "logits": "head", "init": "normal",
            "cap": cap, "optimizer": {"lr": lr, "momentum": momentum}}


def densenet(batch=64, hw=64, growth=32, blocks=(6, 12, 24, 16), stem=64, classes=10,
             lr=0.01, momentum=0.9):
    """DenseNet-shaped network (no bottleneck): inside a block every layer reads the channel
    concatenation of the stem or transition output and of every earlier layer's output
    (BN, ReLU, conv3x3 to ``growth`` channels), so each feature map is read by all later layers
    of its block.  Between blocks: concatenation, BN, ReLU, conv1x1 to half the channels,
    2x2 max pool.  Head: concatenation, BN, ReLU, global average pool, dense."""
    layers = [{"name": "stem", "op": "conv", "in": ["x"], "cin": 3, "cout": stem, "k": 3,
               "stride": 1, "pad": 1}]
    feats, chans = ["stem"], [stem]

    def gather(name):
        if len(feats) == 1:
            return feats[0]
        layers.append({"name": name, "op": "concat", "in": list(feats)})
        return name

    for b, n in enumerate(blocks):
        for i in range(n):
            base = f"b{b + 1}l{i + 1}"
            src = gather(f"{base}.cat")
            layers += [
                {"name": f"{base}.bn", "op": "bn", "in": [src], "c": sum(chans)},
                {"name": f"{base}.relu", "op": "relu", "in": [f"{base}.bn"]},
                {"name": f"{base}.conv", "op": "conv", "in": [f"{base}.relu"], "cin": sum(chans),
                 "cout": growth, "k": 3, "stride": 1, "pad": 1},
            ]
            feats.append(f"{base}.conv")
            chans.append(growth)
        c = sum(chans)
        base = f"t{b + 1}" if b + 1 < len(blocks) else "head"
        src = gather(f"{base}.cat")
        layers += [{"name": f"{base}.bn", "op": "bn", "in": [src], "c": c},
                   {"name": f"{base}.relu", "op": "relu", "in": [f"{base}.bn"]}]
        if b + 1 < len(blocks):
            layers += [
                {"name": f"{base}.conv", "op": "conv", "in": [f"{base}.relu"], "cin": c,
                 "cout": c // 2, "k": 1, "stride": 1, "pad": 0},
                {"name": f"{base}.pool", "op": "maxpool", "in": [f"{base}.conv"], "k": 2,
                 "stride": 2, "pad": 0},
            ]
            feats, chans = [f"{base}.pool"], [c // 2]
        else:
            layers += [{"name": "gap", "op": "avgpool", "in": [f"{base}.relu"]},
                       {"name": "fc", "op": "linear", "in": ["gap"], "in_features": c,
                        "out_features": classes}]
    return {"name": f"densenet{sum(blocks)}_g{growth}_b{batch}_{hw}",
            "input": [batch, hw, hw, 3], "classes": classes, "layers": layers, "logits": "fc",
            "optimizer": {"lr": lr, "momentum": momentum}}


def unet(batch=8, hw=256, base=64, depth=4, classes=8, lr=0.01, momentum=0.9):
    """U-Net-shaped segmentation network: ``depth`` encoder levels of two (conv3x3, BN, ReLU)
    followed by a 2x2 max pool, a bottleneck, and decoder levels that upsample (nearest, 2x),
    convolve to the level's width, concatenate the encoder output of the same level (a skip
    across the whole network) and apply two (conv3x3, BN, ReLU); a conv1x1 gives per-pixel
    logits, trained on per-pixel labels."""
    layers = []

    def cbr(name, src, cin, cout):
        layers.extend([
            {"name": f"{name}.conv", "op": "conv", "in": [src], "cin": cin, "cout": cout, "k": 3,
             "stride": 1, "pad": 1},
            {"name": f"{name}.bn", "op": "bn", "in": [f"{name}.conv"], "c": cout},
            {"name": f"{name}.relu", "op": "relu", "in": [f"{name}.bn"]}])
        return f"{name}.relu"

    prev, cin, skips = "x", 3, []
    for i in range(depth):
        c = base * 2 ** i
        prev = cbr(f"e{i + 1}a", prev, cin, c)
        prev = cbr(f"e{i + 1}b", prev, c, c)
        skips.append((prev, c))
        layers.append({"name": f"e{i + 1}.pool", "op": "maxpool", "in": [prev], "k": 2,
                       "stride": 2, "pad": 0})
        prev, cin = f"e{i + 1}.pool", c
    c = base * 2 ** depth
    prev = cbr("mid.a", prev, cin, c)
    prev = cbr("mid.b", prev, c, c)
    cin = c
    for i in reversed(range(depth)):
        skip, c = skips[i]
        layers.append({"name": f"d{i + 1}.up", "op": "upsample", "in": [prev]})
        prev = cbr(f"d{i + 1}u", f"d{i + 1}.up", cin, c)
        layers.append({"name": f"d{i + 1}.cat", "op": "concat", "in": [prev, skip]})
        prev = cbr(f"d{i + 1}a", f"d{i + 1}.cat", 2 * c, c)
        prev = cbr(f"d{i + 1}b", prev, c, c)
        cin = c
    layers.append({"name": "out", "op": "conv", "in": [prev], "cin": cin, "cout": classes, "k": 1,
                   "stride": 1, "pad": 0})
    return {"name": f"unet{depth}_c{base}_b{batch}_{hw}", "input": [batch, hw, hw, 3],
            "classes": classes, "dense_labels": True, "layers": layers, "logits": "out",
            "optimizer": {"lr": lr, "momentum": momentum}}


#: The workloads: name -> (network description, budget as a fraction of the
#: in-core peak).  seq2seq is an encoder-decoder transformer; packed is a decoder
#: over packed documents; densenet and unet are long-skip networks whose feature maps are read many times; the others are
#: the benchmark configurations.
WORKLOADS = {
    "mlp": (lambda: mlp(), 0.40),
    "cnn": (lambda: plain_cnn(), 0.50),
    "resnet50_b256": (lambda: resnet(batch=256), 0.25),
    "resnet50_b1440": (lambda: resnet(batch=1440), 1.0 / 7.5),
    "transformer": (lambda: transformer(), 0.20),
    "seq2seq": (lambda: seq2seq(), 0.20),
    "densenet": (lambda: densenet(), 0.25),
    "unet": (lambda: unet(), 0.25),
    "packed": (lambda: packed(), 0.20),
}


def workload(name, **overrides):
    """Network description of a named workload, with keyword overrides (e.g. ``batch=8``)."""
    builders = {"mlp": mlp, "cnn": plain_cnn, "resnet50_b256": resnet,
                "resnet50_b1440": resnet, "transformer": transformer, "densenet": densenet,
                "unet": unet, "seq2seq": seq2seq, "packed": packed}
    defaults = {"resnet50_b256": {"batch": 256}, "resnet50_b1440": {"batch": 1440}}
    kw = dict(defaults.get(name, {}))
    kw.update(overrides)
    return builders[name](**kw)


def budget_fraction(name):
    return WORKLOADS[name][1]


# --------------------------------------------------------------------------
# seeded bytes
# --------------------------------------------------------------------------


def param_shapes(spec):
    """Parameter tensors of a network description, in layer order: ``[(name, shape)]``.

    The shapes are read off the layer hyper-parameters only.
    """
    out = []
    length = {"x": spec["input"][1]} if spec.get("tokens") else {}
    length.update((v["name"], v["shape"][1]) for v in spec.get("inputs", ()) if len(v["shape"]) == 2)
    for L in spec["layers"]:
        if L["op"] == "embed":
            out.append((L["name"] + ".E", (L["vocab"], L["d"])))
            out.append((L["name"] + ".pos", (length[L["in"][0]], L["d"])))
        elif L["op"] == "qknorm":
            out.append((L["name"] + ".gain", (2 if L["h2"] else 1, L["dh"])))
        elif L["op"] == "join":
            out.append((L["name"] + ".post", (L["d"],)))
            if "gate" not in L:
                out.append((L["name"] + ".gate", (1, L["d"])))
            out.append((L["name"] + ".pre", (L["d"],)))
        elif L["op"] == "layernorm":
            out.append((L["name"] + ".gamma", (_width(spec, L),)))
            out.append((L["name"] + ".beta", (_width(spec, L),)))
        elif L["op"] == "linear":
            out.append((L["name"] + ".W", (L["out_features"], L["in_features"])))
            out.append((L["name"] + ".b", (L["out_features"],)))
        elif L["op"] == "conv":
            out.append((L["name"] + ".W", (L["cout"], L["k"], L["k"], L["cin"])))
        elif L["op"] == "bn":
            out.append((L["name"] + ".gamma", (L["c"],)))
            out.append((L["name"] + ".beta", (L["c"],)))
    return out


def _width(spec, layer):
    """Feature width of a transformer LayerNorm: the model width of the embedding."""
    return next(L["d"] for L in spec["layers"] if L["op"] == "embed")


def make_inputs(spec, seed=0):
    """``(x, labels)``.  Images: x float32 of the input shape, labels int32 [N] uniform over
    the classes ([N H W], one per pixel, for per-pixel logits).  Tokens: ids [B, T + 1] uniform over the vocabulary; x = ids[:, :T] (int32)
    and the labels are the next tokens ids[:, 1:] flattened to [B T]."""
    g = np.random.Generator(np.random.PCG64(seed))
    if spec.get("tokens"):
        B, T = spec["input"]
        ids = g.integers(0, spec["classes"], size=(B, T + 1)).astype(np.int32)
        return np.ascontiguousarray(ids[:, :T]), np.ascontiguousarray(ids[:, 1:]).reshape(-1)
    x = g.standard_normal(size=tuple(spec["input"]), dtype=np.float32)
    n = int(np.prod(spec["input"][:3])) if spec.get("dense_labels") else spec["input"][0]
    labels = g.integers(0, spec["classes"], size=n).astype(np.int32)
    return x, labels


def make_extra_inputs(spec, tables=None, seed=2):
    """``{name: array}`` of ``spec["inputs"]``.  By the layers that name them: ``fresh`` of a recurrence, the
    first rows of some four documents a sequence; ``span`` of an attention, what each row sees of its own
    document, and its ``mod``, the network's cap, where the layer has one, then falling slopes; ``seed``, two
    words; ``scale`` of a join, 1.  The others by type and name: i32 of two axes are tokens, uniform over the
    vocabulary; i32 ``<tokens>_len`` their lengths, uniform over 1 .. the sequence; i32 ``*pos`` positions
    counting up in each sequence; f64 tables of angles, ``tables[name]`` or 10000^(-2 i / rot) radians per
    position and magnitude 1; f32 standard normal.  Anything else is a ValueError."""
    g = np.random.Generator(np.random.PCG64(seed))
    shapes = {v["name"]: tuple(v["shape"]) for v in spec.get("inputs", ())}
    batch = spec["input"][0]
    out = {}
    use, capped = {}, set()     # what a layer takes an input for
    for L in spec.get("layers", ()):
        for key in {"span_attention": ("span", "mod"), "scan": ("fresh",), "dropout": ("seed",),
                    "join": ("seed", "scale")}.get(L["op"], ()):
            use.setdefault(L.get(key), key)
        if L["op"] == "span_attention" and L.get("cap"):
            capped.add(L.get("mod"))

    def first_rows(rows):
        """Each row's document's first row, by sequence; the same for every input."""
        T = rows // batch
        cuts = np.random.Generator(np.random.PCG64([seed, rows])).integers(0, T, (batch, 3, 1))
        at = np.arange(T)
        return np.where(at >= cuts, cuts, 0).max(1), np.broadcast_to(at, (batch, T))

    for v in spec.get("inputs", ()):
        name, shape = v["name"], tuple(v["shape"])
        kind = (v["dtype"], use.get(name))
        if kind == ("i32", "span") and shape[1:] == (3,) and shape[0] % batch == 0:
            first, at = first_rows(shape[0])
            out[name] = np.stack([first, at + 1, at], -1).reshape(shape).astype(np.int32)
        elif kind == ("i32", "fresh") and len(shape) == 1 and shape[0] % batch == 0:
            first, at = first_rows(shape[0])
            out[name] = (first == at).astype(np.int32).reshape(shape)
        elif kind == ("i32", "seed") and shape == (2,):
            out[name] = g.integers(-2 ** 31, 2 ** 31, 2).astype(np.int32)
        elif kind == ("f32", "mod") and len(shape) == 1:
            cap = [spec["cap"]] if name in capped and spec.get("cap") else []
            n = shape[0] - len(cap)
            out[name] = np.array(cap + [2.0 ** (-8.0 * (h + 1) / n) for h in range(n)], np.float32)
        elif kind == ("f32", "scale") and shape == (1,):
            out[name] = np.ones(1, np.float32)
        elif name in (tables or {}):
            out[name] = np.asarray(tables[name], np.float64).reshape(shape)
        elif v["dtype"] == "f64":
            half = shape[0] - 1
            out[name] = np.append(10000.0 ** (-np.arange(half) / half), 1.0)
        elif v["dtype"] == "f32":
            out[name] = g.standard_normal(shape, np.float32)
        elif v["dtype"] == "i32" and len(shape) == 2:
            out[name] = g.integers(0, spec["classes"], size=shape).astype(np.int32)
        elif v["dtype"] == "i32" and name.endswith("_len") and len(shapes.get(name[:-4], ())) == 2:
            out[name] = g.integers(1, shapes[name[:-4]][1] + 1, size=shape).astype(np.int32)
        elif v["dtype"] == "i32" and name.endswith("pos") and shape[0] % batch == 0:
            out[name] = (np.arange(shape[0]) % (shape[0] // batch)).astype(np.int32)
        else:
            raise ValueError(f"{name}: no synthetic values for {v['dtype']} {shape} of this name")
    return out


def make_params(spec, seed=1):
    """Initial parameters ``{name: float32 array}`` (He-normal fan-in, zero bias, BN 1/0)."""
    g = np.random.Generator(np.random.PCG64(seed))
    params = {}
    normal = spec.get("init") == "normal"
    for name, shape in param_shapes(spec):
        kind = name.rsplit(".", 1)[1]
        if normal and kind in ("W", "E", "pos"):
            params[name] = (g.standard_normal(size=shape, dtype=np.float32)
                            * np.float32(0.02)).astype(np.float32)
        elif kind == "W":
            fan_in = int(np.prod(shape[1:]))
            std = np.float32(np.sqrt(2.0 / fan_in))
            params[name] = (g.standard_normal(size=shape, dtype=np.float32) * std).astype(np.float32)
        elif kind in ("gamma", "gain", "post", "gate", "pre"):
            params[name] = np.ones(shape, np.float32)
        else:  # bias or beta
            params[name] = np.zeros(shape, np.float32)
    return params


def normal_pool(n, seed, threads=16):
    """``n`` standard-normal float32 values drawn by ``threads`` PCG64 streams spawned from
    ``SeedSequence(seed)``, stream i filling the i-th of ``threads`` equal blocks.  The same
    (n, seed, threads) gives the same array on any host.  Large full-size test inputs are
    windows of one such pool."""
    from concurrent.futures import ThreadPoolExecutor
    out = np.empty(n, np.float32)
    streams = np.random.SeedSequence(seed).spawn(threads)
    step = -(-n // threads)

    def fill(i):
        block = out[i * step:(i + 1) * step]
        if block.size:
            np.random.Generator(np.random.PCG64(streams[i])).standard_normal(
                size=block.size, dtype=np.float32, out=block)

    with ThreadPoolExecutor(threads) as ex:
        list(ex.map(fill, range(threads)))
    return out
