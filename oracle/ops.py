"""Textbook forward, backward and SGD of every layer kind, in NumPy (test infrastructure).

The paper trains ordinary networks (ResNet-50 and others, Section 5); it
fixes none of these formulas, so each is the standard definition, computed in
the dtype of its inputs (float64 for parity).  Layouts follow the library
boundary: images NHWC, conv weights [K, R, S, C], dense weights [out, in].

* dense:        Y = X W^T + b
* conv:         cross-correlation with zero padding,
                Y[n,p,q,k] = sum_{r,s,c} Xpad[n, p*st + r, q*st + s, c] W[k,r,s,c]
* BatchNorm:    training mode, batch mean and biased variance over N, H, W,
                eps = 1e-5, y = gamma * (x - mean) / sqrt(var + eps) + beta
* ReLU:         y = max(x, 0); backward through the output: dx = dy * [y > 0]
* max pool:     window max over valid taps; ties go to the first tap in
                row-major window order; backward routes dy to that tap
* global average pool over H, W
* softmax cross-entropy, mean over the batch
* SGD:          w -= lr g;  with momentum mu: v = mu v + g, w -= lr v
* LayerNorm:    per row over the features, biased variance, eps = 1e-5
* GELU:         exact, x Phi(x) with the normal CDF Phi
* attention:    per batch and head, P = softmax(q k^T / sqrt(dh)) with future
                positions masked (causal), context = P v; q, k, v are the
                column thirds of one [rows, 3 d] projection, head h owning
                columns h dh .. (h + 1) dh of each third
* rotation:     the pair (x0, x1) of a head's columns, as x0 + i x1, times m e^(i pos f)
* head norm:    per row and head, gain x / sqrt(mean x^2 + eps), eps = 1e-5, then the rotation
* cross attention: per sequence and head, softmax(q k^T / sqrt(dh)) v over the first klen
                states; no states: zero; query head h reads key head h Hkv / H
* embedding:    x[b, t] = E[id[b, t]] + pos[t]
* concat:       channel (last axis) concatenation; its backward hands each input
                its own channel range of the output gradient
* upsample:     nearest, factor 2: y[n, 2h + i, 2w + j] = x[n, h, w]; backward sums
                each 2 x 2 block of the output gradient
"""

from __future__ import annotations

import numpy as np
from scipy.special import erfc

BN_EPS = 1e-5
LN_EPS = 1e-5


# ---------------------------------------------------------------- dense
def linear_fwd(X, W, b):
    return X @ W.T + b


def linear_bwd_w(X, dY):
    """dW = dY^T X, db = sum_n dY."""
    return dY.T @ X, dY.sum(axis=0)


def linear_bwd_x(W, dY):
    """dX = dY W."""
    return dY @ W


# ---------------------------------------------------------------- conv
def _out_size(h, k, stride, pad):
    return (h + 2 * pad - k) // stride + 1


def conv_fwd(X, Wt, stride, pad):
    N, H, Wd, C = X.shape
    K, R, S, C2 = Wt.shape
    assert C == C2
    P, Q = _out_size(H, R, stride, pad), _out_size(Wd, S, stride, pad)
    Xp = np.pad(X, ((0, 0), (pad, pad), (pad, pad), (0, 0)))
    Y = np.zeros((N, P, Q, K), dtype=X.dtype)
    for r in range(R):
        for s in range(S):
            tap = Xp[:, r:r + stride * (P - 1) + 1:stride, s:s + stride * (Q - 1) + 1:stride, :]
            Y += tap @ Wt[:, r, s, :].T
    return Y


def conv_bwd_x(Wt, dY, x_shape, stride, pad):
    """dX: every output gradient is sent back through the tap that produced it."""
    N, H, Wd, C = x_shape
    K, R, S, _ = Wt.shape
    _, P, Q, _ = dY.shape
    dXp = np.zeros((N, H + 2 * pad, Wd + 2 * pad, C), dtype=dY.dtype)
    for r in range(R):
        for s in range(S):
            dXp[:, r:r + stride * (P - 1) + 1:stride, s:s + stride * (Q - 1) + 1:stride, :] += \
                dY @ Wt[:, r, s, :]
    return dXp[:, pad:pad + H, pad:pad + Wd, :]


def conv_bwd_w(X, dY, w_shape, stride, pad):
    """dW[k,r,s,c] = sum_{n,p,q} dY[n,p,q,k] Xpad[n, p*st + r, q*st + s, c]."""
    K, R, S, C = w_shape
    _, P, Q, _ = dY.shape
    Xp = np.pad(X, ((0, 0), (pad, pad), (pad, pad), (0, 0)))
    dW = np.zeros(w_shape, dtype=dY.dtype)
    for r in range(R):
        for s in range(S):
            tap = Xp[:, r:r + stride * (P - 1) + 1:stride, s:s + stride * (Q - 1) + 1:stride, :]
            dW[:, r, s, :] = np.tensordot(dY, tap, axes=([0, 1, 2], [0, 1, 2]))
    return dW


# ---------------------------------------------------------------- BatchNorm
def bn_fwd(X, gamma, beta):
    """Returns (Y, mean, invstd); statistics over every axis but the channel (last) one."""
    axes = tuple(range(X.ndim - 1))
    mean = X.mean(axis=axes)
    var = ((X - mean) ** 2).mean(axis=axes)
    invstd = 1.0 / np.sqrt(var + BN_EPS)
    xhat = (X - mean) * invstd
    return gamma * xhat + beta, mean, invstd


def bn_bwd(X, gamma, mean, invstd, dY):
    """Returns (dX, dgamma, dbeta) of the training-mode normalisation."""
    axes = tuple(range(X.ndim - 1))
    m = X.size // X.shape[-1]
    xhat = (X - mean) * invstd
    dbeta = dY.sum(axis=axes)
    dgamma = (dY * xhat).sum(axis=axes)
    dX = gamma * invstd / m * (m * dY - dbeta - xhat * dgamma)
    return dX, dgamma, dbeta


# ---------------------------------------------------------------- ReLU
def relu_fwd(X):
    return np.maximum(X, 0)


def relu_bwd(Y, dY):
    return dY * (Y > 0)


# ---------------------------------------------------------------- pooling
def maxpool_fwd(X, k, stride, pad):
    """Returns (Y, idx): idx = r*k + s of the first maximal valid tap (uint8)."""
    N, H, Wd, C = X.shape
    P, Q = _out_size(H, k, stride, pad), _out_size(Wd, k, stride, pad)
    Y = np.full((N, P, Q, C), -np.inf, dtype=X.dtype)
    idx = np.zeros((N, P, Q, C), dtype=np.uint8)
    for p in range(P):
        for q in range(Q):
            for r in range(k):
                for s in range(k):
                    h, w = p * stride + r - pad, q * stride + s - pad
                    if 0 <= h < H and 0 <= w < Wd:
                        v = X[:, h, w, :]
                        better = v > Y[:, p, q, :]
                        Y[:, p, q, :] = np.where(better, v, Y[:, p, q, :])
                        idx[:, p, q, :] = np.where(better, r * k + s, idx[:, p, q, :])
    return Y, idx


def maxpool_bwd(idx, dY, x_shape, k, stride, pad):
    N, H, Wd, C = x_shape
    _, P, Q, _ = dY.shape
    dX = np.zeros(x_shape, dtype=dY.dtype)
    for p in range(P):
        for q in range(Q):
            for r in range(k):
                for s in range(k):
                    h, w = p * stride + r - pad, q * stride + s - pad
                    if 0 <= h < H and 0 <= w < Wd:
                        dX[:, h, w, :] += np.where(idx[:, p, q, :] == r * k + s, dY[:, p, q, :], 0)
    return dX


def avgpool_fwd(X):
    return X.mean(axis=(1, 2))


def avgpool_bwd(dY, x_shape):
    N, H, Wd, C = x_shape
    return np.broadcast_to(dY[:, None, None, :] / (H * Wd), x_shape).copy()


# ---------------------------------------------------------------- loss
def softmax_ce(logits, labels):
    """Returns (per-row losses, mean loss, dlogits) of the mean softmax cross-entropy."""
    N = logits.shape[0]
    z = logits - logits.max(axis=1, keepdims=True)
    lse = np.log(np.exp(z).sum(axis=1))
    rows = lse - z[np.arange(N), labels]
    prob = np.exp(z - lse[:, None])
    onehot = np.zeros_like(prob)
    onehot[np.arange(N), labels] = 1.0
    return rows, rows.mean(), (prob - onehot) / N


# ---------------------------------------------------------------- update
def sgd(w, g, lr):
    return w - lr * g


def sgd_momentum(w, g, v, lr, mu):
    v_new = mu * v + g
    return w - lr * v_new, v_new


# ---------------------------------------------------------------- LayerNorm
def layernorm_fwd(X, gamma, beta):
    """Returns (Y, mean, rstd) over the last axis."""
    mean = X.mean(axis=-1, keepdims=True)
    var = ((X - mean) ** 2).mean(axis=-1, keepdims=True)
    rstd = 1.0 / np.sqrt(var + LN_EPS)
    return (X - mean) * rstd * gamma + beta, mean[..., 0], rstd[..., 0]


def layernorm_bwd(X, gamma, mean, rstd, dY):
    """Returns (dX, dgamma, dbeta)."""
    xhat = (X - mean[..., None]) * rstd[..., None]
    g = dY * gamma
    dX = rstd[..., None] * (g - g.mean(axis=-1, keepdims=True)
                            - xhat * (g * xhat).mean(axis=-1, keepdims=True))
    return dX, (dY * xhat).sum(axis=0), dY.sum(axis=0)


# ---------------------------------------------------------------- GELU
def _normal_cdf(X):
    """Phi(x) = erfc(-x / sqrt 2) / 2; the erfc form keeps full relative precision in the
    lower tail, where 1 + erf(x / sqrt 2) cancels."""
    return 0.5 * erfc(-X / np.sqrt(2.0))


def gelu_fwd(X):
    return X * _normal_cdf(X)


def gelu_bwd(X, dY):
    cdf = _normal_cdf(X)
    pdf = np.exp(-0.5 * X * X) / np.sqrt(2.0 * np.pi)
    return dY * (cdf + X * pdf)


# ---------------------------------------------------------------- attention
def _heads(qkv, B, T, H):
    """Split [B T, 3 d] into q, k, v of shape [B, H, T, dh]."""
    d = qkv.shape[1] // 3
    dh = d // H
    t = qkv.reshape(B, T, 3, H, dh)
    return t[:, :, 0].transpose(0, 2, 1, 3), t[:, :, 1].transpose(0, 2, 1, 3), \
        t[:, :, 2].transpose(0, 2, 1, 3)


def attention_fwd(qkv, B, T, H, causal=True):
    """Returns (P [B, H, T, T], context [B T, d])."""
    q, k, v = _heads(qkv, B, T, H)
    dh = q.shape[-1]
    S = q @ k.transpose(0, 1, 3, 2) / np.sqrt(dh)
    if causal:
        S = np.where(np.tril(np.ones((T, T), dtype=bool)), S, -np.inf)
    S = S - S.max(axis=-1, keepdims=True)
    P = np.exp(S)
    P /= P.sum(axis=-1, keepdims=True)
    ctx = P @ v                                    # [B, H, T, dh]
    return P, ctx.transpose(0, 2, 1, 3).reshape(B * T, H * dh)


def attention_bwd(qkv, P, dctx, B, T, H):
    """Returns dqkv [B T, 3 d] for context = softmax(q k^T / sqrt(dh)) v."""
    q, k, v = _heads(qkv, B, T, H)
    dh = q.shape[-1]
    dO = dctx.reshape(B, T, H, dh).transpose(0, 2, 1, 3)
    dv = P.transpose(0, 1, 3, 2) @ dO
    dP = dO @ v.transpose(0, 1, 3, 2)
    dS = P * (dP - (dP * P).sum(axis=-1, keepdims=True)) / np.sqrt(dh)
    dq = dS @ k
    dk = dS.transpose(0, 1, 3, 2) @ q
    out = np.stack([dq, dk, dv], axis=2)           # [B, H, 3, T, dh]
    return out.transpose(0, 3, 2, 1, 4).reshape(B * T, 3 * H * dh)


# ---------------------------------------------------------------- embedding
def embed_fwd(ids, E, pos):
    B, T = ids.shape
    return (E[ids] + pos[None, :T]).reshape(B * T, E.shape[1])


def concat_fwd(Xs):
    return np.concatenate(Xs, axis=-1)


def concat_bwd(dY, channels):
    edges = np.cumsum([0] + list(channels))
    return [dY[..., edges[j]:edges[j + 1]].copy() for j in range(len(channels))]


def upsample_fwd(X):
    return X.repeat(2, axis=1).repeat(2, axis=2)


def upsample_bwd(dY):
    N, H2, W2, C = dY.shape
    return dY.reshape(N, H2 // 2, 2, W2 // 2, 2, C).sum(axis=(2, 4))


def embed_bwd(ids, dX, vocab):
    B, T = ids.shape
    d = dX.shape[1]
    dE = np.zeros((vocab, d), dtype=dX.dtype)
    np.add.at(dE, ids.reshape(-1), dX)
    return dE, dX.reshape(B, T, d).sum(axis=0)


# ---------------------------------------------------------------- rotary positions, head norms
def _pairs(rot, layout):
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if layout == 0 else (i, i + rot // 2)


def _rotate(heads, pos, table, rot, layout, back):
    """heads [rows, n, dh] with their pairs turned by pos * table."""
    a = np.asarray(pos, np.float64)[:, None] * table[:-1]
    w = table[-1] * np.exp(1j * (-a if back else a))[:, None, :]
    i0, i1 = _pairs(rot, layout)
    z = (heads[..., i0] + 1j * heads[..., i1]) * w
    out = heads.copy()
    out[..., i0], out[..., i1] = z.real, z.imag
    return out


def rope(X, pos, table, a, back=False):
    n = a["heads"] * a["dh"]
    out = X.copy()
    h = X[:, :n].reshape(len(X), a["heads"], a["dh"])
    out[:, :n] = _rotate(h, pos, table, a["rot"], a["layout"], back).reshape(len(X), n)
    return out


def _head_gain(gain, a):
    return gain[(np.arange(a["h1"] + a["h2"]) >= a["h1"]).astype(int)]


def qknorm_fwd(X, gain, pos=None, table=None, *, a):
    heads = a["h1"] + a["h2"]
    n = heads * a["dh"]
    h = X[:, :n].reshape(len(X), heads, a["dh"])
    y = _head_gain(gain, a) * h / np.sqrt((h * h).mean(-1, keepdims=True) + LN_EPS)
    if a["rot"]:
        y = _rotate(y, pos, table, a["rot"], a["layout"], False)
    out = X.copy()
    out[:, :n] = y.reshape(len(X), n)
    return out


def qknorm_bwd(X, gain, dY, pos=None, table=None, *, a):
    """Returns (dX, dgain)."""
    heads = a["h1"] + a["h2"]
    n = heads * a["dh"]
    h = X[:, :n].reshape(len(X), heads, a["dh"])
    z = dY[:, :n].reshape(len(X), heads, a["dh"])
    if a["rot"]:
        z = _rotate(z, pos, table, a["rot"], a["layout"], True)
    r = 1.0 / np.sqrt((h * h).mean(-1, keepdims=True) + LN_EPS)
    u = h * r
    per_head = (z * u).sum(0)
    dgain = np.stack([per_head[s].sum(0) for s in ([slice(0, a["h1"])] +
                     ([slice(a["h1"], None)] if a["h2"] else []))])
    w = _head_gain(gain, a) * z
    out = dY.copy()
    out[:, :n] = (r * (w - u * (w * u).mean(-1, keepdims=True))).reshape(len(X), n)
    return out, dgain


# ---------------------------------------------------------------- cross attention
def _cross_parts(q, kv, a):
    B, Tq, Tk, H, Hkv, dh = (a[k] for k in ("B", "Tq", "Tk", "H", "Hkv", "dh"))
    k, v = kv.reshape(B, Tk, 2, Hkv, dh).transpose(2, 0, 3, 1, 4)
    return q.reshape(B, Tq, H, dh).transpose(0, 2, 1, 3), k, v, H // Hkv


def _cross_probs(q, k, n):
    """(P, lse) of one head over its first n keys (n >= 1)."""
    S = q @ k[:n].T / np.sqrt(q.shape[-1])
    top = S.max(-1, keepdims=True)
    e = np.exp(S - top)
    total = e.sum(-1, keepdims=True)
    return e / total, (top + np.log(total))[:, 0]


def cross_attention_fwd(q, kv, klen, a):
    """Returns (Y [B Tq, H dh], lse [B, H, Tq])."""
    Q, K, V, G = _cross_parts(q, kv, a)
    Y, lse = np.zeros_like(Q), np.full(Q.shape[:3], -np.inf)
    for b in range(a["B"]):
        n = int(klen[b])
        for h in range(a["H"] if n else 0):
            P, lse[b, h] = _cross_probs(Q[b, h], K[b, h // G], n)
            Y[b, h] = P @ V[b, h // G, :n]
    return Y.transpose(0, 2, 1, 3).reshape(q.shape), lse


def cross_attention_bwd(q, kv, klen, dY, a):
    """Returns (dq, dkv, delta [B, H, Tq])."""
    Q, K, V, G = _cross_parts(q, kv, a)
    g = dY.reshape(a["B"], a["Tq"], a["H"], a["dh"]).transpose(0, 2, 1, 3)
    dQ, dK, dV = np.zeros_like(Q), np.zeros_like(K), np.zeros_like(V)
    delta = np.zeros(Q.shape[:3])
    scale = 1.0 / np.sqrt(a["dh"])
    for b in range(a["B"]):
        n = int(klen[b])
        for h in range(a["H"] if n else 0):
            j = h // G
            P, _ = _cross_probs(Q[b, h], K[b, j], n)
            dP = g[b, h] @ V[b, j, :n].T
            delta[b, h] = (P * dP).sum(-1)
            dS = P * (dP - delta[b, h][:, None]) * scale
            dQ[b, h] = dS @ K[b, j, :n]
            dK[b, j, :n] += dS.T @ Q[b, h]
            dV[b, j, :n] += P.T @ g[b, h]
    dkv = np.stack([dK, dV]).transpose(1, 3, 0, 2, 4).reshape(kv.shape)
    return dQ.transpose(0, 2, 1, 3).reshape(q.shape), dkv, delta


# ---------------------------------------------------------------- dropout
def philox(counters, salt, seed):
    """The four words [n, 4] of Philox 4x32-10 (Salmon et al., 2011) at each counter of 64 bits, its
    upper half being ``salt``, under the key ``seed`` (two uint32)."""
    low = np.uint64(0xFFFFFFFF)
    i = np.asarray(counters, np.uint64)
    c = [i & low, i >> np.uint64(32), np.full_like(i, int(salt) & 0xFFFFFFFF),
         np.full_like(i, int(salt) >> 32)]
    key = [int(np.uint32(k)) for k in np.asarray(seed).astype(np.uint32)]
    for r in range(10):
        k = [np.uint64((key[0] + r * 0x9E3779B9) & 0xFFFFFFFF),
             np.uint64((key[1] + r * 0xBB67AE85) & 0xFFFFFFFF)]
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> np.uint64(32)) ^ c[1] ^ k[0], q & low, (p >> np.uint64(32)) ^ c[3] ^ k[1], p & low]
    return np.stack(c, -1).astype(np.uint32)


def dropout_factor(shape, seed, a):
    """What each value of a tensor is multiplied by: 0, or 1 / (1 - drop / 2^32)."""
    n = int(np.prod(shape))
    if not a["drop"]:
        return np.ones(shape)
    words = philox(np.arange((n + 3) // 4), a["salt"], seed).reshape(-1)[:n]
    return ((words >= a["drop"]) / (1.0 - a["drop"] / 2.0 ** 32)).reshape(shape)


def dropout(X, seed, a):
    m = dropout_factor(X.shape, seed, a)
    return np.where(m > 0, X * m, 0.0)


# ---------------------------------------------------------------- a block's join
def _gate_rows(gate, rows):
    return np.repeat(gate, rows // len(gate), 0)


def join_fwd(X, F, post, gate, pre, scale, a, seed=None):
    """Returns (H, N, stats [rows, 2])."""
    r = 1.0 / np.sqrt((F * F).mean(-1, keepdims=True) + LN_EPS)
    w = dropout(post * F * r, seed, a)
    H = scale * X + _gate_rows(gate, len(X)) * w
    s = 1.0 / np.sqrt((H * H).mean(-1, keepdims=True) + LN_EPS)
    return H, pre * H * s, np.concatenate([r, s], 1)


def join_bwd(F, H, post, gate, pre, scale, dH, dN, a, seed=None):
    """Returns (dX, dF, dpost, dgate, dpre); dH may be None."""
    rows, d = F.shape
    g = _gate_rows(gate, rows)
    r = 1.0 / np.sqrt((F * F).mean(-1, keepdims=True) + LN_EPS)
    s = 1.0 / np.sqrt((H * H).mean(-1, keepdims=True) + LN_EPS)
    m = dropout_factor(F.shape, seed, a)
    v, t = F * r, H * s
    dt = pre * dN
    dh = s * (dt - t * (dt * t).mean(-1, keepdims=True)) + (0.0 if dH is None else dH)
    du = g * dh * m
    dv = post * du
    dF = r * (dv - v * (dv * v).mean(-1, keepdims=True))
    dgate = (dh * post * v * m).reshape(len(gate), -1, d).sum(1)
    return scale * dh, dF, (du * v).sum(0), dgate, (dN * t).sum(0)


# ---------------------------------------------------------------- gated recurrence
def _gates(FX, fresh, a):
    f, x = FX.reshape(a["B"], a["T"], 2, a["C"]).transpose(2, 0, 1, 3)
    gate, rest = (1.0 / (1.0 + np.exp(-np.clip(s * f, -700, None))) for s in (1, -1))
    live = np.ones((a["B"], a["T"], 1)) if fresh is None else \
        (np.asarray(fresh).reshape(a["B"], a["T"], 1) == 0).astype(np.float64)
    return x, gate, rest, live


def _cut(gate, live):
    """Rows that start afresh, and gates that are 0 in fp32: the state before does not count, whatever it
    holds."""
    return (live == 0) | (gate.astype(np.float32) == 0)


def _passed(gate, live, state):
    """What a row takes of the state before it."""
    with np.errstate(invalid="ignore"):
        return np.where(_cut(gate, live), 0.0, gate * state)


def scan_fwd(FX, a, h0=None, fresh=None):
    x, gate, rest, live = _gates(FX, fresh, a)
    H, state = np.zeros(x.shape), np.zeros(x[:, 0].shape) if h0 is None else h0
    for t in range(a["T"]):
        state = _passed(gate[:, t], live[:, t], state) + rest[:, t] * x[:, t]
        H[:, t] = state
    return H.reshape(-1, a["C"])


def scan_bwd(FX, H, dH, a, h0=None, fresh=None):
    """Returns (dFX, dh0)."""
    x, gate, rest, live = _gates(FX, fresh, a)
    H, dH = H.reshape(x.shape), dH.reshape(x.shape)
    first = np.zeros(x[:, :1].shape) if h0 is None else h0[:, None]
    before = np.where(_cut(gate, live), 0.0, np.concatenate([first, H[:, :-1]], 1))
    g, later = np.zeros(x.shape), np.zeros(x[:, 0].shape)
    for t in range(a["T"] - 1, -1, -1):
        g[:, t] = dH[:, t] + later
        later = _passed(gate[:, t], live[:, t], g[:, t])
    dFX = np.stack([g * (before - x) * gate * rest, g * rest], 2)
    return dFX.reshape(FX.shape), later


# ---------------------------------------------------------------- attention to a span of states
def _span_scores(q, k, span, head, a, mod):
    """(scores with -inf where nothing is seen, what the cap multiplies their gradients by)."""
    S = q @ k.T / np.sqrt(a["dh"])
    turn = 1.0
    mod = np.asarray([] if mod is None else mod, np.float64)
    if a["cap"]:
        t = np.tanh(S / mod[0])
        S, turn = mod[0] * t, 1.0 - t * t
    lo, hi, at = np.asarray(span, np.int64)[:, :, None].transpose(1, 0, 2)
    j = np.arange(a["Tk"])
    if a["bias"]:
        S = S - mod[a["cap"] + head] * np.abs(at - j)
    return np.where((j >= lo) & (j < hi), S, -np.inf), turn


def _span_probs(S):
    top = S.max(-1, keepdims=True)
    none = top == -np.inf
    e = np.exp(S - np.where(none, 0.0, top))
    total = e.sum(-1, keepdims=True)
    with np.errstate(divide="ignore"):
        return e / np.where(none, 1.0, total), (np.where(none, -np.inf, top + np.log(total)))[:, 0]


def span_attention_fwd(q, kv, span, a, mod=None):
    """Returns (Y [B Tq, H dh], lse [B, H, Tq])."""
    Q, K, V, G = _cross_parts(q, kv, a)
    Y, lse = np.zeros_like(Q), np.zeros(Q.shape[:3])
    sp = np.asarray(span).reshape(a["B"], a["Tq"], 3)
    for b in range(a["B"]):
        for h in range(a["H"]):
            P, lse[b, h] = _span_probs(_span_scores(Q[b, h], K[b, h // G], sp[b], h, a, mod)[0])
            Y[b, h] = P @ V[b, h // G]
    return Y.transpose(0, 2, 1, 3).reshape(q.shape), lse


def span_attention_bwd(q, kv, span, dY, a, mod=None):
    """Returns (dq, dkv, delta [B, H, Tq])."""
    Q, K, V, G = _cross_parts(q, kv, a)
    g = dY.reshape(a["B"], a["Tq"], a["H"], a["dh"]).transpose(0, 2, 1, 3)
    dQ, dK, dV = np.zeros_like(Q), np.zeros_like(K), np.zeros_like(V)
    delta = np.zeros(Q.shape[:3])
    sp = np.asarray(span).reshape(a["B"], a["Tq"], 3)
    for b in range(a["B"]):
        for h in range(a["H"]):
            j = h // G
            S, turn = _span_scores(Q[b, h], K[b, j], sp[b], h, a, mod)
            P, _ = _span_probs(S)
            dP = g[b, h] @ V[b, j].T
            delta[b, h] = (P * dP).sum(-1)
            dS = P * (dP - delta[b, h][:, None]) * turn / np.sqrt(a["dh"])
            dQ[b, h] = dS @ K[b, j]
            dK[b, j] += dS.T @ Q[b, h]
            dV[b, j] += P.T @ g[b, h]
    dkv = np.stack([dK, dV]).transpose(1, 3, 0, 2, 4).reshape(kv.shape)
    return dQ.transpose(0, 2, 1, 3).reshape(q.shape), dkv, delta
