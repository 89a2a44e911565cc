"""The training-node operators in 64 bits (numpy), from their definitions: test infrastructure only.

Dropout by counter, layer norm, the attention softmax, the gated feed-forward and the
vocabulary's cross entropy with their gradients, and the norm over many arrays,
written as the formulas read, one array operation after another. Nothing here
is rounded to the operators' types.
"""
from __future__ import annotations

import math

import numpy as np


def draws(rows: int, cols: int, seed: int, site: int, row0: int = 0, group0: int = 0) -> np.ndarray:
    """16-bit draws [rows][cols]: half col % 2 of word col % 8 / 2 of Philox4x32-10 (key = seed, counter =
    (col / 8, row, site low, site high)); from row row0 and column 8 group0 on."""
    mask = np.uint64(0xFFFFFFFF)
    sh = np.uint64(32)
    groups = (cols + 7) // 8
    c = [np.broadcast_to(group0 + np.arange(groups, dtype=np.uint64), (rows, groups)),
         np.broadcast_to(row0 + np.arange(rows, dtype=np.uint64)[:, None], (rows, groups)),
         np.full((rows, groups), site & 0xFFFFFFFF, np.uint64), np.full((rows, groups), site >> 32, np.uint64)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> sh) ^ c[1] ^ np.uint64(k0), b & mask, (a >> sh) ^ c[3] ^ np.uint64(k1), a & mask]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    u = np.stack([(c[j // 2] >> np.uint64(16 * (j % 2))) & np.uint64(0xFFFF) for j in range(8)], -1)
    return u.reshape(rows, 8 * groups)[:, :cols].astype(np.int64)


def factors(rows: int, cols: int, seed: int, site: int, keep: int) -> np.ndarray:
    """What the dropout multiplies each element by: 65536 / keep, or 0."""
    return np.where(draws(rows, cols, seed, site) < keep, 65536.0 / max(keep, 1), 0.0)


def dropout(x, f, residual=None):
    """x, f [rows][cols]; a factor of 0 gives 0 whatever x is."""
    y = np.where(f > 0, x * np.where(f > 0, f, 1.0), 0.0)
    return y if residual is None else residual + y


def layer_norm(h, weight, bias, eps):
    """(y, mean, rstd)"""
    n = h.shape[1]
    mean = h.sum(1) / n
    var = ((h - mean[:, None]) ** 2).sum(1) / n
    rstd = 1.0 / np.sqrt(var + eps)
    return (h - mean[:, None]) * rstd[:, None] * weight + bias, mean, rstd


def layer_norm_backward(dy, h, mean, rstd, weight):
    """(dh, dweight, dbias)"""
    n = h.shape[1]
    xh = (h - mean[:, None]) * rstd[:, None]
    g = dy * weight
    dh = rstd[:, None] * (g - g.sum(1, keepdims=True) / n - xh * (g * xh).sum(1, keepdims=True) / n)
    return dh, (dy * xh).sum(0), dy.sum(0)


def visible(shape, causal=False, lengths=None, mask=None):
    """Truth values [batch][heads][queries][keys]: the keys each row sees. mask: 0 / nonzero, or added values."""
    B, H, Q, K = shape
    seen = np.ones(shape, bool)
    if lengths is not None:
        seen &= np.arange(K)[None, :] < np.asarray(lengths)[:, None, None, None]
    if causal:
        seen &= np.arange(K)[None, :] <= np.arange(Q)[:, None] + K - Q
    if mask is not None:
        seen &= np.broadcast_to(mask != 0 if mask.dtype.kind in "bu" else mask > -np.inf, shape)
    return seen


def logits(x, scale, seen, mask=None):
    add = 0.0 if mask is None or mask.dtype.kind in "bu" else mask
    with np.errstate(invalid="ignore"):
        return np.where(seen, x * scale + add, -np.inf)


def softmax(t):
    """(probabilities, largest logit, 1 / sum of exponentials) of logits; zeros for a row of -inf alone."""
    if t.shape[-1] == 0:
        return t, np.zeros(t.shape[:-1]), np.zeros(t.shape[:-1])
    m = t.max(-1)
    m = np.where(m == -np.inf, 0.0, m)
    e = np.exp(t - m[..., None])
    s = e.sum(-1)
    z = np.where(s == 0.0, 0.0, 1.0 / np.where(s == 0.0, 1.0, s))
    return e * z[..., None], m, z


def softmax_backward(g, p, scale):
    """The scores' gradient from the gradient g that reaches the probabilities p."""
    return scale * p * (g - (p * g).sum(-1, keepdims=True))


def activation(z, act):
    """(act(z), its derivative); act: silu, gelu or relu."""
    if act == "silu":
        s = 1.0 / (1.0 + np.exp(-z))
        return z * s, s * (1.0 + z * (1.0 - s))
    if act == "gelu":
        c = 0.5 * (1.0 + np.vectorize(math.erf, otypes=[float])(z / math.sqrt(2.0)))
        return z * c, c + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    return np.maximum(z, 0.0), (z > 0.0).astype(float)


def gated(x, w_gate, w_up, act):
    """h = act(x w_gate) * (x w_up)"""
    return activation(x @ w_gate, act)[0] * (x @ w_up)


def gated_backward(dh, x, w_gate, w_up, act):
    """(dx, dw_gate, dw_up)"""
    a, da = activation(x @ w_gate, act)
    dg, du = dh * (x @ w_up) * da, dh * a
    return dg @ w_gate.T + du @ w_up.T, x.T @ dg, x.T @ du


def cross_entropy(x, w, targets):
    """(loss, lse) of each row of x against the table w; a target outside it has loss 0."""
    t = x @ w.T
    m = t.max(1)
    lse = m + np.log(np.exp(t - m[:, None]).sum(1))
    some = (targets >= 0) & (targets < len(w))
    return np.where(some, lse - t[np.arange(len(x)), np.where(some, targets, 0)], 0.0), lse


def cross_entropy_backward(dloss, x, w, targets, lse):
    """(dx, dw)"""
    some = (targets >= 0) & (targets < len(w))
    d = np.exp(x @ w.T - lse[:, None])
    d[np.arange(len(x))[some], targets[some]] -= 1.0
    d = np.where(some[:, None], d * np.where(some, dloss, 0.0)[:, None], 0.0)
    return d @ w, d.T @ x


def norm(arrays):
    """The 2-norm over all elements of all arrays."""
    return math.sqrt(math.fsum(math.fsum(float(v) * float(v) for v in a.ravel()) for a in arrays))
