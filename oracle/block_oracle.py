"""fp64 statements of the operators around the expert layer: layer norm, the linear layer, the router's balance loss, AdamW.

Plain numpy, written from the formulas in include/grouter.h; nothing is rounded in between.  Test infrastructure only.
"""
from __future__ import annotations

import math

import numpy as np


# ---- layer norm ----
def layer_norm(x, w, b, eps):
    x = np.asarray(x, np.float64)
    mean = x.mean(1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    h = (x - mean[:, None]) * rstd[:, None]
    return h * w + (0.0 if b is None else b), mean, rstd


def layer_norm_backward(dy, x, w, mean, rstd):
    h = (np.asarray(x, np.float64) - mean[:, None]) * rstd[:, None]
    g = dy * w
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True) - h * (g * h).mean(1, keepdims=True))
    return dx, (dy * h).sum(0), dy.sum(0)


# ---- linear layer ----
def _sigmoid(z):
    e = np.exp(-np.abs(z))
    return np.where(z >= 0, 1.0 / (1.0 + e), e / (1.0 + e))


_G = math.sqrt(2.0 / math.pi)


def act(z, kind):
    if kind == "relu":
        return np.maximum(z, 0.0)
    if kind == "silu":
        return z * _sigmoid(z)
    if kind == "gelu":
        return 0.5 * z * (1.0 + np.tanh(_G * (z + 0.044715 * z ** 3)))
    return z


def act_slope(z, kind):
    if kind == "relu":
        return (z > 0).astype(np.float64)
    if kind == "silu":
        s = _sigmoid(z)
        return s * (1.0 + z * (1.0 - s))
    if kind == "gelu":
        t = np.tanh(_G * (z + 0.044715 * z ** 3))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * _G * (1.0 + 3 * 0.044715 * z * z)
    return np.ones_like(z)


def linear(x, W, b, r, kind):
    z = x @ W.T + (0.0 if b is None else b)
    return act(z, kind) + (0.0 if r is None else r), z


def linear_backward(dy, x, W, z, kind):
    dz = dy * act_slope(z, kind)
    return dz @ W, dz.T @ x, dz.sum(0), dz


# ---- router: counts, losses, gradient of the scores ----
def expert_counts(idx, E, mask=None):
    live = np.ones(idx.shape[0], bool) if mask is None else np.asarray(mask) != 0
    ids = idx[live].reshape(-1).astype(np.int64)
    ids = ids[(ids >= 0) & (ids < E)]
    return np.bincount(ids, minlength=E).astype(np.int64), int(live.sum())


def _softmax(s):
    top = s.max(1, keepdims=True)
    top = np.where(np.isfinite(top), top, 0.0)
    e = np.exp(s - top)
    total = e.sum(1, keepdims=True)
    some = total > 0
    p = np.where(some, e / np.where(some, total, 1.0), 0.0)
    lse = np.where(some, top + np.log(np.where(some, total, 1.0)), 0.0)[:, 0]
    return p, lse


def balance_loss(logits, counts, n, ca, cz, mask=None):
    """-> (loss, balance, z)"""
    live = np.ones(logits.shape[0], bool) if mask is None else np.asarray(mask) != 0
    if n == 0:
        return 0.0, 0.0, 0.0
    s = logits[live]
    p, lse = _softmax(s) if len(s) else (s, np.zeros(0))
    total = counts.sum()
    f = counts * (s.shape[1] / total) if total else np.zeros(len(counts))
    balance, z = (p @ f).sum() / n, (lse ** 2).sum() / n
    return (ca * balance if ca else 0.0) + (cz * z if cz else 0.0), balance, z


def balance_gradient(logits, counts, n, ca, cz, mask=None, idx=None, dgates=None, norm="softmax"):
    T, E = logits.shape
    live = np.ones(T, bool) if mask is None else np.asarray(mask) != 0
    out = np.zeros((T, E))
    total = counts.sum()
    f = counts * (E / total) if total else np.zeros(E)
    for t in range(T):
        if not live[t]:
            continue
        p, lse = _softmax(logits[t:t + 1])
        if n:
            out[t] = ca / n * p[0] * (f - (p[0] * f).sum()) + 2 * cz / n * lse[0] * p[0]
        if dgates is not None:
            s, dg = logits[t, idx[t].astype(np.int64)], dgates[t]
            q = gates(s[None], norm)[0]
            back = q * (dg - (q * dg).sum()) if norm == "softmax" else q * (1.0 - q) * dg
            for j, e in enumerate(idx[t]):
                out[t, int(e)] += back[j]
    return out


def gates(kept, norm):
    return _softmax(kept)[0] if norm == "softmax" else _sigmoid(kept)


# ---- AdamW and its 8-bit moments ----
def adamw(p, g, m, v, lr, b1, b2, eps, wd, step, scale=1.0):
    g = g * scale
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    mh, vh = m / (1 - b1 ** step), v / (1 - b2 ** step)
    return p * (1 - lr * wd) - lr * mh / (np.sqrt(vh) + eps), m, v


def e4m3_values():
    """The 127 finite magnitudes of e4m3, code 0 .. 126: 3 mantissa bits, exponent bias 7, subnormals below 2^-6."""
    out = []
    for code in range(127):
        e, f = code >> 3, code & 7
        out.append(f / 8.0 * 2.0 ** -6 if e == 0 else (1 + f / 8.0) * 2.0 ** (e - 7))
    return np.array(out)


def encode8(x, root):
    """Codes and exponent bytes of a flat array (a multiple of 32 finite values), by searching the nearest code."""
    vals = e4m3_values()
    x = np.asarray(x, np.float64)
    codes, exps = np.zeros(len(x), np.uint8), np.zeros(len(x) // 32, np.uint8)
    for b in range(len(x) // 32):
        blk = x[32 * b:32 * b + 32]
        top = np.abs(blk).max()
        e = -126
        while top > 448.0 * 2.0 ** e and e < 126:
            e += 1
        exps[b] = e + 127
        for i, val in enumerate(blk):
            a = abs(val) * 2.0 ** -e
            d = np.abs(vals - a)
            near = np.flatnonzero(d == d.min())
            c = int(near[0]) if len(near) == 1 else int([k for k in near if k % 2 == 0][0])      # a tie goes to the even code
            if root and c == 0 and val > 0:
                c = 1
            codes[32 * b + i] = c | (0x80 if np.signbit(val) else 0)
    return codes, exps


def decode8(codes, exps):
    vals = np.concatenate([e4m3_values(), [np.nan]])
    v = vals[codes & 0x7F] * np.where(codes & 0x80, -1.0, 1.0)
    return v * np.repeat(2.0 ** (exps.astype(np.float64) - 127), 32)
