"""fp64 statements of the dense gated branch: root-mean-square norm, matrices in 8 bits, products on them, the gated feed-forward block.

Plain numpy, written from the formulas in include/grouter.h; nothing is rounded but what the definition puts into 8 bits.  Test
infrastructure only.
"""
from __future__ import annotations

import numpy as np

from oracle.block_oracle import act, act_slope

BLOCK = 128


# ---- root-mean-square norm ----
def rms_norm(h, w, eps):
    h = np.asarray(h, np.float64)
    rstd = 1.0 / np.sqrt((h * h).mean(1) + eps)
    return h * rstd[:, None] * w, rstd


def rms_norm_backward(dy, h, w, rstd, dh=None):
    u = np.asarray(h, np.float64) * rstd[:, None]
    g = dy * w
    dx = rstd[:, None] * (g - u * (g * u).mean(1, keepdims=True))
    return dx + (0.0 if dh is None else dh), (dy * u).sum(0)


# ---- 8 bits ----
def _e4m3_numbers():
    """The 127 numbers of e4m3 that are not negative, in the order of their codes: 3 bits of mantissa, exponent bias 7."""
    m, e = np.arange(8), np.arange(16)
    v = np.where(e[:, None] == 0, m * 2.0 ** -9, (1 + m / 8.0) * 2.0 ** (e[:, None] - 7.0)).reshape(-1)
    return v[:-1]                                          # the last code is NaN


NUMBERS = _e4m3_numbers()


def e4m3(v):
    """v rounded to the nearest of them, ties to the even code; |v| <= 448; what is not finite becomes NaN."""
    a = np.abs(v)
    ok = np.isfinite(a)
    a = np.where(ok, a, 0.0)
    hi = np.clip(np.searchsorted(NUMBERS, a), 1, len(NUMBERS) - 1)
    lo = hi - 1
    mid = (NUMBERS[lo] + NUMBERS[hi]) / 2
    up = (a > mid) | ((a == mid) & (hi % 2 == 0))
    return np.where(ok, np.copysign(np.where(up, NUMBERS[hi], NUMBERS[lo]), v), np.nan)


def exponent(top):
    """The smallest e >= -126 with top <= 448 * 2^e."""
    e = np.full(np.shape(top), -126, np.int64)
    t = np.maximum(np.asarray(top, np.float64), 1e-300)
    e = np.maximum(e, np.ceil(np.log2(t / 448.0)).astype(np.int64))
    e = np.where((e > -126) & (t <= 448.0 * 2.0 ** (e - 1)), e - 1, e)
    return np.where(t > 448.0 * 2.0 ** e, e + 1, e)


def exponents(x, square=False):
    """[rows, blocks of 128] of a matrix."""
    x = np.asarray(x, np.float64)
    R, C = x.shape
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    a = np.pad(a, ((0, -R % BLOCK if square else 0), (0, -C % BLOCK)))
    top = a.reshape(a.shape[0], -1, BLOCK).max(2)
    if square:
        top = top.reshape(-1, BLOCK, top.shape[1]).max(1).repeat(BLOCK, 0)[:R]
    return exponent(top)


def quantized(x, square=False, exps=None):
    """What 8 bits hold of x (values, exponents)."""
    e = exponents(x, square) if exps is None else exps
    s = 2.0 ** np.repeat(e, BLOCK, 1)[:, :np.shape(x)[1]].astype(np.float64)
    return e4m3(np.asarray(x, np.float64) / s) * s, e


# ---- gated feed-forward block ----
def gated(x, Wg, Wu, kind):
    g, u = x @ Wg.T, x @ Wu.T
    return act(g, kind) * u, g, u


def gated_backward(dy, x, Wg, Wu, Wd, g, u, kind):
    """-> dx, dW_gu, dW_d, and dg, du, h."""
    dh, a = dy @ Wd, act(g, kind)
    dg, du, h = dh * u * act_slope(g, kind), dh * a, a * u
    return dg @ Wg + du @ Wu, np.concatenate([dg.T @ x, du.T @ x]), dy.T @ h, dg, du, h
