"""Gradients against differences of the forward pass, for the gated block and the norm, with bounds tight enough that a gradient without one of its
terms is outside them.  The passes are arguments: kernels, or plain statements of the same roundings with a mistake planted in them.

The derivative of f = sum(y dy) along a direction v is taken twice, as sum(gradient v) and as (f(p + s v) - f(p - s v)) / 2s.  v holds the
signs of the gradient that fp64 gives, so that the derivative is the sum of its magnitudes and a term that is left out takes its share of it
away; and then the signs of the gradient under test, along which a term too many adds its own.  (Along a direction of any other kind the terms
cancel one another, and what is left is no larger than what their roundings come to.)  The points p + s v are numbers of the type exactly.  What the two may differ by:
  rounding    bf16: every rounding is off by at most 2^-8 of its value, is as often up as down and independent of the others, so of variance
              (2^-8 value)^2 / 3 at most; the sum over all of them is within eight standard deviations.  f32: by the sum of their largest values.
  truncation  what the same difference in fp64 is off by at this step, taken from two steps (of the forward pass alone, no gradient)
"""
import numpy as np

from oracle import branch_oracle as orc
from oracle.block_oracle import act, act_slope

R = 2.0 ** -8


def truncation(f, s):
    """f(t) along the direction -> |difference at s - difference at a step whose third-order term is nothing|."""
    d = lambda t: (f(t) - f(-t)) / (2 * t)  # noqa: E731
    return abs(d(s) - d(s * 2.0 ** -10))


def grid(rng, shape, most, unit):
    """Whole numbers up to `most` times a power of two."""
    return rng.integers(-most, most + 1, shape).astype(np.float64) * unit


class Gated:
    """One block on grids, small enough for fp64: its tensors p = dict(x, Wg, Wu, Wd) and the gradient's dy."""

    def __init__(self, T, kind, seed=0, d=128, H=136):
        rng = np.random.default_rng(seed + T)
        self.T, self.kind = T, kind
        self.p = dict(x=grid(rng, (T, d), 12, 2.0 ** -3), Wg=grid(rng, (H, d), 12, 2.0 ** -6), Wu=grid(rng, (H, d), 12, 2.0 ** -6),
                      Wd=grid(rng, (d, H), 12, 2.0 ** -6))
        # f is linear in Wu and Wd: longer steps, over which the forward pass's roundings count for less
        self.step = dict(x=2.0 ** -4, Wg=2.0 ** -7, Wu=2.0 ** -5, Wd=2.0 ** -5)
        self.dy = grid(rng, (T, d), 12, 2.0 ** -3)

    def f64(self, p):
        return float(((orc.gated(p["x"], p["Wg"], p["Wu"], self.kind)[0] @ p["Wd"].T) * self.dy).sum())

    def forward_noise(self, p):
        """Variance of f at a point: y and h are rounded to bf16."""
        h = orc.gated(p["x"], p["Wg"], p["Wu"], self.kind)[0]
        dh = self.dy @ p["Wd"]
        return R * R / 3 * (np.square(h @ p["Wd"].T * self.dy).sum() + np.square(h * dh).sum())

    def gradient_noise(self, name, v, grad):
        """Variance of sum(gradient v): the gradient itself (bf16), dg, du and h on their way into it, the saved g and u they are formed from."""
        p = self.p
        h, g, u = orc.gated(p["x"], p["Wg"], p["Wu"], self.kind)
        a, s, dh = act(g, self.kind), act_slope(g, self.kind), self.dy @ p["Wd"]
        total = np.square(grad * v).sum()
        if name == "Wd":                                   # h formed again from g and u
            e = self.dy @ v
            terms = (h * e, s * u * e * g, a * e * u)
        else:
            vg = v @ p["Wg"].T if name == "x" else p["x"] @ v.T if name == "Wg" else 0.0 * g
            vu = v @ p["Wu"].T if name == "x" else p["x"] @ v.T if name == "Wu" else 0.0 * g
            bend = 0.0 if self.kind == "none" else 1.2     # no activation's second derivative is above it
            terms = (dh * u * s * vg, dh * a * vu, dh * (np.abs(u * bend * vg) + np.abs(s * vu)) * g, dh * s * vg * u)
        return R * R / 3 * (total + sum(np.square(t).sum() for t in terms))

    def gradient(self, name):
        p = self.p
        _, g, u = orc.gated(p["x"], p["Wg"], p["Wu"], self.kind)
        dx, dWgu, dWd, _, _, _ = orc.gated_backward(self.dy, p["x"], p["Wg"], p["Wu"], p["Wd"], g, u, self.kind)
        return dict(x=dx, Wg=dWgu[:len(p["Wg"])], Wu=dWgu[len(p["Wg"]):], Wd=dWd)[name]

    def more_directions(self, name):
        return ()

    def bound(self, name, v, gradient):
        s, p = self.step[name], self.p
        at = lambda t: {**p, name: p[name] + t * v}  # noqa: E731
        noise = (self.forward_noise(at(s)) + self.forward_noise(at(-s))) / (2 * s) ** 2 + self.gradient_noise(name, v, gradient)
        # fp32 sums of at most 2 H + d terms: a thousandth of the bf16 roundings at most, each of them
        return 1.01 * 8 * noise ** 0.5 + truncation(lambda t: self.f64(at(t)), s)


class Norm:
    """The norm on a residual stream in f32, f = sum(y dy) + sum(h dh): p = dict(x, r, w)."""

    def __init__(self, T, d, seed=0, eps=1e-6):
        rng = np.random.default_rng(seed + d)
        x = grid(rng, (T, d), 60, 2.0 ** -5)
        self.eps, self.d = eps, d
        self.p = dict(x=x, r=grid(rng, (T, d), 60, 2.0 ** -6), w=grid(rng, (d,), 60, 2.0 ** -5))
        # the norm's own term of the gradient is as large as the others where dy goes along with h
        self.dy, self.dh = grid(rng, (T, d), 60, 2.0 ** -5) + x, grid(rng, (T, d), 60, 2.0 ** -5)
        self.step = dict(x=2.0 ** -6, r=2.0 ** -6, w=2.0 ** -3)      # f is linear in w

    def f64(self, p):
        h = p["x"] + p["r"]
        return float((orc.rms_norm(h, p["w"], self.eps)[0] * self.dy).sum() + (h * self.dh).sum())

    def gradient(self, name):
        h = self.p["x"] + self.p["r"]
        dx, dw = orc.rms_norm_backward(self.dy, h, self.p["w"], orc.rms_norm(h, self.p["w"], self.eps)[1], self.dh)
        return dw if name == "w" else dx

    def more_directions(self, name):
        """The norm's own term of the gradient runs along h."""
        return () if name == "w" else (self.p["x"] + self.p["r"],)

    def bound(self, name, v, gradient):
        """In units of 2^-24 of the value: the sum of squares is off by 26 (16 terms of a thread, 10 halvings), rstd by half of that, mean, root and
        quotient: 16; y by two products more; h is exact here.  dx has rstd three times, another such sum and a few products: 100 of its
        terms' magnitudes; dw has u, 18, its product and a sum over the rows: 40 and one a row."""
        s, p = self.step[name], self.p
        h = p["x"] + p["r"]
        y, rstd = orc.rms_norm(h, p["w"], self.eps)
        u, g = h * rstd[:, None], self.dy * p["w"]
        size = 2.0 ** -24 * 20 * np.abs(y * self.dy).sum() * 1.1 / s
        if name == "w":
            size += 2.0 ** -24 * (40 + len(h)) * np.abs(self.dy * u).sum()
        else:
            size += 2.0 ** -24 * 100 * (np.abs(self.dh) + rstd[:, None] * (np.abs(g) + np.abs(u) * np.abs(g * u).mean(1, keepdims=True))).sum()
        return size + truncation(lambda t: self.f64({**p, name: p[name] + t * v}), s)


def check(case, name, forward, gradient):
    """forward(p) -> f; gradient: the passes' gradient of p[name].  -> [(difference, bound)] along every direction"""
    out, s, p = [], case.step[name], case.p
    for signs in (case.gradient(name), gradient, *case.more_directions(name)):
        v = np.sign(signs)
        num = (forward({**p, name: p[name] + s * v}) - forward({**p, name: p[name] - s * v})) / (2 * s)
        out.append((abs(num - float((gradient * v).sum())), float(case.bound(name, v, gradient))))
    return out


def passes(case, name, forward, gradient):
    return all(off <= bound for off, bound in check(case, name, forward, gradient))
