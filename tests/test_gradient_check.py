"""The checks of gradients against differences, on plain statements of what the kernels round: the right gradient passes them, one with a
term left out, a wrong slope or a wrong factor does not."""
import numpy as np
import pytest
import torch

from oracle import branch_oracle as orc
from oracle.block_oracle import act, act_slope
from tests.gradient_check import Gated, Norm, check, passes

NAMES = ["x", "Wg", "Wu", "Wd"]


def bf(a):
    return torch.from_numpy(np.ascontiguousarray(a)).bfloat16().double().numpy()


def forward(case):
    def f(p):
        assert all(np.array_equal(bf(v), v) for v in p.values())          # the points are numbers of the type
        h = bf(orc.gated(p["x"], p["Wg"], p["Wu"], case.kind)[0])
        return float((bf(h @ p["Wd"].T) * case.dy).sum())
    return f


def gradients(case, mistake=None):
    p, kind = case.p, case.kind
    _, g, u = orc.gated(p["x"], p["Wg"], p["Wu"], kind)
    g, u = bf(g), bf(u)
    a, s, dh = act(g, kind), act_slope(g, kind), case.dy @ p["Wd"]
    if mistake == "sigmoid for the slope":
        s = 1 / (1 + np.exp(-g))
    if mistake == "slope at u":
        s = act_slope(u, kind)
    dg, du, h = bf(dh * u * s), bf(dh * a), bf(a * u)
    if mistake == "du of the gate":
        du = bf(dh * g)
    if mistake == "h without the activation":
        h = bf(g * u)
    if mistake == "a row left out":
        dg[7], du[7], h[7] = 0.0, 0.0, 0.0
    dx = dg @ p["Wg"] * (mistake != "no gate term") + du @ p["Wu"] * (mistake != "no up term")
    if mistake == "halves exchanged":
        dg, du = du, dg
    return dict(zip(NAMES, (bf(v) for v in (dx, dg.T @ p["x"], du.T @ p["x"], case.dy.T @ h))))


def wrong(case, name, f, grad):
    """Outside the bound by a factor of two along one of the directions."""
    return any(off > 2 * bound for off, bound in check(case, name, f, grad))


@pytest.mark.parametrize("T", [64, 320])
@pytest.mark.parametrize("kind", ["none", "silu", "gelu"])
def test_the_right_gradient_passes(T, kind):
    case = Gated(T, kind)
    for name, grad in gradients(case).items():
        for off, bound in check(case, name, forward(case), grad):
            assert off <= bound <= 0.02 * np.abs(grad).sum(), (name, off, bound, np.abs(grad).sum())


@pytest.mark.parametrize("T", [64, 320])
@pytest.mark.parametrize("mistake,seen_in", [("no gate term", ["x"]), ("no up term", ["x"]), ("sigmoid for the slope", ["x", "Wg"]),
                                             ("slope at u", ["x", "Wg"]), ("du of the gate", ["x", "Wu"]), ("h without the activation", ["Wd"]),
                                             ("halves exchanged", ["Wg", "Wu"])])
def test_a_wrong_gradient_does_not(T, mistake, seen_in):
    case = Gated(T, "silu")
    grads = gradients(case, mistake)
    for name in seen_in:
        assert wrong(case, name, forward(case), grads[name]), (mistake, name, check(case, name, forward(case), grads[name]))


def test_a_token_that_is_left_out_of_the_weights_gradients_is_seen():
    case = Gated(64, "silu")
    grads = gradients(case, "a row left out")
    for name in ("Wu", "Wd"):
        assert not passes(case, name, forward(case), grads[name]), (name, check(case, name, forward(case), grads[name]))


def norm_gradients(case, mistake=None):
    p, h = case.p, case.p["x"] + case.p["r"]
    _, rstd = orc.rms_norm(h, p["w"], case.eps)
    r, u, g = rstd[:, None], h * rstd[:, None], case.dy * p["w"]
    own = u * (g * u).mean(1, keepdims=True)
    dx = case.dh * (mistake != "no stream") + r * (g - own * (mistake != "no term of the norm"))
    dw = (case.dy * (h if mistake == "dw of h" else u)).sum(0)
    return dict(x=dx, r=dx, w=dw)


@pytest.mark.parametrize("d", [96, 640, 1023])
def test_the_norm(d):
    case = Norm(48, d)

    def f(p):
        assert all(np.array_equal(v.astype(np.float32), v) for v in p.values())
        h = (p["x"] + p["r"]).astype(np.float32)
        assert np.array_equal(h, p["x"] + p["r"])
        y = orc.rms_norm(h.astype(np.float64), p["w"], case.eps)[0].astype(np.float32)
        return float((y.astype(np.float64) * case.dy).sum() + (h.astype(np.float64) * case.dh).sum())

    for name, grad in norm_gradients(case).items():
        for off, bound in check(case, name, f, grad.astype(np.float32).astype(np.float64)):
            assert off <= bound <= 2e-3 * np.abs(grad).sum(), (name, off, bound, np.abs(grad).sum())
    for mistake, name in (("no term of the norm", "x"), ("no stream", "x"), ("dw of h", "w")):
        assert wrong(case, name, f, norm_gradients(case, mistake)[name]), (mistake, check(case, name, f, norm_gradients(case, mistake)[name]))
