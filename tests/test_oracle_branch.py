"""Pins of the fp64 statements of the dense gated branch: the format against torch's e4m3, gradients against differences."""
import numpy as np
import pytest
import torch

from oracle import branch_oracle as orc


def test_e4m3_numbers_and_rounding_against_torch():
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(codes, orc.NUMBERS) and orc.NUMBERS[-1] == 448.0
    rng = np.random.default_rng(0)
    v = np.concatenate([rng.normal(size=5000) * 2.0 ** rng.integers(-12, 8, 5000), orc.NUMBERS, (orc.NUMBERS[1:] + orc.NUMBERS[:-1]) / 2])
    v = np.clip(np.concatenate([v, -v]), -448, 448).astype(np.float32)
    assert np.array_equal(orc.e4m3(v.astype(np.float64)), torch.from_numpy(v).to(torch.float8_e4m3fn).double().numpy())
    assert np.isnan(orc.e4m3(np.array([np.inf, -np.inf, np.nan]))).all()


def test_the_exponent_is_the_smallest_that_holds_the_largest():
    top = np.array([0.0, 1e-45, 448.0, 448.0001, 447.9, 3.4e38, 1.0, 0.875, 0.8751, 2.0 ** -140])
    e = orc.exponent(top)
    assert (top <= 448.0 * 2.0 ** e).all() and ((e == -126) | (top > 448.0 * 2.0 ** (e - 1))).all()
    assert list(e[[2, 3, 4]]) == [0, 1, 0] and e[0] == -126


def test_a_square_shares_one_scale():
    x = np.random.default_rng(1).normal(size=(200, 300))
    e = orc.exponents(x, square=True)
    assert (e[:128] == e[0]).all() and (e[128:] == e[128]).all() and e.shape == (200, 3)
    et = orc.exponents(x.T, square=True)
    assert np.array_equal(et[::128], e[::128].T)


@pytest.mark.parametrize("kind", ["none", "silu", "gelu"])
def test_gradients_against_differences(kind):
    rng = np.random.default_rng(2)
    T, d, H = 5, 7, 6
    x, dy = rng.normal(size=(T, d)), rng.normal(size=(T, d))
    Wg, Wu, Wd = rng.normal(size=(H, d)), rng.normal(size=(H, d)), rng.normal(size=(d, H))
    h, g, u = orc.gated(x, Wg, Wu, kind)
    dx, dWgu, dWd, _, _, _ = orc.gated_backward(dy, x, Wg, Wu, Wd, g, u, kind)
    f = lambda x, Wg, Wu, Wd: ((orc.gated(x, Wg, Wu, kind)[0] @ Wd.T) * dy).sum()  # noqa: E731
    s = 1e-5
    for i, grad in enumerate([dx, dWgu[:H], dWgu[H:], dWd]):
        args = [x, Wg, Wu, Wd]
        step = rng.normal(size=args[i].shape)
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + s * step, args[i] - s * step
        num = (f(*up) - f(*down)) / (2 * s)
        assert abs(num - (grad * step).sum()) <= 1e-7 * (1 + np.abs(grad * step).sum())


def test_norm_gradient_against_differences():
    rng = np.random.default_rng(3)
    h, dy, dh, w = rng.normal(size=(4, 9)), rng.normal(size=(4, 9)), rng.normal(size=(4, 9)), rng.normal(size=9)
    _, rstd = orc.rms_norm(h, w, 1e-6)
    dx, dw = orc.rms_norm_backward(dy, h, w, rstd, dh)
    f = lambda h, w: (orc.rms_norm(h, w, 1e-6)[0] * dy).sum() + (h * dh).sum()  # noqa: E731
    s, v, vw = 1e-5, rng.normal(size=h.shape), rng.normal(size=9)
    assert abs((f(h + s * v, w) - f(h - s * v, w)) / (2 * s) - (dx * v).sum()) <= 1e-7 * np.abs(dx * v).sum()
    assert abs((f(h, w + s * vw) - f(h, w - s * vw)) / (2 * s) - (dw * vw).sum()) <= 1e-7 * np.abs(dw * vw).sum()
