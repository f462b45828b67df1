"""The gated feed-forward block, in bf16 and in 8 bits, against the fp64 oracle: one token to several tiles, ragged in every dimension.

Bounds, per element, as for the linear layer: a product of K terms is off by (K/16 + 32) 2^-23 of the sum of magnitudes; no activation
stretches an error by more than 1.2, its own evaluation is within 2^-18 of |z|, and so are the few operations that form h, dg and du.
Rounding to bf16 adds 2^-8 of the value (twice the half ulp); h, dg and du are rounded so on their way into the next product.
8 bits: h is rounded to codes from a value within those bounds, so it may stand for anything between what the value less and the value
plus its bound are rounded to (the scales' borders are not near: that is checked).
"""
import numpy as np
import pytest
import torch

from oracle import branch_oracle as orc
from oracle.block_oracle import act, act_slope
from oracle.grouter_oracle import rel_frobenius
from tests.gpu_util import bf16_to_f64 as f64

pytestmark = pytest.mark.gpu

U = 2.0 ** -23
KINDS = ["none", "relu", "silu", "gelu"]


def _bf(rng, *shape, std=1.0):
    return torch.from_numpy((rng.normal(size=shape) * std).astype(np.float32)).to("cuda:0").bfloat16()


def _act(kind):
    from paper_2603_06626_b200 import binding as B
    return dict(none=B.ACT_NONE, relu=B.ACT_RELU, silu=B.ACT_SILU, gelu=B.ACT_GELU)[kind]


def _off(a, b):
    return (a.shape[1] / 16 + 32) * U * (np.abs(a) @ np.abs(b).T)


def _weights(rng, d, H):
    return _bf(rng, 2 * H, d, std=d ** -0.5), _bf(rng, d, H, std=H ** -0.5)


def _forward(T, d, H, kind="silu", residual=False, pre=False):
    from paper_2603_06626_b200 import binding as B
    rng = np.random.default_rng(T + d + H)
    x, (Wgu, Wd) = _bf(rng, T, d), _weights(rng, d, H)
    r = _bf(rng, T, d) if residual else None
    y, p = B.gated_ffn(x, Wgu, Wd, act=_act(kind), residual=r, save_pre=pre)
    again = B.gated_ffn(x, Wgu, Wd, act=_act(kind), residual=r, save_pre=not pre)
    B.check_status()
    assert torch.equal(y, again[0])
    xr, Wg, Wu, Wdr = f64(x), f64(Wgu[:H]), f64(Wgu[H:]), f64(Wd)
    h, g, u = orc.gated(xr, Wg, Wu, kind)
    og, ou = _off(xr, Wg), _off(xr, Wu)
    oh = 1.2 * og * (np.abs(u) + ou) + np.abs(act(g, kind)) * ou + 2.0 ** -18 * np.abs(g * u) + 2.0 ** -8 * np.abs(h)
    want = h @ Wdr.T + (0 if r is None else f64(r))
    size = _off(h, Wdr) + oh @ np.abs(Wdr).T + (0 if r is None else 4 * U * np.abs(f64(r)))
    assert (np.abs(f64(y) - want) <= 1.01 * size + 2.0 ** -8 * np.abs(want)).all()
    assert rel_frobenius(f64(y), want) <= 5e-3
    if pre:
        assert (np.abs(f64(p[:, :H]) - g) <= og + 2.0 ** -8 * np.abs(g)).all() and (np.abs(f64(p[:, H:]) - u) <= ou + 2.0 ** -8 * np.abs(u)).all()
    else:
        assert p is None


SIZES = [(1, 8, 8), (1, 128, 64), (2, 72, 24), (5, 520, 136), (16, 256, 128), (17, 1024, 264), (33, 264, 520), (64, 512, 384), (65, 640, 72),
         (130, 136, 1000), (256, 256, 256), (300, 392, 904), (1, 4096, 1536), (515, 1032, 200)]


@pytest.mark.parametrize("T,d,H", SIZES)
def test_forward(T, d, H):
    _forward(T, d, H, pre=True)
    _forward(T, d, H, residual=True)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T", [3, 200])
def test_activations(kind, T):
    _forward(T, 264, 328, kind, residual=True, pre=True)


def test_more_tiles_than_pairs():
    _forward(5000, 72, 1000, "gelu", pre=True)
    _forward(2600, 200, 1032, residual=True)


def _backward(T, d, H, kind="silu", dtype=torch.bfloat16):
    from paper_2603_06626_b200 import binding as B
    rng = np.random.default_rng(T + d + H)
    x, dy, (Wgu, Wd), p = _bf(rng, T, d), _bf(rng, T, d), _weights(rng, d, H), _bf(rng, T, 2 * H, std=1.5)
    got = B.gated_ffn_backward(dy, x, Wgu, Wd, p, act=_act(kind), dW_dtype=dtype)
    again = B.gated_ffn_backward(dy, x, Wgu, Wd, p, act=_act(kind), dW_dtype=dtype)
    B.check_status()
    assert all(torch.equal(a, b) for a, b in zip(got, again)) and got[1].dtype == got[2].dtype == dtype
    xr, g0, Wg, Wu, Wdr, g, u = f64(x), f64(dy), f64(Wgu[:H]), f64(Wgu[H:]), f64(Wd), f64(p[:, :H]), f64(p[:, H:])
    dx, dWgu, dWd, dg, du, h = orc.gated_backward(g0, xr, Wg, Wu, Wdr, g, u, kind)
    oh = _off(g0, Wdr.T)                                       # of dh
    a, s = act(g, kind), act_slope(g, kind)
    dh = np.abs(g0 @ Wdr)
    r = 2.0 ** -8
    odg = oh * np.abs(u * s) + 2.0 ** -17 * dh * np.abs(u) * (1 + np.abs(g)) + r * np.abs(dg)
    odu = oh * np.abs(a) + 2.0 ** -17 * dh * np.abs(g) + r * np.abs(du)
    ohh = 2.0 ** -17 * np.abs(g * u) + r * np.abs(h)
    odp, dp, Wall = np.concatenate([odg, odu], 1), np.concatenate([dg, du], 1), np.concatenate([Wg, Wu])
    bounds = (odp @ np.abs(Wall) + _off(dp, Wall.T), odp.T @ np.abs(xr) + _off(dp.T, xr.T), np.abs(g0).T @ ohh + _off(g0.T, h.T))
    for out, want, off, kind_of in zip(got, (dx, dWgu, dWd), bounds, (torch.bfloat16, dtype, dtype)):
        assert (np.abs(f64(out) - want) <= 1.01 * off + (r if kind_of == torch.bfloat16 else 0.0) * np.abs(want) + 1e-30).all()
        assert rel_frobenius(f64(out), want) <= 5e-3


@pytest.mark.parametrize("T,d,H", [(1, 8, 8), (2, 128, 72), (17, 264, 136), (64, 512, 256), (100, 136, 520), (257, 392, 264), (1030, 256, 1000)])
def test_backward(T, d, H):
    _backward(T, d, H)
    _backward(T, d, H, "gelu", torch.float32)


@pytest.mark.parametrize("kind", KINDS)
def test_backward_of_activations(kind):
    _backward(300, 200, 328, kind)
    _backward(9, 72, 264, kind)


def test_backward_of_more_tiles_than_pairs():
    _backward(4700, 136, 1032)


def test_gradients_one_by_one_and_into_given_tensors():
    from paper_2603_06626_b200 import binding as B
    rng = np.random.default_rng(3)
    T, d, H = 150, 136, 200
    x, dy, (Wgu, Wd), p = _bf(rng, T, d), _bf(rng, T, d), _weights(rng, d, H), _bf(rng, T, 2 * H)
    dx, dWgu, dWd = B.gated_ffn_backward(dy, x, Wgu, Wd, p)
    only = B.gated_ffn_backward(dy, x, Wgu, Wd, p, want_dW=False)
    assert torch.equal(only[0], dx) and only[1] is None and only[2] is None
    into = torch.full((2 * H, d), 7.0, device="cuda:0")
    only = B.gated_ffn_backward(dy, x, Wgu, Wd, p, want_dx=False, want_dW=False, dW_gu=into)
    assert only[0] is None and only[1] is into and only[2] is None and torch.equal(into.bfloat16(), dWgu)
    gu, down = torch.empty_like(Wgu), torch.empty_like(Wd)
    B.gated_ffn_backward(dy, x, Wgu, Wd, p, dW_gu=gu, dW_d=down)
    assert torch.equal(gu, dWgu) and torch.equal(down, dWd)


def test_rows_that_are_not_finite_stay_alone():
    from paper_2603_06626_b200 import binding as B
    rng = np.random.default_rng(5)
    Wgu, Wd = _weights(rng, 264, 200)
    W8 = [B.quantize_fp8(W.contiguous(), square=True)[0] for W in (Wgu[:200], Wgu[200:], Wd)]
    for T in (6, 300):
        x = _bf(rng, T, 264)
        clean = B.gated_ffn(x, Wgu, Wd)[0], B.gated_ffn_fp8(x, *W8)
        x[2, 5] = float("nan")
        keep = torch.arange(T, device="cuda:0") != 2
        for y, c in zip((B.gated_ffn(x, Wgu, Wd)[0], B.gated_ffn_fp8(x, *W8)), clean):
            assert torch.isnan(y[2]).all() and torch.equal(y[keep], c[keep])


def test_no_tokens():
    from paper_2603_06626_b200 import binding as B
    rng = np.random.default_rng(6)
    Wgu, Wd = _weights(rng, 128, 72)
    x, p = torch.empty(0, 128, dtype=torch.bfloat16, device="cuda:0"), torch.empty(0, 144, dtype=torch.bfloat16, device="cuda:0")
    y, pre = B.gated_ffn(x, Wgu, Wd, save_pre=True)
    assert y.shape == (0, 128) and pre.shape == (0, 144)
    dx, dWgu, dWd = B.gated_ffn_backward(x, x, Wgu, Wd, p)
    assert dx.shape == (0, 128) and (dWgu == 0).all() and (dWd == 0).all()
    W8 = [B.quantize_fp8(W.contiguous(), square=True)[0] for W in (Wgu[:72], Wgu[72:], Wd)]
    assert B.gated_ffn_fp8(x, *W8).shape == (0, 128)


def _eight(T, d, H, kind="silu", residual=False, codes=False):
    from paper_2603_06626_b200 import binding as B
    rng = np.random.default_rng(T + d + H)
    x, (Wgu, Wd) = _bf(rng, T, d), _weights(rng, d, H)
    r = _bf(rng, T, d) if residual else None
    W8 = [B.quantize_fp8(W.contiguous(), square=True)[0] for W in (Wgu[:H], Wgu[H:], Wd)]
    arg = B.quantize_fp8(x)[0] if codes else x
    y = B.gated_ffn_fp8(arg, *W8, act=_act(kind), residual=r)
    assert torch.equal(y, B.gated_ffn_fp8(arg, *W8, act=_act(kind), residual=r))
    B.check_status()
    xr = orc.quantized(f64(x))[0]
    Wg, Wu, Wdr = (orc.quantized(f64(W), square=True)[0] for W in (Wgu[:H], Wgu[H:], Wd))
    h, g, u = orc.gated(xr, Wg, Wu, kind)
    og, ou = _off(xr, Wg), _off(xr, Wu)
    oh = 1.2 * og * (np.abs(u) + ou) + np.abs(act(g, kind)) * ou + 2.0 ** -18 * np.abs(g * u)
    e = orc.exponents(h)
    near = (orc.exponents(np.maximum(np.abs(h) - oh, 0)) != e) | (orc.exponents(np.abs(h) + oh) != e)
    top = 448.0 * 2.0 ** np.repeat(e, 128, 1)[:, :H]
    q = orc.quantized(h, exps=e)[0]
    lo, hi = (orc.quantized(np.clip(h + s * oh, -top, top), exps=e)[0] for s in (-1, 1))
    off = np.maximum(hi - q, q - lo)
    off = np.where(np.repeat(near, 128, 1)[:, :H], off + 2.0 ** -3 * np.abs(q) + top * 2.0 ** -17, off)      # half a step of the coarser scale on top
    want = q @ Wdr.T + (0 if r is None else f64(r))
    bound = off @ np.abs(Wdr).T + 1.2 * _off(q, Wdr) + (0 if r is None else 4 * U * np.abs(f64(r))) + 2.0 ** -8 * np.abs(want)
    assert (np.abs(f64(y) - want) <= bound).all()
    assert rel_frobenius(f64(y), want) <= 5e-3


@pytest.mark.parametrize("T,d,H", SIZES)
def test_eight_bits(T, d, H):
    _eight(T, d, H)
    _eight(T, d, H, residual=True, codes=True)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T", [3, 300])
def test_eight_bits_of_activations(kind, T):
    _eight(T, 264, 328, kind)


def test_eight_bits_of_more_tiles_than_pairs():
    _eight(5000, 72, 1000, "gelu")
    _eight(2600, 520, 1032, residual=True)


@pytest.mark.parametrize("T", [1, 7, 16, 17, 300])
def test_eight_bits_of_tokens_and_of_codes_are_the_same(T):
    from paper_2603_06626_b200 import binding as B
    rng = np.random.default_rng(T)
    d, H = 1032, 264
    x, (Wgu, Wd) = _bf(rng, T, d + 8)[:, :d], _weights(rng, d, H)
    W8 = [B.quantize_fp8(W.contiguous(), square=True)[0] for W in (Wgu[:H], Wgu[H:], Wd)]
    y = B.gated_ffn_fp8(x, *W8, act=B.ACT_GELU)
    assert torch.equal(y, B.gated_ffn_fp8(B.quantize_fp8(x)[0], *W8, act=B.ACT_GELU))


@pytest.mark.parametrize("T", [4, 300])
def test_a_hidden_state_beyond_the_largest_number(T):
    """g u overflows in one row: an infinity there has the code of NaN, the row's output is NaN and no other row's changes."""
    from paper_2603_06626_b200 import binding as B
    rng = np.random.default_rng(9)
    Wgu, Wd = _weights(rng, 264, 200)
    W8 = [B.quantize_fp8(W.contiguous(), square=True)[0] for W in (Wgu[:200], Wgu[200:], Wd)]
    x = _bf(rng, T, 264)
    clean = B.gated_ffn_fp8(x, *W8)
    x[1] *= 2.0 ** 90
    y = B.gated_ffn_fp8(x, *W8)
    keep = torch.arange(T, device="cuda:0") != 1
    assert torch.isnan(y[1]).all() and torch.equal(y[keep], clean[keep])


def test_streams_and_graphs():
    from paper_2603_06626_b200 import binding as B
    rng = np.random.default_rng(7)
    T, d, H = 200, 256, 384
    x, dy, (Wgu, Wd) = _bf(rng, T, d), _bf(rng, T, d), _weights(rng, d, H)
    W8 = [B.quantize_fp8(W.contiguous(), square=True)[0] for W in (Wgu[:H], Wgu[H:], Wd)]

    def step():
        y, p = B.gated_ffn(x, Wgu, Wd, residual=x, save_pre=True)
        return (y, p, *B.gated_ffn_backward(dy, x, Wgu, Wd, p), B.gated_ffn_fp8(x, *W8, residual=x))

    want = step()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = step()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    graphs, held = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for g in graphs:
        with torch.cuda.graph(g):
            held.append(step())
    for g in graphs + graphs:
        g.replay()
    torch.cuda.synchronize()
    B.check_status()
    for h in held:
        assert all(torch.equal(p, q) for p, q in zip(want, h))


def test_gradient_against_differences_of_the_kernel():
    """Directional derivative of sum(y * dy), by central differences of the forward pass with bf16 inputs: the steps x + s u and x - s u are
    bf16 numbers (x and u are small integers times powers of two), so the only errors are the outputs' roundings (2^-9 of y, T d of
    them, independent) over the step, the roundings on the way of the gradient (2^-8 of its terms) and the third-order term s^2."""
    from paper_2603_06626_b200 import binding as B
    rng = np.random.default_rng(12)
    T, d, H = 64, 128, 128
    x = torch.from_numpy(rng.integers(-8, 9, (T, d)).astype(np.float32) / 8).to("cuda:0").bfloat16()
    u = torch.from_numpy(rng.integers(-1, 2, (T, d)).astype(np.float32)).to("cuda:0")
    s = 2.0 ** -4
    Wgu, Wd = _weights(rng, d, H)
    dy = _bf(rng, T, d)
    f = lambda v: (B.gated_ffn(v.bfloat16(), Wgu, Wd)[0].double() * dy.double()).sum().item()  # noqa: E731
    y, p = B.gated_ffn(x, Wgu, Wd, save_pre=True)
    dx, _, _ = B.gated_ffn_backward(dy, x, Wgu, Wd, p)
    num, ana = (f(x.float() + s * u) - f(x.float() - s * u)) / (2 * s), (dx.double() * u.double()).sum().item()
    # 8 standard deviations of the sum of roundings (uniform within 2^-9 of |y dy|, on both sides, two roundings deep)
    noise = 8 * 2 * 2.0 ** -9 * float((y.double() * dy.double()).square().sum().sqrt()) / (2 * s) * 2 ** 0.5
    scale = float((dx.double() * u.double()).square().sum().sqrt())
    assert abs(num - ana) <= noise + 8 * 2.0 ** -8 * scale + 4 * s * s * float((dx.double() * u.double()).abs().sum())
