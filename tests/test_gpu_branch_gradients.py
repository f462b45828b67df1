"""Gradients of the gated block and of the norm against differences of their forward passes, within bounds that a gradient without one of its terms
does not meet (tests/test_gradient_check.py plants such mistakes)."""
import numpy as np
import pytest
import torch

from tests.gradient_check import Gated, Norm, check

pytestmark = pytest.mark.gpu

NAMES = ["x", "Wg", "Wu", "Wd"]


def _bf(a):
    t = torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0").bfloat16()
    assert torch.equal(t.double().cpu(), torch.from_numpy(np.ascontiguousarray(a)))
    return t


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["none", "silu", "gelu"])
@pytest.mark.parametrize("T", [5, 64, 320, 700])          # the kernel for few tokens, with one tile of them and several, and that on tiles
def test_gated_block(T, kind, dtype):
    from paper_2603_06626_b200 import binding as B
    case, act = Gated(T, kind), dict(none=B.ACT_NONE, silu=B.ACT_SILU, gelu=B.ACT_GELU)[kind]
    dy = _bf(case.dy)

    def run(p, **kw):
        x, W, D = _bf(p["x"]), torch.cat([_bf(p["Wg"]), _bf(p["Wu"])]), _bf(p["Wd"])
        return x, W, D, *B.gated_ffn(x, W, D, act=act, **kw)

    x, W, D, _, pre = run(case.p, save_pre=True)
    dx, dW, dD = B.gated_ffn_backward(dy, x, W, D, pre, act=act, dW_dtype=dtype)
    B.check_status()
    H = D.shape[1]
    forward = lambda p: float((run(p)[3].double() * dy.double()).sum())  # noqa: E731
    for name, grad in zip(NAMES, (dx, dW[:H], dW[H:], dD)):
        for off, bound in check(case, name, forward, grad.double().cpu().numpy()):
            assert off <= bound, (name, off, bound)


@pytest.mark.parametrize("T,d", [(48, 96), (48, 640), (48, 1023), (300, 2048)])
def test_norm_on_a_residual_stream(T, d):
    from paper_2603_06626_b200 import binding as B
    case = Norm(T, d)
    f32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to("cuda:0")  # noqa: E731
    dy, dh = f32(case.dy), f32(case.dh)

    def run(p):
        return B.rms_norm(f32(p["x"]), f32(p["w"]), residual=f32(p["r"]), eps=case.eps)

    def forward(p):
        y, h, _ = run(p)
        return float((y.double() * dy.double()).sum() + (h.double() * dh.double()).sum())

    _, h, rstd = run(case.p)
    dx, dw = B.rms_norm_backward(dy, h, f32(case.p["w"]), rstd, dh=dh)
    for name, grad in (("x", dx), ("r", dx), ("w", dw)):
        for off, bound in check(case, name, forward, grad.double().cpu().numpy()):
            assert off <= bound, (name, off, bound)
