"""The dense block, its form in 8 bits and the projection trained in 8 bits: the operators of the dense gated branch in a row, against the
fp64 oracles.

Tolerance: every tensor passes through a few bf16 roundings (activations, gradients), each at most 2^-9 relative; 2e-2 in relative
Frobenius norm covers eight of them in a row.  What is put into 8 bits is put there by the oracle too, from values that differ by those
roundings: a code then differs by a step, 2^-3 of it, wherever such a difference crosses a border between codes, which is at most one value
in 2^-8 / 2^-4 = 16 for each rounding before; the root mean square of that, 2^-3 / 4, is 3e-2 of the values it touches in an independent
direction, and it passes through the projections once before the output and twice before a weight's gradient: 6e-2.
"""
import numpy as np
import pytest
import torch

from oracle import branch_oracle as orc
from oracle.grouter_oracle import rel_frobenius
from tests.gpu_util import bf16_to_f64 as f64

pytestmark = pytest.mark.gpu

T, D, H, N = 300, 256, 400, 144


def _data(seed=3):
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    return [torch.empty(T, n, device="cuda:0").normal_(generator=g).bfloat16() for n in (D, D, D)]


def _forward(block, xr):
    w = {n: f64(t) for n, t in block.w.items()}
    y, rstd = orc.rms_norm(xr, w["norm_w"], block.eps)
    h, g, u = orc.gated(y, w["W_gu"][:H], w["W_gu"][H:], "silu")
    return w, y, rstd, g, u, h @ w["W_d"].T


def test_gradients_of_every_tensor():
    from paper_2603_06626_b200.dense import DenseBlock
    x, r, dout = _data()
    block = DenseBlock(D, H)
    block.w["norm_w"].copy_(torch.linspace(0.5, 1.5, D))
    out = block.forward(x, r)
    dx = block.backward(dout)
    block.check_status()
    hr = f64(x) + f64(r)
    w, y, rstd, g, u, f = _forward(block, hr)
    assert rel_frobenius(f64(out), hr + f) < 2e-2
    d = f64(dout)
    dy, dWgu, dWd, _, _, _ = orc.gated_backward(d, y, w["W_gu"][:H], w["W_gu"][H:], w["W_d"], g, u, "silu")
    dxr, dw = orc.rms_norm_backward(dy, hr, w["norm_w"], rstd, d)
    errs = {"dx": rel_frobenius(f64(dx), dxr)}
    for name, want in (("norm_w", dw), ("W_gu", dWgu), ("W_d", dWd)):
        errs[name] = rel_frobenius(f64(block.grad[name]), want)
    assert max(errs.values()) < 2e-2, errs


def test_served_in_8_bits():
    from paper_2603_06626_b200.dense import DenseBlock
    x, r, _ = _data(4)
    block = DenseBlock(D, H)
    served = block.served()
    out = served.forward(x, r)
    one = served.forward(x[5:6], r[5:6])
    served.check_status()
    hr = f64(x) + f64(r)
    w = {n: f64(t) for n, t in block.w.items()}
    y = orc.quantized(orc.rms_norm(hr, w["norm_w"], block.eps)[0])[0]
    Wg, Wu, Wd = (orc.quantized(W, square=True)[0] for W in (w["W_gu"][:H], w["W_gu"][H:], w["W_d"]))
    f = orc.quantized(orc.gated(y, Wg, Wu, "silu")[0])[0] @ Wd.T
    assert rel_frobenius(f64(out) - hr, f) < 6e-2
    assert rel_frobenius(f64(one) - hr[5:6], f[5:6]) < 6e-2
    block.w["W_d"].zero_()                                        # what is served is what was there when it was made
    assert torch.equal(served.forward(x, r), out)


def test_projection_in_8_bits():
    from paper_2603_06626_b200.dense import Projection8
    x, _, _ = _data(5)
    dz = torch.randn(T, N, device="cuda:0").bfloat16()
    p = Projection8(D, N)
    z = p.forward(x)
    dx = p.backward(dz)
    p.check_status()
    Wr = f64(p.W)
    assert rel_frobenius(f64(z), orc.quantized(f64(x))[0] @ orc.quantized(Wr, square=True)[0].T) < 1e-2
    assert rel_frobenius(f64(dx), orc.quantized(f64(dz))[0] @ orc.quantized(Wr.T, square=True)[0].T) < 1e-2
    assert rel_frobenius(f64(p.grad), orc.quantized(f64(dz).T)[0] @ orc.quantized(f64(x).T)[0].T) < 1e-2


@pytest.mark.parametrize("bits", [32, 8])
def test_a_training_step_of_all_of_them(bits):
    """Block and projection in a row: gradients against the oracle's, then a few steps that change every weight."""
    from paper_2603_06626_b200.dense import DenseBlock, Projection8
    x, r, _ = _data(6)
    block, head = DenseBlock(D, H, state_bits=bits), Projection8(D, N, state_bits=bits)
    dz = (torch.randn(T, N, device="cuda:0") / T).bfloat16()
    head.forward(block.forward(x, r))
    block.backward(head.backward(dz))
    hr = f64(x) + f64(r)
    w, y, rstd, g, u, f = _forward(block, hr)
    dout = orc.quantized(f64(dz))[0] @ orc.quantized(f64(head.W).T, square=True)[0].T
    _, dWgu, dWd, _, _, _ = orc.gated_backward(dout, y, w["W_gu"][:H], w["W_gu"][H:], w["W_d"], g, u, "silu")
    dW = orc.quantized(f64(dz).T)[0] @ orc.quantized((hr + f).T)[0].T
    errs = [rel_frobenius(f64(a), b) for a, b in ((block.grad["W_gu"], dWgu), (block.grad["W_d"], dWd), (head.grad, dW))]
    assert max(errs[:2]) < 2e-2 and errs[2] < 6e-2, errs
    before = {n: t.clone() for n, t in block.w.items()} | {"W": head.W.clone()}
    for _ in range(3):
        diff = head.forward(block.forward(x, r))
        block.backward(head.backward((diff.float() * (2.0 / T)).bfloat16()))
        block.step()
        head.step()
    block.check_status()
    head.check_status()
    after = block.w | {"W": head.W}
    assert all(torch.isfinite(after[n].float()).all() and not torch.equal(after[n], before[n]) for n in after)


def test_a_captured_step():
    """Forward and backward of the block in a graph, replayed on new inputs."""
    from paper_2603_06626_b200.dense import DenseBlock
    x, r, dout = _data(7)
    block = DenseBlock(D, H)
    block.backward(dout if block.forward(x, r) is not None else None)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block.forward(x, r)
        dx = block.backward(dout)
    x2, r2, dout2 = _data(8)
    for to, new in ((x, x2), (r, r2), (dout, dout2)):
        to.copy_(new)
    graph.replay()
    held = out.clone(), dx.clone(), block.grad["W_gu"].clone()
    again = block.forward(x2, r2), block.backward(dout2), block.grad["W_gu"]
    block.check_status()
    assert all(torch.equal(a, b) for a, b in zip(held, again))


def test_the_command_runs(capsys, monkeypatch):
    import sys

    from paper_2603_06626_b200 import dense
    monkeypatch.setattr(sys, "argv", ["dense", "--steps", "2", "--state-bits", "8"])
    dense.main()
    assert "served in 8 bits" in capsys.readouterr().out
