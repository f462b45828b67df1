"""The block around the expert layer: gradients of every tensor against the fp64 oracles, and training in both state widths.

Tolerance: every tensor passes through a few bf16 roundings (activations, gates, gradients), each at most 2^-9 relative; 2e-2 in
relative Frobenius norm covers eight of them in a row.
"""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from oracle import grouter_oracle as orc
from tests.gpu_util import bf16_to_f64 as f64

pytestmark = pytest.mark.gpu

T, D, F, E, K, H = 256, 128, 128, 8, 2, 192


def _block(bits=32, **kw):
    from paper_2603_06626_b200.block import RoutedBlock
    return RoutedBlock(T, D, F, E, K, H, state_bits=bits, **kw)


def test_gradients_of_every_tensor():
    blk = _block(balance_coef=0.5, z_coef=0.05)
    g = torch.Generator(device="cuda:0").manual_seed(3)
    x = torch.empty(T, D, device="cuda:0").normal_(generator=g).bfloat16()
    dout = torch.empty(T, D, device="cuda:0").normal_(generator=g).bfloat16()
    mask = torch.ones(T, dtype=torch.uint8, device="cuda:0")
    mask[::7] = 0
    out, losses = blk.forward(x, mask)
    dx = blk.backward(dout)
    blk.check_status()
    idx, gates = blk._saved[5].cpu().numpy(), f64(blk._saved[6])          # the kept experts are the kernels' own choice

    w = {n: f64(t) for n, t in blk.w.items()}
    xr, dy, m = f64(x), f64(dout), mask.cpu().numpy()
    h, mean, rstd = bo.layer_norm(xr, w["norm_w"], w["norm_b"], 1e-5)
    s = h @ w["W_s"].T
    q = bo.gates(np.take_along_axis(s, idx.astype(np.int64), 1), "softmax")
    assert np.abs(q - gates).max() < 2e-2
    counts, n = bo.expert_counts(idx, E, m)
    W = orc.Weights(w["W_gu"], w["W_d"])
    y = orc.moe_forward(h, idx, q, W, E)
    u, pre = bo.linear(h, w["W_1"], w["b_1"], None, "silu")
    dense, _ = bo.linear(u, w["W_2"], w["b_2"], None, "none")
    assert orc.rel_frobenius(f64(out), xr + y + dense) < 2e-2
    assert np.allclose(f64(losses), bo.balance_loss(s, counts, n, 0.5, 0.05, m), rtol=2e-2)
    dh, dg, dW = orc.moe_backward(dy, h, idx, q, W, E)
    du, dW2, db2, _ = bo.linear_backward(dy, u, w["W_2"], np.zeros_like(dy), "none")
    dh2, dW1, db1, _ = bo.linear_backward(du, h, w["W_1"], pre, "silu")
    ds = bo.balance_gradient(s, counts, n, 0.5, 0.05, m, idx, dg, "softmax")
    dh = dh + dh2 + ds @ w["W_s"]
    dxr, dnw, dnb = bo.layer_norm_backward(dh, xr, w["norm_w"], mean, rstd)
    want = {"norm_w": dnw, "norm_b": dnb, "W_s": ds.T @ h, "W_gu": np.stack([dW[e][0] for e in range(E)]),
            "W_d": np.stack([dW[e][1] for e in range(E)]), "W_1": dW1, "b_1": db1, "W_2": dW2, "b_2": db2}
    errs = {n: orc.rel_frobenius(f64(blk.grad[n]), want[n]) for n in want}
    errs["dx"] = orc.rel_frobenius(f64(dx), dy + dxr)
    assert max(errs.values()) < 2e-2, errs


@pytest.mark.parametrize("bits", [32, 8])
def test_it_learns(bits):
    blk = _block(bits, lr=3e-3)
    g = torch.Generator(device="cuda:0").manual_seed(1)
    x = torch.empty(T, D, device="cuda:0").normal_(generator=g).bfloat16()
    want = x.float() + torch.sin(x.float())
    errors = []
    for _ in range(30):
        out, losses = blk.forward(x)
        diff = out.float() - want
        errors.append(float(diff.square().mean()))
        blk.backward((diff * (2.0 / T)).bfloat16())
        blk.step()
    blk.check_status()
    assert errors[-1] < 0.2 * errors[0] and all(torch.isfinite(t.float()).all() for t in blk.w.values())


def test_only_the_router_moves_when_only_its_losses_count():
    """dout = 0: the experts' and the dense branch's gradients vanish, the balance loss goes down."""
    blk = _block(balance_coef=1.0, z_coef=0.0, lr=1e-2, weight_decay=0.0)
    g = torch.Generator(device="cuda:0").manual_seed(2)
    x = (torch.empty(T, D, device="cuda:0").normal_(generator=g) + 0.5).bfloat16()      # a shared direction: some experts are liked more
    zero = torch.zeros(T, D, device="cuda:0").bfloat16()
    seen = []
    for _ in range(25):
        _, losses = blk.forward(x)
        seen.append(float(losses[1]))
        blk.backward(zero)
        assert (blk.grad["W_gu"] == 0).all() and (blk.grad["W_1"] == 0).all() and (blk.grad["b_2"] == 0).all()
        blk.step()
    blk.check_status()
    assert seen[-1] < seen[0] and seen[-1] < 1.1
