"""Calls of the dense branch's operators that are allowed and easily overlooked: scales whose unused bytes hold anything, a residual that is
the output itself, one tensor in several places, weights with a scale for every row.  Each is compared, bit for bit, with the plain call
that computes the same numbers.
"""
import numpy as np
import pytest
import torch

from oracle import branch_oracle as orc
from tests.gpu_util import bf16_to_f64 as f64

pytestmark = pytest.mark.gpu

U = 2.0 ** -23


def _bf(seed, *shape, std=1.0):
    return torch.from_numpy((np.random.default_rng(seed).normal(size=shape) * std).astype(np.float32)).to("cuda:0").bfloat16()


def _poisoned(q, byte):
    """q with every scale byte that belongs to no row or no block of the matrix set to `byte` (255 stands for NaN)."""
    from paper_2603_06626_b200 import binding as B
    rows, cols = q.shape
    a, b = q.scales.shape[:2]
    used = torch.zeros(128 * a, 4 * b, dtype=torch.bool, device=q.device)
    used[:rows, :(cols + 127) // 128] = True
    used = used.view(a, 4, 32, b, 4).permute(0, 3, 2, 1, 4)
    return B.Fp8Blocks(q.codes, torch.where(used, q.scales, torch.full_like(q.scales, byte)).contiguous(), cols)


@pytest.mark.parametrize("byte", [0, 255])
@pytest.mark.parametrize("T", [1, 20, 150, 700])
def test_unused_scale_bytes_hold_anything(T, byte):
    from paper_2603_06626_b200 import binding as B
    for d, H in ((72, 136), (520, 264), (1160, 72)):
        x, r = _bf(T, T, d), _bf(T + 1, T, d)
        Wg, Wu, Wd = (_bf(k, *s, std=s[1] ** -0.5) for k, s in ((1, (H, d)), (2, (H, d)), (3, (d, H))))
        q = [B.quantize_fp8(W, square=True)[0] for W in (Wg, Wu, Wd)]
        (x8, xt), Wt = B.quantize_fp8(x, transposed=True), B.quantize_fp8(Wg, square=True, transposed=True)[1]
        p = [_poisoned(v, byte) for v in q]
        p8, pt, pw = (_poisoned(v, byte) for v in (x8, xt, Wt))
        dy = _bf(T + 2, T, H)
        want = [B.linear_fp8(x8, q[0]), B.gated_ffn_fp8(x8, *q, residual=r), *B.linear_fp8_backward(dy, xt, Wt), B.dequantize_fp8(x8)]
        got = [B.linear_fp8(p8, p[0]), B.gated_ffn_fp8(p8, *p, residual=r), *B.linear_fp8_backward(dy, pt, pw), B.dequantize_fp8(p8)]
        for w, g in zip(want, got):
            assert w is None and g is None or torch.equal(w, g)
        assert torch.isfinite(want[1]).all()
    B.check_status()


@pytest.mark.parametrize("T", [1, 8, 40, 300, 2500])
def test_a_residual_that_is_the_output(T):
    from paper_2603_06626_b200 import binding as B
    lib, dev = B.load_library(), torch.device("cuda:0")
    d, H = 264, 392
    x, r, Wgu, Wd = _bf(T, T, d), _bf(T + 1, T, d), _bf(1, 2 * H, d, std=d ** -0.5), _bf(2, d, H, std=H ** -0.5)
    W8 = [B.quantize_fp8(W.contiguous(), square=True)[0] for W in (Wgu[:H], Wgu[H:], Wd)]
    x8 = B.quantize_fp8(_bf(3, T, H))[0]
    status, stream = torch.zeros(1, dtype=torch.int32, device=dev), torch.cuda.current_stream().cuda_stream
    ws = torch.empty(lib.grouter_gated_ffn_fp8_fwd_workspace_bytes(T, d, H), dtype=torch.uint8, device=dev)
    h = torch.empty(T, H, dtype=torch.bfloat16, device=dev)

    y = r.clone()
    assert lib.grouter_gated_ffn_fwd(x.data_ptr(), Wgu.data_ptr(), Wd.data_ptr(), y.data_ptr(), T, d, H, B.ACT_SILU, h.data_ptr(), y.data_ptr(), None,
                                     status.data_ptr(), stream) == 0
    assert torch.equal(y, B.gated_ffn(x, Wgu, Wd, residual=r)[0])

    y = r.clone()
    assert lib.grouter_linear_fp8_fwd(x8.codes.data_ptr(), x8.scales.data_ptr(), 0, W8[2].codes.data_ptr(), W8[2].scales.data_ptr(), None, y.data_ptr(),
                                      T, H, d, y.data_ptr(), None, status.data_ptr(), stream) == 0
    assert torch.equal(y, B.linear_fp8(x8, W8[2], residual=r))

    y = r.clone()
    parts = [p for q in W8 for p in (q.codes.data_ptr(), q.scales.data_ptr())]
    assert lib.grouter_gated_ffn_fp8_fwd(x.data_ptr(), None, d, *parts, y.data_ptr(), T, d, H, B.ACT_SILU, y.data_ptr(), ws.data_ptr(),
                                         status.data_ptr(), stream) == 0
    assert torch.equal(y, B.gated_ffn_fp8(x, *W8, residual=r))
    B.check_status(status=status)


@pytest.mark.parametrize("T", [4, 600])
def test_one_tensor_in_several_places(T):
    from paper_2603_06626_b200 import binding as B
    d = 136
    x, w = _bf(T, T, d), _bf(1, d)
    W = _bf(2, 2 * d, d, std=d ** -0.5)
    other = x.clone()
    for got, want in ((B.rms_norm(x, w, residual=x), B.rms_norm(x, w, residual=other)),
                      (B.gated_ffn(x, W, W[d:], residual=x, save_pre=True), B.gated_ffn(x, W, W[d:].clone(), residual=other, save_pre=True))):
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    pre = B.gated_ffn(x, W, W[d:], save_pre=True)[1]
    for a, b in zip(B.gated_ffn_backward(x, x, W, W[d:], pre), B.gated_ffn_backward(other, x, W, W[d:].clone(), pre)):
        assert torch.equal(a, b)
    _, h, rstd = B.rms_norm(x, w)
    for a, b in zip(B.rms_norm_backward(x, h, w, rstd, dh=x), B.rms_norm_backward(other, h, w, rstd, dh=x.clone())):
        assert torch.equal(a, b)
    q = B.quantize_fp8(W[:d], square=True)[0]
    for arg in (x, B.quantize_fp8(x)[0]):
        assert torch.equal(B.gated_ffn_fp8(arg, q, q, q, residual=x), B.gated_ffn_fp8(arg, q, B.quantize_fp8(W[:d], square=True)[0], q, residual=other))
    B.check_status()


@pytest.mark.parametrize("T,K,N", [(1, 640, 264), (33, 136, 392), (300, 1032, 520)])
def test_weights_with_a_scale_for_every_row(T, K, N):
    """A weight put into 8 bits without `square`: its scales differ from row to row.  The bound is that of the other products: (K/16 + 32) 2^-23
    of the sum of magnitudes, and 2^-8 of the value."""
    from paper_2603_06626_b200 import binding as B
    rng = np.random.default_rng(K)
    x = _bf(T, T, K)
    W = (_bf(1, N, K, std=K ** -0.5).float() * torch.from_numpy(2.0 ** rng.integers(-6, 7, (N, 1))).to("cuda:0")).bfloat16()
    W8, Wt = B.quantize_fp8(W, transposed=True)
    xr, Wr = orc.quantized(f64(x))[0], orc.quantized(f64(W))[0]
    want = xr @ Wr.T
    y = B.linear_fp8(x, W8)
    assert (np.abs(f64(y) - want) <= (K / 16 + 32) * U * (np.abs(xr) @ np.abs(Wr).T) + 2.0 ** -8 * np.abs(want)).all()
    dy = _bf(5, T, N)
    dx = B.linear_fp8_backward(dy, None, Wt, want_dW=False)[0]
    g, Wtr = orc.quantized(f64(dy))[0], orc.quantized(f64(W).T)[0]
    want = g @ Wtr.T
    assert (np.abs(f64(dx) - want) <= (N / 16 + 32) * U * (np.abs(g) @ np.abs(Wtr).T) + 2.0 ** -8 * np.abs(want)).all()
    B.check_status()


@pytest.mark.parametrize("T,K,N", [(700, 264, 2056), (1500, 1032, 4104), (9000, 1544, 2056), (40000, 72, 264), (6001, 2056, 24)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_both_gradients_in_one_launch(T, K, N, dtype):
    """Either product may be the one with the longer contraction, with fewer tiles than pairs of SMs or several rounds; dx does not depend on
    whether dW is wanted, and bounds as for each alone."""
    from paper_2603_06626_b200 import binding as B
    from tests.test_gpu_fp8 import _backward
    _backward(T, K, N, dtype=dtype, bias=False)
    dy, W = _bf(T, T, N), B.quantize_fp8(_bf(1, N, K, std=K ** -0.5), square=True, rows=False, transposed=True)[1]
    xt = B.quantize_fp8(_bf(2, T, K), rows=False, transposed=True)[1]
    assert torch.equal(B.linear_fp8_backward(dy, xt, W, dW_dtype=dtype)[0], B.linear_fp8_backward(dy, None, W, want_dW=False)[0])
