"""Weight gradients that are contracted over matrices of more than 2^31 elements, and the backward pass in 8 bits on them: every row counts in
the sums, so a row offset that wraps, a piece that starts at another token or rows past the border left out would all show.

Tolerances as in the tests of the single operators: a sum of n terms is within (n/16 + 32) 2^-23 of the sum of magnitudes, bf16 outputs within
2^-8 of the value on top; the gated block, whose dp is rounded to bf16 on the way, within 5e-3 in relative Frobenius norm, for the whole
gradient and for the part that each stretch of tokens has in it."""
import pytest
import torch

from tests.test_gpu_branch_large import U, _rand, _slices

pytestmark = pytest.mark.gpu


def test_gated_block_weights():
    from paper_2603_06626_b200 import binding as B
    T, d, H = 140000, 16, 8192
    x, dy, Wgu, Wd, p = _rand(T, d, 1), _rand(T, d, 2), _rand(2 * H, d, 3, d ** -0.5), _rand(d, H, 4, H ** -0.5), _rand(T, 2 * H, 5)
    assert T * 2 * H > 2 ** 31
    # tokens of a stretch around the place where 32-bit offsets of dp end, and the last ones, weigh a hundred times as much as the others:
    # what they add is most of the gradient, so that their absence or a wrong place is far outside the bound
    middle = 2 ** 31 // (2 * H)
    heavy = torch.zeros(T, dtype=torch.bool, device="cuda:0")
    heavy[middle - 300:middle + 300] = True
    heavy[-200:] = True
    dy[heavy] *= 100
    dx, dWgu, dWd = B.gated_ffn_backward(dy, x, Wgu, Wd, p, dW_dtype=torch.float32)
    B.check_status()
    want, part = torch.zeros(2 * H, d, dtype=torch.float64, device="cuda:0"), torch.zeros(2 * H, d, dtype=torch.float64, device="cuda:0")
    D = Wd.double()
    for a, b, c, k in zip(dy.split(8192), x.split(8192), p.split(8192), heavy.split(8192)):
        g, u, dh = c[:, :H].double(), c[:, H:].double(), a.double() @ D
        s = torch.sigmoid(g)
        dp = torch.cat([dh * u * s * (1 + g * (1 - s)), dh * g * s], 1)
        want += dp.t() @ b.double()
        part += dp[k].t() @ b[k].double()
        del g, u, dh, s, dp
    assert float(part.norm()) > 0.9 * float(want.norm())
    assert float((dWgu.double() - want).norm()) <= 5e-3 * float(want.norm())
    for rows in (slice(0, 128), slice(H - 64, H + 64), slice(2 * H - 128, 2 * H)):      # gate, both, up
        assert float((dWgu[rows].double() - want[rows]).norm()) <= 5e-3 * float(want[rows].norm())


@pytest.mark.parametrize("both", [True, False])
def test_eight_bits_backward(both):
    from paper_2603_06626_b200 import binding as B
    T, K, N = 280000, 48, 8192
    dy, x, W = _rand(T, N, 6), _rand(T, K, 7), _rand(N, K, 8, K ** -0.5)
    middle = 2 ** 31 // N
    dy[middle - 200:middle + 200] *= 64
    dy[-100:] *= 64
    xt = B.quantize_fp8(x, rows=False, transposed=True)[1]
    Wt = B.quantize_fp8(W, square=True, rows=False, transposed=True)[1]
    if both:
        dx, dW, db = B.linear_fp8_backward(dy, xt, Wt, want_bias=True, dW_dtype=torch.float32)
    else:                                   # each product in a launch of its own
        dx = B.linear_fp8_backward(dy, None, Wt, want_dW=False)[0]
        _, dW, db = B.linear_fp8_backward(dy, xt, None, want_dx=False, want_bias=True, dW_dtype=torch.float32)
    B.check_status()
    Wv = B.dequantize_fp8(Wt, torch.float32).double()                       # [K, N]
    for s in _slices(T, N, 128):
        v = B.dequantize_fp8(B.quantize_fp8(dy[s])[0], torch.float32).double()
        want = v @ Wv.t()
        assert ((dx[s].double() - want).abs() <= (N / 16 + 32) * U * (v.abs() @ Wv.abs().t()) + 2.0 ** -8 * want.abs()).all()
    f64 = dict(dtype=torch.float64, device="cuda:0")
    want, size, sums, most = torch.zeros(N, K, **f64), torch.zeros(N, K, **f64), torch.zeros(N, **f64), torch.zeros(N, **f64)
    xv = B.dequantize_fp8(xt, torch.float32).double()                       # [K, T]
    step = 8192                                                             # whole blocks of 128 tokens: their scales are the same alone
    for t in range(0, T, step):
        g = dy[t:t + step]
        v = B.dequantize_fp8(B.quantize_fp8(g, rows=False, transposed=True)[1], torch.float32).double()
        want += v @ xv[:, t:t + step].t()
        size += v.abs() @ xv[:, t:t + step].abs().t()
        sums += g.double().sum(0)
        most += g.double().abs().sum(0)
    assert ((dW.double() - want).abs() <= (T / 16 + 32) * U * size).all()
    assert float((dW.double() - want).norm()) <= 1e-5 * float(want.norm())
    assert ((db.double() - sums).abs() <= (T / 16 + 32) * U * most).all()
    assert float((db.double() - sums).norm()) <= 1e-5 * float(sums.norm())
