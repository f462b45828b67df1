"""The dense branch's operators on matrices of more than 2^31 elements: rows on both sides of the place where 32-bit offsets end, against the
same rows given alone (bit by bit where a row's arithmetic does not depend on how many there are) or against fp64.

Tolerances: as in the tests of the single operators, bf16 outputs are within 2^-8 of the value and (K/16 + 32) 2^-23 of the sum of magnitudes;
the gated block, whose hidden state is rounded to bf16 on the way, within 5e-3 in relative Frobenius norm."""
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -23


def _rand(rows, cols, seed, std=1.0):
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda:0")
    for part in x.split(1 << 14):
        part.normal_(0.0, std, generator=g)
    return x


def _slices(rows, cols, n):
    """Row ranges at the start, around offset 2^31 and at the end, starting on multiples of 128."""
    middle = (2 ** 31 // cols) // 128 * 128
    assert rows * cols > 2 ** 31 + 2 ** 27
    return [slice(a, a + n) for a in (0, middle - 128, (rows - n) // 128 * 128)]


def test_norm_and_quantizer():
    from paper_2603_06626_b200 import binding as B
    T, d = 142000, 16384
    x, w = _rand(T, d, 0), torch.linspace(0.5, 1.5, d, device="cuda:0")
    y, _, rstd = B.rms_norm(x, w)
    q8 = B.rms_norm(x, w, fp8=True)[0]
    back = B.dequantize_fp8(q8)
    dx, dw = B.rms_norm_backward(y, x, w, rstd, dh=x)
    for s in _slices(T, d, 256):
        one = B.rms_norm(x[s], w)
        assert torch.equal(y[s], one[0]) and torch.equal(rstd[s], one[2])
        assert torch.equal(back[s], B.dequantize_fp8(B.rms_norm(x[s], w, fp8=True)[0]))
        assert torch.equal(dx[s], B.rms_norm_backward(y[s], x[s], w, rstd[s], dh=x[s])[0])
    want = sum((a.double() * b.double() * r.double()[:, None]).sum(0) for a, b, r in zip(y.split(4096), x.split(4096), rstd.split(4096)))
    size = sum((a.double() * b.double() * r.double()[:, None]).abs().sum(0) for a, b, r in zip(y.split(4096), x.split(4096), rstd.split(4096)))
    assert ((dw.double() - want).abs() <= (T + 64) * 2.0 ** -24 * size).all()
    del y, back, dx, q8
    q, t = B.quantize_fp8(x, transposed=True)
    for s in _slices(T, d, 256):
        one, turned = B.quantize_fp8(x[s], transposed=True)
        codes = lambda m: m.codes.view(torch.uint8)  # noqa: E731
        assert torch.equal(codes(q)[s], codes(one)) and torch.equal(q.scale_exponents()[s], one.scale_exponents())
        assert torch.equal(codes(t)[:, s], codes(turned))
        assert torch.equal(t.scale_exponents()[:, s.start // 128:s.start // 128 + 2], turned.scale_exponents())


def test_linear_in_8_bits():
    from paper_2603_06626_b200 import binding as B
    T, K, N = 280000, 48, 8192
    x, r = _rand(T, K, 1), _rand(T, N, 2)
    W8 = B.quantize_fp8(_rand(N, K, 3, K ** -0.5), square=True)[0]
    y = B.linear_fp8(x, W8, residual=r)
    B.check_status()
    W = B.dequantize_fp8(W8, torch.float32).double()
    for s in _slices(T, N, 128):
        v = B.dequantize_fp8(B.quantize_fp8(x[s])[0], torch.float32).double()
        want = v @ W.t() + r[s].double()
        off = (K / 16 + 32) * U * (v.abs() @ W.abs().t() + r[s].double().abs())
        assert ((y[s].double() - want).abs() <= off + 2.0 ** -8 * want.abs()).all()


def test_gated_block():
    from paper_2603_06626_b200 import binding as B
    T, d, H = 140000, 16, 8192
    x, Wgu, Wd = _rand(T, d, 4), _rand(2 * H, d, 5, d ** -0.5), _rand(d, H, 6, H ** -0.5)
    y, p = B.gated_ffn(x, Wgu, Wd, residual=x, save_pre=True)
    W8 = [B.quantize_fp8(W.contiguous(), square=True)[0] for W in (Wgu[:H], Wgu[H:], Wd)]
    y8 = B.gated_ffn_fp8(x, *W8, residual=x)
    dy = _rand(T, d, 7)
    dx, dWgu, dWd = B.gated_ffn_backward(dy, x, Wgu, Wd, p)
    B.check_status()

    def near(got, want):
        return float((got.double() - want).norm() / want.norm()) <= 5e-3

    G, Uw, D = Wgu[:H].double(), Wgu[H:].double(), Wd.double()
    for s in _slices(T, 2 * H, 256):
        v = x[s].double()
        g, u = v @ G.t(), v @ Uw.t()
        assert near(p[s], torch.cat([g, u], 1)) and near(y[s].double() - v, (torch.nn.functional.silu(g) * u) @ D.t())
        small = B.gated_ffn_fp8(x[s].contiguous(), *W8, residual=x[s].contiguous())
        assert near(y8[s].double() - v, small.double() - v)
        g, u = p[s, :H].double(), p[s, H:].double()
        a, sig, dh = torch.nn.functional.silu(g), torch.sigmoid(g), dy[s].double() @ D
        assert near(dx[s], (dh * u * sig * (1 + g * (1 - sig))) @ G + (dh * a) @ Uw)
    want = torch.zeros(d, H, dtype=torch.float64, device="cuda:0")
    for a, b in zip(dy.split(8192), p.split(8192)):
        want += a.double().t() @ (torch.nn.functional.silu(b[:, :H].double()) * b[:, H:].double())
    assert near(dWd, want) and torch.isfinite(dWgu.float()).all()
