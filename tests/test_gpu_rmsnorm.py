"""Root-mean-square norm on a residual stream against the fp64 oracle: every thread layout, odd widths, strided and unaligned rows, codes.

Bounds, per element.  A sum of n squares added in a tree or in runs of at most 16 errs by less than 32 * 2^-24 of the sum; rstd takes the
root of it, and a handful of single operations follow: 128 * 2^-24 of the magnitudes covers them.  The output's rounding adds 2^-8 of the
value for bf16 (twice its half-ulp bound, since the fp32 value may sit on the other side of a tie), nothing for f32.  h is one sum,
rounded to fp32 and to its type: 2^-8 of it for bf16 by the same argument, 2^-24 for f32.  Codes may stand for anything between what
the value less and the value plus its error bound are rounded to, under one of the scales that these bounds have.
dw adds up `rows` terms one after the other: (rows + 64) 2^-24 of the sum of magnitudes.
"""
import numpy as np
import pytest
import torch

from oracle import branch_oracle as orc
from tests.gpu_util import bf16_to_f64 as f64

pytestmark = pytest.mark.gpu

EPS = 1e-6
U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _matrix(rng, T, d, ty, pad=0, shift=0, std=1.5):
    """A [T,d] view into a wider tensor: rows `pad` further apart than they are long, first row `shift` elements in."""
    base = torch.from_numpy(rng.normal(size=(T, d + pad)).astype(np.float32) * std + 0.2).to("cuda:0").to(TYPES[ty]).reshape(-1)
    flat = torch.empty(base.numel() + shift + pad, dtype=TYPES[ty], device="cuda:0")
    flat[shift:shift + base.numel()] = base
    return flat[shift:].as_strided((T, d), (d + pad, 1))


def _weights(rng, d, wt, shift=0):
    return torch.from_numpy((rng.normal(size=d + shift) * 0.3 + 1).astype(np.float32)).to("cuda:0").to(TYPES[wt])[shift:]


def _between(v, err, got):
    """Whether `got` lies between what v - err and v + err are rounded to, under a scale that one of the bounds asks for."""
    lo, hi = np.minimum(v - err, v + err), np.maximum(v - err, v + err)
    a = np.maximum(np.abs(v) - err, 0.0)
    ok = np.zeros(v.shape, bool)
    least, most = orc.exponents(a), orc.exponents(np.abs(v) + err)
    for e in (least, most):
        ql, _ = orc.quantized(np.maximum(lo, -448.0 * 2.0 ** np.repeat(e, 128, 1)[:, :v.shape[1]]), exps=e)
        qh, _ = orc.quantized(np.minimum(hi, 448.0 * 2.0 ** np.repeat(e, 128, 1)[:, :v.shape[1]]), exps=e)
        ok |= (got >= ql) & (got <= qh)
    return ok, least, most


def _forward(x, w, r, ty, fp8=False):
    from paper_2603_06626_b200 import binding as B
    y, h, rstd = B.rms_norm(x, w, residual=r, eps=EPS, fp8=fp8)
    again = B.rms_norm(x, w, residual=r, eps=EPS, fp8=fp8)
    assert torch.equal(again[1], h) and torch.equal(again[2], rstd)
    if r is None:
        assert h is x
    else:
        hr = f64(x) + f64(r)
        assert h.is_contiguous() and (np.abs(f64(h) - hr) <= (2.0 ** -8 if ty == "bf16" else U) * np.abs(hr)).all()
    yr, rr = orc.rms_norm(f64(h), f64(w), EPS)
    assert (np.abs(f64(rstd) - rr) <= 64 * U * rr).all()
    off = 128 * U * np.abs(yr) + 1e-30
    if not fp8:
        assert torch.equal(again[0], y)
        assert (np.abs(f64(y) - yr) <= off + (2.0 ** -8 if ty == "bf16" else 0.0) * np.abs(yr)).all()
        return y, h, rstd
    assert torch.equal(again[0].codes.view(torch.uint8), y.codes.view(torch.uint8))
    assert torch.equal(again[0].scale_exponents(), y.scale_exponents())
    ok, least, most = _between(yr, off, f64(B.dequantize_fp8(y, torch.float32)))
    assert ok.all()
    e = y.scale_exponents().cpu().numpy().astype(np.int64) - 127
    assert ((e == least) | (e == most)).all()
    return y, h, rstd


def _backward(rng, h, w, ty, dh):
    from paper_2603_06626_b200 import binding as B
    T, d = h.shape
    dy = _matrix(rng, T, d, ty)
    dy, along = dy.contiguous(), _matrix(rng, T, d, ty).contiguous() if dh else None
    _, _, rstd = B.rms_norm(h, w, eps=EPS)
    dx, dw = B.rms_norm_backward(dy, h, w, rstd, dh=along)
    again = B.rms_norm_backward(dy, h, w, rstd, dh=along)
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])          # bit-reproducible
    g, hr, wr, rr = f64(dy), f64(h), f64(w), f64(rstd)
    a = None if along is None else f64(along)
    dxr, dwr = orc.rms_norm_backward(g, hr, wr, rr, a)
    u = np.abs(hr) * rr[:, None]
    gw = np.abs(g * wr)
    mags = rr[:, None] * (gw + u * (gw * u).mean(1, keepdims=True)) + (0 if a is None else np.abs(a))
    assert (np.abs(f64(dx) - dxr) <= 128 * U * mags + (2.0 ** -8 * np.abs(dxr) if ty == "bf16" else 0.0) + 1e-30).all()
    assert (np.abs(f64(dw) - dwr) <= (T + 64) * U * (np.abs(g) * u).sum(0) + 1e-30).all()


# (rows, width, activations, weights, row padding, first element): aligned and not, every thread layout, widths of one element
CASES = [(1, 1, "f32", "f32", 0, 0), (3, 2, "bf16", "bf16", 0, 0), (1, 8, "bf16", "f32", 0, 0), (9, 31, "f32", "bf16", 0, 0),
         (7, 64, "bf16", "bf16", 8, 0), (17, 100, "f32", "f32", 4, 0), (300, 511, "bf16", "bf16", 0, 0), (33, 512, "f32", "f32", 0, 0),
         (40, 513, "f32", "bf16", 0, 1), (65, 520, "bf16", "f32", 8, 8), (1000, 1000, "bf16", "bf16", 0, 0), (5, 2048, "f32", "f32", 0, 0),
         (300, 2048, "bf16", "f32", 0, 3), (6, 2056, "bf16", "bf16", 0, 0), (700, 4096, "bf16", "bf16", 0, 0), (4, 4096, "f32", "f32", 1, 0),
         (5, 8192, "f32", "bf16", 0, 0), (3, 8191, "bf16", "f32", 0, 0), (160, 8200, "bf16", "bf16", 0, 0), (4, 16384, "f32", "f32", 0, 0),
         (200, 16384, "bf16", "f32", 0, 0), (2, 16383, "f32", "bf16", 0, 0), (4096, 96, "bf16", "bf16", 0, 0), (37, 66, "bf16", "f32", 0, 0),
         (17, 4094, "f32", "bf16", 0, 0), (3, 16382, "bf16", "bf16", 0, 0), (9999, 128, "f32", "f32", 0, 0), (9475, 100, "bf16", "bf16", 0, 0),
         (1, 127, "bf16", "f32", 0, 0), (2049, 1024, "bf16", "bf16", 0, 0), (514, 4104, "bf16", "bf16", 0, 0), (130, 16384, "f32", "f32", 0, 0),
         (2, 24, "bf16", "bf16", 0, 0), (3001, 264, "f32", "f32", 0, 0)]


@pytest.mark.parametrize("T,d,ty,wt,pad,shift", CASES)
def test_both_passes(T, d, ty, wt, pad, shift):
    rng = np.random.default_rng(T * 7 + d)
    x, w = _matrix(rng, T, d, ty, pad, shift), _weights(rng, d, wt)
    _forward(x, w, None, ty)
    _, h, _ = _forward(x, w, _matrix(rng, T, d, ty, 0, shift), ty)
    _backward(rng, h, w, ty, True)
    _backward(rng, x, w, ty, False)


CODES = [(1, 16, "bf16", "bf16", 0), (5, 48, "f32", "f32", 0), (129, 128, "bf16", "f32", 8), (33, 272, "f32", "bf16", 4), (260, 512, "bf16", "bf16", 0),
         (7, 1008, "bf16", "bf16", 0), (1, 4096, "bf16", "bf16", 0), (1000, 2048, "bf16", "f32", 16), (300, 2064, "f32", "f32", 0),
         (3, 8192, "bf16", "bf16", 0), (131, 16384, "bf16", "f32", 0), (3, 16384, "f32", "f32", 0), (2, 16368, "bf16", "bf16", 0),
         (2100, 1024, "bf16", "bf16", 0), (10001, 144, "bf16", "bf16", 0)]


@pytest.mark.parametrize("T,d,ty,wt,pad", CODES)
def test_codes(T, d, ty, wt, pad):
    rng = np.random.default_rng(T * 3 + d)
    x, w = _matrix(rng, T, d, ty, pad), _weights(rng, d, wt)
    x[:, ::17] *= 30
    _forward(x, w, None, ty, fp8=True)
    _forward(x, w, _matrix(rng, T, d, ty, 16), ty, fp8=True)


def test_strides_of_both_inputs_and_unaligned_weights():
    rng = np.random.default_rng(4)
    x, r = _matrix(rng, 50, 256, "bf16", 8), _matrix(rng, 50, 256, "bf16", 24, 8)
    for first in (0, 1, 2):
        w = _weights(rng, 256, "bf16", first)
        _forward(x, w, r, "bf16")
        _backward(rng, x, w, "bf16", True)
    _forward(x, _weights(rng, 256, "f32", 1), _matrix(rng, 50, 256, "bf16", 0, 1), "bf16")


@pytest.mark.parametrize("d", [96, 1024, 4096])
def test_a_row_that_is_not_finite_stays_alone(d):
    from paper_2603_06626_b200 import binding as B
    x, w = torch.randn(20, d, device="cuda:0"), torch.ones(d, device="cuda:0")
    bad = torch.zeros(20, dtype=torch.bool, device="cuda:0")
    bad[3] = bad[11] = True
    clean, clean8 = B.rms_norm(x, w)[0], B.dequantize_fp8(B.rms_norm(x, w, fp8=True)[0])
    x[3, 5], x[11, 0] = float("nan"), float("inf")
    y, y8 = B.rms_norm(x, w)[0], B.dequantize_fp8(B.rms_norm(x, w, fp8=True)[0])
    assert torch.isnan(y[3]).all() and torch.isnan(y8[3]).all() and torch.isnan(y[11, 0]) and torch.isnan(y8[11, 0])
    assert torch.equal(y[~bad], clean[~bad]) and torch.equal(y8[~bad], clean8[~bad])


def test_rows_of_zeros():
    from paper_2603_06626_b200 import binding as B
    x, w = torch.zeros(3, 256, device="cuda:0", dtype=torch.bfloat16), torch.ones(256, device="cuda:0")
    y, h, rstd = B.rms_norm(x, w, residual=x, eps=EPS)
    assert (y == 0).all() and (h == 0).all() and torch.isfinite(rstd).all()
    q = B.rms_norm(x, w, eps=EPS, fp8=True)[0]
    assert (B.dequantize_fp8(q) == 0).all() and (q.scale_exponents() == 1).all()
    dx, dw = B.rms_norm_backward(x, x, w, rstd, dh=x)
    assert (dx == 0).all() and (dw == 0).all()


def test_no_rows():
    from paper_2603_06626_b200 import binding as B
    x, w = torch.empty(0, 256, device="cuda:0"), torch.ones(256, device="cuda:0")
    y, h, rstd = B.rms_norm(x, w, residual=x)
    assert y.shape == h.shape == (0, 256) and rstd.shape == (0,)
    assert B.rms_norm(x, w, fp8=True)[0].shape == (0, 256)
    dx, dw = B.rms_norm_backward(x, x, w, rstd)
    assert dx.shape == (0, 256) and (dw == 0).all()


def test_another_stream_and_a_graph():
    from paper_2603_06626_b200 import binding as B
    x, w = torch.randn(500, 2048, device="cuda:0"), torch.randn(2048, device="cuda:0")
    want = B.rms_norm(x, w, residual=x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = B.rms_norm(x, w, residual=x)
        back = B.rms_norm_backward(x, got[1], w, got[2], dh=x)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = B.rms_norm_backward(x, want[1], w, want[2], dh=x)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(held, back))


def test_gradient_against_differences_of_the_kernel():
    """Directional derivative of sum(y * dy) by central differences of the f32 kernel.  Step 2^-6: the third-order term is below
    h^2 of the value's scale, and rounding (1e-6 of it) over the step below 1e-4."""
    from paper_2603_06626_b200 import binding as B
    torch.manual_seed(0)
    x, w, dy, u = (torch.randn(64, 640, device="cuda:0") for _ in range(4))
    w = w[0].contiguous()
    _, _, rstd = B.rms_norm(x, w)
    dx, _ = B.rms_norm_backward(dy, x, w, rstd)
    s = 2.0 ** -6
    f = lambda v: (B.rms_norm(v, w)[0].double() * dy.double()).sum()  # noqa: E731
    num = ((f(x + s * u) - f(x - s * u)) / (2 * s)).item()
    ana, scale = (dx.double() * u.double()).sum().item(), (dx.double() * u.double()).abs().sum().item()
    assert abs(num - ana) <= 1e-3 * scale
