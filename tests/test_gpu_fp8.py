"""Matrices in 8 bits and products on them against the fp64 oracle: whole and ragged blocks, both forms, one token to several tiles.

Putting a matrix into 8 bits is exact but for the one rounding that the definition has: codes and scales are equal to the oracle's.
Products: two e4m3 numbers multiply exactly in fp32, powers of two change nothing; the tensor cores add 32 products at a time into an
fp32 accumulator, each addition off by at most 2^-23 of the magnitudes added so far: (K/16 + 32) 2^-23 sum |x w| covers the sum, bias and
residual (in steps of 16, as for bf16, since how many products meet in one step is the hardware's).  Rounding to bf16 adds 2^-8 of the value
(twice the half ulp), to f32 nothing more.  The column sums of dy are fp32: (T/128 + 64) 2^-24 of the magnitudes.
"""
import numpy as np
import pytest
import torch

from oracle import branch_oracle as orc
from oracle.grouter_oracle import rel_frobenius
from tests.gpu_util import bf16_to_f64 as f64

pytestmark = pytest.mark.gpu

U = 2.0 ** -23


def _rand(rng, R, C, dtype=torch.bfloat16, std=1.0):
    x = rng.normal(size=(R, C)) * std * 2.0 ** rng.integers(-3, 4, (R, 1))
    x[:, ::37] *= 20
    return torch.from_numpy(x.astype(np.float32)).to("cuda:0").to(dtype)


def _same(q, x, square=False):
    """Codes, scales and values of q are those of the oracle for x.  A code's value has 4 bits: exact in f32 and bf16, but that the very
    largest elements are rounded up to 2^128 (3.4e38 = 255.8 * 2^120, between the codes 240 and 256), which both types call infinity."""
    from paper_2603_06626_b200 import binding as B
    want, e = orc.quantized(x, square)
    want = np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)
    assert np.array_equal(q.scale_exponents().cpu().numpy().astype(np.int64), e + 127)
    for dtype in (torch.float32, torch.bfloat16):
        assert np.array_equal(f64(B.dequantize_fp8(q, dtype)), want, equal_nan=True)
    pad = q.codes.view(torch.uint8)[:, q.cols:]
    assert (pad == 0).all()


SHAPES = [(1, 1), (1, 16), (3, 100), (128, 128), (129, 127), (17, 513), (200, 1000), (1000, 136), (5, 4096), (300, 2056), (1, 8200), (1025, 24)]


@pytest.mark.parametrize("R,C", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("square", [False, True])
def test_codes_and_scales_of_both_forms(R, C, dtype, square):
    from paper_2603_06626_b200 import binding as B
    x = _rand(np.random.default_rng(R + C), R, C, dtype)
    if C > 2:
        x[R // 2, C // 2] = 0
    xr = f64(x)
    q, t = B.quantize_fp8(x, square=square, transposed=True)
    assert q.shape == (R, C) and t.shape == (C, R)
    _same(q, xr, square)
    _same(t, xr.T, square)
    only, none = B.quantize_fp8(x, square=square)
    assert none is None and torch.equal(only.codes.view(torch.uint8), q.codes.view(torch.uint8))
    none, only = B.quantize_fp8(x, square=square, rows=False, transposed=True)
    assert none is None and torch.equal(only.codes.view(torch.uint8), t.codes.view(torch.uint8))


@pytest.mark.parametrize("pad,shift", [(8, 0), (0, 1), (3, 5)])
def test_strided_and_unaligned_rows(pad, shift):
    from paper_2603_06626_b200 import binding as B
    rng = np.random.default_rng(5)
    flat = torch.from_numpy(rng.normal(size=70 * (264 + pad) + shift).astype(np.float32)).to("cuda:0").bfloat16()
    x = flat[shift:].as_strided((70, 264), (264 + pad, 1))
    q, t = B.quantize_fp8(x, transposed=True)
    _same(q, f64(x))
    _same(t, f64(x).T)


def test_extremes():
    """Zeros, the largest and smallest numbers, values on ties and on the borders of a scale, infinities and NaN."""
    from paper_2603_06626_b200 import binding as B
    x = torch.zeros(8, 256, device="cuda:0")
    x[1, :4] = torch.tensor([3.4e38, -3.4e38, 1.0, 1e-38])
    x[2, :3] = torch.tensor([1e-40, 1e-45, -3e-39])
    x[3, 0], x[3, 128] = 448.0, 448.0 * (1 + 2.0 ** -23)
    x[4, :127] = torch.from_numpy(orc.NUMBERS.astype(np.float32))
    x[4, 128:254] = torch.from_numpy(((orc.NUMBERS[1:] + orc.NUMBERS[:-1]) / 2).astype(np.float32))
    x[4, 254] = 448.0
    x[5] = -x[4]
    x[6, 3], x[6, 5], x[6, 7], x[6, 9] = float("inf"), float("-inf"), float("nan"), 2.0
    x[7] = float("nan")
    q, t = B.quantize_fp8(x, transposed=True)
    _same(q, f64(x))
    _same(t, f64(x).T)
    assert int(torch.isnan(B.dequantize_fp8(q)[6]).sum()) == 3


def _product(T, K, N, bias=False, residual=False, codes=True):
    from paper_2603_06626_b200 import binding as B
    rng = np.random.default_rng(T + K + N)
    x, W = _rand(rng, T, K), _rand(rng, N, K, std=K ** -0.5)
    b = torch.from_numpy(rng.normal(size=N).astype(np.float32)).to("cuda:0").bfloat16() if bias else None
    r = _rand(rng, T, N) if residual else None
    Wq = B.quantize_fp8(W, square=True)[0]
    arg = B.quantize_fp8(x)[0] if codes else x
    y = B.linear_fp8(arg, Wq, bias=b, residual=r)
    assert torch.equal(y, B.linear_fp8(arg, Wq, bias=b, residual=r))
    B.check_status()
    xr, Wr = orc.quantized(f64(x))[0], orc.quantized(f64(W), square=True)[0]
    extra = (0 if b is None else f64(b)) + (0 if r is None else f64(r))
    size = (0 if b is None else np.abs(f64(b))) + (0 if r is None else np.abs(f64(r)))
    want = xr @ Wr.T + extra
    off = (K / 16 + 32) * U * (np.abs(xr) @ np.abs(Wr).T + size)
    assert (np.abs(f64(y) - want) <= off + 2.0 ** -8 * np.abs(want)).all()
    assert rel_frobenius(f64(y), want) <= 2.0 ** -8
    return y


PRODUCTS = [(1, 1, 8), (1, 128, 8), (2, 16, 16), (7, 72, 24), (16, 512, 136), (33, 520, 264), (64, 4096, 256), (65, 1000, 1000), (130, 129, 128),
            (255, 640, 520), (256, 512, 256), (257, 1536, 264), (500, 2056, 384), (1, 4096, 4096), (1031, 896, 1032), (3, 8192, 64)]


@pytest.mark.parametrize("T,K,N", PRODUCTS)
def test_forward(T, K, N):
    _product(T, K, N)
    _product(T, K, N, bias=True, residual=True, codes=False)


def test_more_tiles_than_pairs():
    """Several rounds of the resident pairs: both accumulators in turn, contractions of one step and of a few."""
    _product(5000, 128, 2048, bias=True)
    _product(4100, 640, 1800, residual=True)


def test_rows_that_are_not_finite_stay_alone():
    from paper_2603_06626_b200 import binding as B
    rng = np.random.default_rng(8)
    W = B.quantize_fp8(_rand(rng, 264, 384), square=True)[0]
    for T in (5, 300):
        x = _rand(rng, T, 384)
        clean = B.linear_fp8(x, W)
        x[3, 7] = float("nan")
        y = B.linear_fp8(x, W)
        keep = torch.arange(T, device="cuda:0") != 3
        assert torch.isnan(y[3]).all() and torch.equal(y[keep], clean[keep])


@pytest.mark.parametrize("T", [1, 5, 8, 9, 16, 17, 40])
@pytest.mark.parametrize("K,N,pad", [(8, 8, 0), (72, 264, 8), (520, 136, 0), (1000, 392, 24), (4096, 1032, 0), (2056, 64, 3)])
def test_tokens_as_they_are_and_as_codes_give_the_same(T, K, N, pad):
    """Few tokens are put into 8 bits on their way into the product, others by a kernel before it: the codes are the same ones."""
    from paper_2603_06626_b200 import binding as B
    rng = np.random.default_rng(T + K)
    x = _rand(rng, T, K + pad)[:, :K]
    x[T // 2, K // 2] = 0
    if T > 4:
        x[3, 1], x[2, K - 1], x[1, 0] = float("nan"), float("inf"), float("-inf")
    W, b = B.quantize_fp8(_rand(rng, N, K, std=K ** -0.5), square=True)[0], _rand(rng, 1, N)[0]
    y = B.linear_fp8(x, W, bias=b)
    assert torch.equal(y.view(torch.int16), B.linear_fp8(B.quantize_fp8(x)[0], W, bias=b).view(torch.int16))
    bad = torch.isnan(y).any(1).cpu()
    assert bad[1:4].all() and int(bad.sum()) == 3 if T > 4 else not bad.any()


def _backward(T, K, N, dtype=torch.bfloat16, bias=True):
    from paper_2603_06626_b200 import binding as B
    rng = np.random.default_rng(T + K + N)
    x, W, dy = _rand(rng, T, K), _rand(rng, N, K, std=K ** -0.5), _rand(rng, T, N)
    xt, Wt = B.quantize_fp8(x, rows=False, transposed=True)[1], B.quantize_fp8(W, square=True, rows=False, transposed=True)[1]
    got = B.linear_fp8_backward(dy, xt, Wt, want_bias=bias, dW_dtype=dtype)
    again = B.linear_fp8_backward(dy, xt, Wt, want_bias=bias, dW_dtype=dtype)
    B.check_status()
    assert all(p is None and q is None or torch.equal(p, q) for p, q in zip(got, again))
    dx, dW, db = got
    assert dW.dtype == dtype and (db is not None) == bias
    g, xr, Wr = f64(dy), orc.quantized(f64(x).T)[0], orc.quantized(f64(W).T, square=True)[0]
    for out, a, b, kind in ((dx, orc.quantized(g)[0], Wr, torch.bfloat16), (dW, orc.quantized(g.T)[0], xr, dtype)):
        want = a @ b.T
        off = (a.shape[1] / 16 + 32) * U * (np.abs(a) @ np.abs(b).T)
        assert (np.abs(f64(out) - want) <= off + (2.0 ** -8 if kind == torch.bfloat16 else 0.0) * np.abs(want)).all()
    if bias:
        assert (np.abs(f64(db) - g.sum(0)) <= (T / 128 + 64) * 2.0 ** -24 * np.abs(g).sum(0) + 1e-30).all()


@pytest.mark.parametrize("T,K,N", [(1, 8, 8), (3, 128, 16), (130, 256, 136), (257, 72, 264), (1000, 520, 384), (2050, 384, 640), (129, 1032, 8)])
def test_backward(T, K, N):
    _backward(T, K, N)
    _backward(T, K, N, torch.float32, False)


@pytest.mark.parametrize("T,K,N", [(8200, 264, 136), (5000, 1032, 520), (20001, 16, 24)])
def test_backward_of_many_tokens_and_a_small_weight(T, K, N):
    """The weight gradient's contraction is cut into pieces that are added up: one more rounding for each piece, which the bound's 32 covers."""
    _backward(T, K, N)
    _backward(T, K, N, torch.float32, False)


def test_gradients_one_by_one_and_into_given_tensors():
    from paper_2603_06626_b200 import binding as B
    rng = np.random.default_rng(9)
    x, W, dy = _rand(rng, 200, 136), _rand(rng, 72, 136), _rand(rng, 200, 72)
    xt, Wt = B.quantize_fp8(x, transposed=True)[1], B.quantize_fp8(W, square=True, transposed=True)[1]
    dx, dW, db = B.linear_fp8_backward(dy, xt, Wt, want_bias=True)
    a = B.linear_fp8_backward(dy, None, Wt, want_dW=False)
    b = B.linear_fp8_backward(dy, xt, None, want_dx=False)
    c = B.linear_fp8_backward(dy, None, None, want_dx=False, want_dW=False, want_bias=True)
    assert torch.equal(a[0], dx) and a[1] is None and torch.equal(b[1], dW) and b[0] is None and torch.equal(c[2], db)
    into, sums = torch.full((72, 136), 7.0, device="cuda:0"), torch.full((72,), 7.0, device="cuda:0")
    d = B.linear_fp8_backward(dy, xt, Wt, dW=into, db=sums)
    assert d[1] is into and d[2] is sums and torch.equal(sums, db) and torch.equal(into.bfloat16(), dW)


def test_no_tokens():
    from paper_2603_06626_b200 import binding as B
    rng = np.random.default_rng(10)
    W = _rand(rng, 24, 128)
    x = torch.empty(0, 128, dtype=torch.bfloat16, device="cuda:0")
    Wq, Wt = B.quantize_fp8(W, square=True, transposed=True)
    q, xt = B.quantize_fp8(x, transposed=True)
    assert B.linear_fp8(q, Wq).shape == (0, 24) and B.linear_fp8(x, Wq).shape == (0, 24) and B.dequantize_fp8(q).shape == (0, 128)
    dx, dW, db = B.linear_fp8_backward(B.linear_fp8(x, Wq), xt, Wt, want_bias=True)
    assert dx.shape == (0, 128) and (dW == 0).all() and (db == 0).all()


def test_streams_graphs_and_a_status_word_of_its_own():
    from paper_2603_06626_b200 import binding as B
    rng = np.random.default_rng(11)
    x, dy = _rand(rng, 300, 256), _rand(rng, 300, 128)
    Wq, Wt = B.quantize_fp8(_rand(rng, 128, 256), square=True, transposed=True)
    status = torch.zeros(1, dtype=torch.int32, device="cuda:0")

    def step():
        q, t = B.quantize_fp8(x, transposed=True)
        return (B.linear_fp8(q, Wq, status=status), *B.linear_fp8_backward(dy, t, Wt, want_bias=True, status=status))

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
    B.check_status(status=status)
    for h in held:
        assert all(torch.equal(p, q) for p, q in zip(want, h))
