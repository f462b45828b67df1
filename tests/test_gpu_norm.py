"""Layer norm against the fp64 oracle: widths on both sides of every thread layout, odd widths, strided and unaligned rows.

Bounds, per element.  An fp32 sum of n terms added in a tree or in runs of at most 16 errs by less than (log2 n + 16) 2^-24 of the
sum of magnitudes, below 32 * 2^-24 here; mean, variance and the two sums of the backward pass each enter once, and a handful
of single operations follow: 128 * 2^-24 of the magnitudes involved covers them.  On top comes the rounding of the output:
2^-8 of the value for bf16 (twice its half-ulp bound, since the fp32 value may sit on the other side of a tie), nothing for f32.
dw and db add up to `rows` terms one after the other: (rows + 64) 2^-24 of the sum of magnitudes.
"""
import numpy as np
import pytest
import torch

from oracle import block_oracle as orc
from tests.gpu_util import bf16_to_f64 as f64

pytestmark = pytest.mark.gpu

EPS = 1e-5
U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _out_bound(ty, ref, mags):
    return (2.0 ** -8 * np.abs(ref) if ty == "bf16" else 0.0) + 128 * U * mags + 1e-30


def _matrix(rng, T, d, ty, pad, shift):
    """A [T,d] view into a wider tensor: rows `pad` further apart than they are long, first row `shift` elements in."""
    base = torch.from_numpy(rng.normal(size=(T, d + pad)).astype(np.float32) * 1.5 + 0.3).to("cuda:0").to(TYPES[ty]).reshape(-1)
    flat = torch.empty(base.numel() + shift + pad, dtype=TYPES[ty], device="cuda:0")
    flat[shift:shift + base.numel()] = base
    return flat[shift:].as_strided((T, d), (d + pad, 1))


def _check_forward(x, w, b, ty, eps=EPS):
    from paper_2603_06626_b200 import binding as B
    y, mean, rstd = B.layer_norm(x, w, b, eps)
    xr, wr, br = f64(x), f64(w), None if b is None else f64(b)
    yr, mr, rr = orc.layer_norm(xr, wr, br, eps)
    mags = (np.abs(xr) + np.abs(mr)[:, None]) * rr[:, None] * np.abs(wr) + (0 if br is None else np.abs(br))
    # the centred values feed the variance: their error relative to the spread grows with |mean| rstd
    grow = 1 + np.abs(mr * rr)[:, None]
    assert (np.abs(f64(y) - yr) <= _out_bound(ty, yr, mags * grow)).all()
    assert (np.abs(f64(mean) - mr) <= 128 * U * np.abs(xr).mean(1) + 1e-30).all()
    assert (np.abs(f64(rstd) - rr) <= 128 * U * rr * (1 + np.abs(mr * rr)) ** 2).all()
    return y, mean, rstd


def _check_backward(dy, x, w, ty):
    from paper_2603_06626_b200 import binding as B
    T, d = x.shape
    _, mean, rstd = B.layer_norm(x, w, None, EPS)
    dx, dw, db = B.layer_norm_backward(dy, x, w, mean, rstd)
    again = B.layer_norm_backward(dy, x, w, mean, rstd)
    assert all(torch.equal(p, q) for p, q in zip((dx, dw, db), again))          # bit-reproducible
    only, dw2, none = B.layer_norm_backward(dy, x, w, mean, rstd, want_bias=False)
    assert none is None and torch.equal(only, dx) and torch.equal(dw2, dw)
    g, xr, wr, mr, rr = f64(dy), f64(x), f64(w), f64(mean), f64(rstd)
    dxr, dwr, dbr = orc.layer_norm_backward(g, xr, wr, mr, rr)
    h = (np.abs(xr) + np.abs(mr)[:, None]) * rr[:, None]
    gw = np.abs(g * wr)
    mags = rr[:, None] * (gw + gw.mean(1, keepdims=True) + h * (gw * h).mean(1, keepdims=True))
    assert (np.abs(f64(dx) - dxr) <= _out_bound(ty, dxr, mags)).all()
    assert (np.abs(f64(dw) - dwr) <= (T + 64) * U * (np.abs(g) * h).sum(0) + 1e-30).all()
    assert (np.abs(f64(db) - dbr) <= (T + 64) * U * np.abs(g).sum(0) + 1e-30).all()


# (rows, width, activations, weights, row padding, first element): aligned and not, every thread layout, widths of one element
CASES = [(1, 1, "f32", "f32", 0, 0), (3, 2, "bf16", "bf16", 0, 0), (1, 8, "bf16", "f32", 0, 0), (9, 31, "f32", "bf16", 0, 0),
         (7, 64, "bf16", "bf16", 8, 0), (17, 100, "f32", "f32", 4, 0), (300, 511, "bf16", "bf16", 0, 0), (33, 512, "f32", "f32", 0, 0),
         (40, 513, "f32", "bf16", 0, 1), (65, 520, "bf16", "f32", 8, 8), (1000, 1000, "bf16", "bf16", 0, 0), (5, 2048, "f32", "f32", 0, 0),
         (300, 2048, "bf16", "f32", 0, 3), (6, 2056, "bf16", "bf16", 0, 0), (700, 4096, "bf16", "bf16", 0, 0), (4, 4096, "f32", "f32", 1, 0),
         (3, 4104, "bf16", "bf16", 0, 0), (5, 8192, "f32", "bf16", 0, 0), (3, 8191, "bf16", "f32", 0, 0), (160, 8200, "bf16", "bf16", 0, 0),
         (4, 16384, "f32", "f32", 0, 0), (200, 16384, "bf16", "f32", 0, 0), (2, 16383, "f32", "bf16", 0, 0), (4096, 96, "bf16", "bf16", 0, 0)]


@pytest.mark.parametrize("T,d,ty,wt,pad,shift", CASES)
def test_both_passes(T, d, ty, wt, pad, shift):
    rng = np.random.default_rng(T * 7 + d)
    x = _matrix(rng, T, d, ty, pad, shift)
    w = torch.from_numpy((rng.normal(size=d) * 0.3 + 1).astype(np.float32)).to("cuda:0").to(TYPES[wt])
    b = torch.from_numpy(rng.normal(size=d).astype(np.float32)).to("cuda:0").to(TYPES[wt])
    _check_forward(x, w, b, ty)
    _check_forward(x, w, None, ty)
    if d > 1:
        dy = torch.from_numpy(rng.normal(size=(T, d)).astype(np.float32)).to("cuda:0").to(TYPES[ty])
        _check_backward(dy, x, w, ty)


def test_unaligned_gradient_and_weights():
    rng = np.random.default_rng(1)
    x = _matrix(rng, 50, 256, "f32", 0, 0)
    dy = _matrix(rng, 50, 256, "f32", 0, 1)
    w = torch.randn(257, device="cuda:0")[1:]
    _check_backward(dy, x, w, "f32")
    _check_forward(x, w, w, "f32")


def test_constant_rows_and_rows_far_from_zero():
    x = torch.full((4, 1024), 3.0, device="cuda:0")
    x[1] = 0.0
    x[2] = 1000.0 + torch.randn(1024, device="cuda:0")
    w, b = torch.ones(1024, device="cuda:0"), torch.full((1024,), 0.5, device="cuda:0")
    y, mean, rstd = _check_forward(x, w, b, "f32")
    assert (y[:2] == 0.5).all() and torch.isfinite(y).all()


@pytest.mark.parametrize("d", [96, 1024, 4096])
def test_a_row_that_is_not_finite_stays_alone(d):
    from paper_2603_06626_b200 import binding as B
    x = torch.randn(20, d, device="cuda:0")
    clean = B.layer_norm(x, torch.ones(d, device="cuda:0"))[0]
    x[3, 5], x[11, 0] = float("nan"), float("inf")
    y = B.layer_norm(x, torch.ones(d, device="cuda:0"))[0]
    bad = torch.zeros(20, dtype=torch.bool, device="cuda:0")
    bad[3] = bad[11] = True
    assert torch.isnan(y[3]).all() and torch.isnan(y[11]).any()
    assert torch.equal(y[~bad], clean[~bad])


def test_no_rows():
    from paper_2603_06626_b200 import binding as B
    x = torch.empty(0, 256, device="cuda:0")
    w = torch.ones(256, device="cuda:0")
    y, mean, rstd = B.layer_norm(x, w)
    assert y.shape == (0, 256) and mean.shape == (0,)
    dx, dw, db = B.layer_norm_backward(x, x, w, mean, rstd)
    assert dx.shape == (0, 256) and (dw == 0).all() and (db == 0).all()


def test_another_stream_and_a_graph():
    from paper_2603_06626_b200 import binding as B
    x, w = torch.randn(500, 2048, device="cuda:0"), torch.randn(2048, device="cuda:0")
    want = B.layer_norm(x, w)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = B.layer_norm(x, w)
        back = B.layer_norm_backward(x, x, w, got[1], got[2])
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = B.layer_norm_backward(x, x, w, want[1], want[2])
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
    y, mean, rstd = B.layer_norm(x, w)
    dx, _, _ = B.layer_norm_backward(dy, x, w, mean, rstd)
    h = 2.0 ** -6
    f = lambda v: (B.layer_norm(v, w)[0].double() * dy.double()).sum()  # noqa: E731
    num = ((f(x + h * u) - f(x - h * u)) / (2 * h)).item()
    ana = (dx.double() * u.double()).sum().item()
    scale = (dx.double() * u.double()).abs().sum().item()
    assert abs(num - ana) <= 1e-3 * scale


# rows on boundaries of two elements only, and of more where the weights are not; matrices on both sides of 2^21 elements, which is
# where aligned rows go from two accesses a lane to four: every number of warps a row
PAIRS = [(1, 2, "bf16", "bf16", 0, 2), (37, 66, "bf16", "f32", 0, 0), (19, 514, "f32", "bf16", 0, 0), (300, 1022, "bf16", "bf16", 2, 4),
         (65, 1026, "f32", "f32", 6, 2), (40, 2050, "bf16", "bf16", 0, 0), (17, 4094, "f32", "bf16", 0, 0), (7, 8190, "bf16", "f32", 8, 0),
         (5, 8194, "f32", "f32", 0, 0), (3, 16382, "bf16", "bf16", 0, 0), (2, 16382, "f32", "bf16", 0, 0), (4, 4095, "bf16", "bf16", 0, 0),
         (4, 4097, "f32", "f32", 0, 0)]
SPREADS = [(2049, 1024, "bf16", "bf16", 0, 0), (2048, 1024, "f32", "f32", 0, 0), (2051, 1032, "bf16", "f32", 8, 0), (1025, 2048, "f32", "bf16", 0, 0),
           (514, 4104, "bf16", "bf16", 0, 0), (257, 8200, "f32", "f32", 0, 0), (129, 16384, "bf16", "bf16", 0, 0), (130, 16384, "f32", "f32", 0, 0),
           (9, 1024, "f32", "bf16", 0, 0), (9, 4100, "f32", "f32", 0, 0), (9, 8192, "bf16", "bf16", 0, 0)]


@pytest.mark.parametrize("T,d,ty,wt,pad,shift", PAIRS + SPREADS)
def test_pairs_and_spreads(T, d, ty, wt, pad, shift):
    test_both_passes(T, d, ty, wt, pad, shift)


@pytest.mark.parametrize("ty", ["bf16", "f32"])
def test_pairs_of_activations_over_unaligned_weights(ty):
    rng = np.random.default_rng(2)
    x = _matrix(rng, 33, 514, ty, 2, 2)
    dy = _matrix(rng, 33, 514, ty, 0, 2)
    for first in (1, 2):
        w = torch.randn(514 + first, device="cuda:0").to(TYPES[ty])[first:]
        _check_forward(x, w, w, ty)
        _check_backward(dy, x, w, ty)


# several rows to a warp: more than one round of resident blocks whose last round is not full, and fewer rows than a warp takes
SHARED = [(9999, 128, "f32", "f32", 0, 0), (20001, 64, "bf16", "bf16", 0, 0), (10007, 200, "bf16", "f32", 8, 0), (9475, 100, "bf16", "bf16", 0, 0),
          (9473, 33, "f32", "bf16", 0, 1), (9474, 255, "bf16", "bf16", 0, 0), (2, 128, "bf16", "bf16", 0, 0), (3, 256, "f32", "f32", 0, 0),
          (5, 24, "bf16", "bf16", 0, 0), (31, 129, "f32", "f32", 0, 0), (1, 127, "bf16", "f32", 0, 0), (33, 16, "f32", "f32", 0, 0)]


@pytest.mark.parametrize("T,d,ty,wt,pad,shift", SHARED)
def test_rows_that_share_a_warp(T, d, ty, wt, pad, shift):
    """Thousands of rows hold elements whose value and mean are both next to zero, where the error of the mean (a part of mean |x|,
    not of |mean|) is what counts: 128 * 2^-24 of mean |x|, the bound of the mean itself, is added to the magnitudes."""
    from paper_2603_06626_b200 import binding as B
    rng = np.random.default_rng(T * 7 + d)
    x = _matrix(rng, T, d, ty, pad, shift)
    w = torch.from_numpy((rng.normal(size=d) * 0.3 + 1).astype(np.float32)).to("cuda:0").to(TYPES[wt])
    b = torch.from_numpy(rng.normal(size=d).astype(np.float32)).to("cuda:0").to(TYPES[wt])
    xr, wr = f64(x), f64(w)
    for bias in (b, None):
        br = 0 * wr if bias is None else f64(bias)
        y, mean, rstd = B.layer_norm(x, w, bias, EPS)
        yr, mr, rr = orc.layer_norm(xr, wr, br, EPS)
        size = np.abs(xr).mean(1)
        mags = (np.abs(xr) + np.abs(mr)[:, None] + size[:, None]) * rr[:, None] * np.abs(wr) + np.abs(br)
        assert (np.abs(f64(y) - yr) <= _out_bound(ty, yr, mags * (1 + np.abs(mr * rr)[:, None]))).all()
        assert (np.abs(f64(mean) - mr) <= 128 * U * size + 1e-30).all()
        assert (np.abs(f64(rstd) - rr) <= 128 * U * rr * (1 + np.abs(mr * rr)) ** 2).all()
    dy = torch.from_numpy(rng.normal(size=(T, d)).astype(np.float32)).to("cuda:0").to(TYPES[ty])
    _check_backward(dy, x, w, ty)
