"""The linear layer and its gradients against the fp64 oracle: one token to several tiles, ragged in every dimension.

Bounds, per element.  Operands are bf16 and their products exact in fp32; the tensor cores add 16 products at a time into an fp32
accumulator, each addition off by at most 2^-23 of the magnitudes added so far: (K/16 + 32) 2^-23 sum |x w| covers the sum, bias
and residual.  No activation stretches an error by more than 1.2; its own evaluation (fast exponential and quotient) is within
2^-18 of |z|.  Rounding to bf16 adds 2^-8 of the value (twice the half ulp).  In the backward pass dz is rounded to bf16 before the products:
2^-8 of sum |dz| |w|.  That bound is a worst case, so the relative Frobenius error is held to 5e-3 as well: two bf16 roundings,
each at most 2^-9 relative.
"""
import numpy as np
import pytest
import torch

from oracle import block_oracle as orc
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


def _forward(T, K, N, kind, bias, residual, pre, seed=0):
    from paper_2603_06626_b200 import binding as B
    rng = np.random.default_rng(seed + T + K + N)
    x, W = _bf(rng, T, K), _bf(rng, N, K, std=K ** -0.5)
    b = _bf(rng, N) if bias else None
    r = _bf(rng, T, N) if residual else None
    y, z = B.linear(x, W, bias=b, act=_act(kind), residual=r, save_pre=pre)
    y2, _ = B.linear(x, W, bias=b, act=_act(kind), residual=r, save_pre=pre)
    B.check_status()
    assert torch.equal(y, y2)
    xr, Wr, br, rr = f64(x), f64(W), None if b is None else f64(b), None if r is None else f64(r)
    yr, zr = orc.linear(xr, Wr, br, rr, kind)
    off = (K / 16 + 32) * U * (np.abs(xr) @ np.abs(Wr).T + (0 if br is None else np.abs(br)))
    bound = 1.2 * off + 2.0 ** -18 * np.abs(zr) + 2.0 ** -8 * np.abs(yr) + (0 if rr is None else 4 * U * np.abs(rr))
    assert (np.abs(f64(y) - yr) <= bound).all()
    if pre:
        assert (np.abs(f64(z) - zr) <= off + 2.0 ** -8 * np.abs(zr)).all()
    else:
        assert z is None


def _backward(T, K, N, kind, bias, dtype, seed=0):
    from paper_2603_06626_b200 import binding as B
    rng = np.random.default_rng(seed + T + K + N)
    x, W, dy = _bf(rng, T, K), _bf(rng, N, K, std=K ** -0.5), _bf(rng, T, N)
    z = None if kind == "none" else _bf(rng, T, N, std=2.0)
    dx, dW, db = B.linear_backward(dy, x, W, pre=z, act=_act(kind), want_bias=bias, dW_dtype=dtype)
    again = B.linear_backward(dy, x, W, pre=z, act=_act(kind), want_bias=bias, dW_dtype=dtype)
    B.check_status()
    for p, q in zip((dx, dW, db), again):
        assert p is None and q is None or torch.equal(p, q)
    assert dW.dtype == dtype and (db is not None) == bias
    xr, Wr, g = f64(x), f64(W), f64(dy)
    dxr, dWr, dbr, dz = orc.linear_backward(g, xr, Wr, np.zeros_like(g) if z is None else f64(z), kind)
    r = 0.0 if kind == "none" else 2.0 ** -8 + 2.0 ** -17
    mag = np.abs(dz) @ np.abs(Wr)
    assert (np.abs(f64(dx) - dxr) <= ((N / 16 + 32) * U + r) * mag + 2.0 ** -8 * np.abs(dxr)).all()
    mag = np.abs(dz).T @ np.abs(xr)
    assert (np.abs(f64(dW) - dWr) <= ((T / 16 + 32) * U + r) * mag + (2.0 ** -8 * np.abs(dWr) if dtype == torch.bfloat16 else 0)).all()
    if T * N >= 512:
        assert rel_frobenius(f64(dx), dxr) < 5e-3 and rel_frobenius(f64(dW), dWr) < 5e-3
    if bias:       # unrounded dz: only the slope's evaluation and the sum
        assert (np.abs(f64(db) - dbr) <= ((T + 64) * 2.0 ** -24 + 2.0 ** -17) * np.abs(g).sum(0) * 1.2 + 1e-30).all()


SIZES = [(1, 8, 8), (1, 64, 16), (1, 1024, 2048), (2, 4096, 520), (3, 72, 24), (8, 2048, 1408), (16, 264, 4096), (17, 512, 1000), (31, 2816, 128),
         (32, 1536, 4096), (33, 128, 136), (64, 1000, 1000), (65, 192, 256), (127, 256, 512), (128, 64, 264), (129, 320, 8), (255, 136, 248),
         (257, 1032, 520), (1000, 512, 1000), (4095, 136, 128), (2500, 72, 3000)]


@pytest.mark.parametrize("T,K,N", SIZES)
def test_forward_sizes(T, K, N):
    i = SIZES.index((T, K, N))
    _forward(T, K, N, KINDS[i % 4], bias=i % 2 == 0, residual=i % 3 == 0, pre=i % 5 < 2)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("bias,residual,pre", [(False, False, False), (True, True, True), (False, True, True), (True, False, True), (True, True, False)])
@pytest.mark.parametrize("T", [5, 300])
def test_forward_epilogues(kind, bias, residual, pre, T):
    _forward(T, 96, 328, kind, bias, residual, pre)


@pytest.mark.parametrize("T,K,N", SIZES)
def test_backward_sizes(T, K, N):
    i = SIZES.index((T, K, N))
    _backward(T, K, N, KINDS[i % 4], bias=i % 2 == 1, dtype=torch.float32 if i % 3 == 1 else torch.bfloat16)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_backward_variants(kind, bias, dtype):
    _backward(200, 136, 264, kind, bias, dtype)


def test_a_long_contraction_in_pieces():
    # a weight of one tile: the tokens are what there is to share out; f32 shows what the pieces' sum loses
    _backward(9000, 256, 256, "none", True, torch.float32)
    _backward(9000, 256, 256, "silu", True, torch.bfloat16)


def test_only_what_is_wanted():
    from paper_2603_06626_b200 import binding as B
    rng = np.random.default_rng(2)
    x, W, dy = _bf(rng, 70, 64), _bf(rng, 48, 64), _bf(rng, 70, 48)
    z = _bf(rng, 70, 48)
    full = B.linear_backward(dy, x, W, pre=z, act=B.ACT_GELU, want_bias=True)
    dx, none_w, none_b = B.linear_backward(dy, x, W, pre=z, act=B.ACT_GELU, want_dW=False)
    assert none_w is None and none_b is None and torch.equal(dx, full[0])
    none_x, dW, db = B.linear_backward(dy, x, W, pre=z, act=B.ACT_GELU, want_dx=False, want_bias=True)
    assert none_x is None and torch.equal(dW, full[1]) and torch.equal(db, full[2])


def test_extreme_pre_activations_and_values_that_are_not_finite():
    """Saturated activations stay finite; a NaN or infinity in one token's row touches that row only."""
    from paper_2603_06626_b200 import binding as B
    K = N = 64
    eye = torch.eye(K, device="cuda:0").bfloat16()
    x = torch.zeros(200, K, device="cuda:0").bfloat16()
    big = torch.tensor([0.0, 20.0, -20.0, 1e4, -1e4, 1e30, -1e30, 3e38], device="cuda:0").bfloat16()
    x[0, :8] = big
    for kind in KINDS:
        y, z = B.linear(x, eye, act=_act(kind), save_pre=True)
        want = orc.act(np.clip(f64(big), -50, 50), kind)
        got = f64(y[0, :8])
        assert np.isfinite(got).all() and torch.equal(z[0, :8], big)
        small = np.abs(f64(big)) <= 50
        assert (np.abs(got - want)[small] <= 2.0 ** -8 * np.abs(want[small]) + 1e-6).all()
        if kind != "none":
            assert (got[f64(big) <= -50] == 0).all() and (got[f64(big) >= 50] == f64(big)[f64(big) >= 50]).all()
            dy = torch.ones(200, N, device="cuda:0").bfloat16()
            dx, _, db = B.linear_backward(dy, x, eye, pre=z, act=_act(kind), want_bias=True)
            assert torch.isfinite(dx).all() and torch.isfinite(db).all()
    clean = B.linear(x, eye)[0]
    x[7, 3], x[150, 0] = float("nan"), float("inf")
    y = B.linear(x, eye)[0]
    rows = torch.ones(200, dtype=torch.bool, device="cuda:0")
    rows[7] = rows[150] = False
    assert torch.equal(y[rows], clean[rows]) and torch.isnan(y[7]).any() and not torch.isfinite(y[150]).all()


def test_no_tokens_and_the_residual_in_place():
    from paper_2603_06626_b200 import binding as B
    rng = np.random.default_rng(4)
    W = _bf(rng, 40, 64)
    none = torch.empty(0, 64, device="cuda:0").bfloat16()
    y, _ = B.linear(none, W)
    assert y.shape == (0, 40)
    dx, dW, db = B.linear_backward(torch.empty(0, 40, device="cuda:0").bfloat16(), none, W, want_bias=True)
    assert dx.shape == (0, 64) and (dW == 0).all() and (db == 0).all()
    for T in (4, 300):
        x, r = _bf(rng, T, 64), _bf(rng, T, 40)
        want, _ = B.linear(x, W, residual=r)
        status = torch.zeros(1, dtype=torch.int32, device="cuda:0")
        lib = B.load_library()
        assert lib.grouter_linear_fwd(x.data_ptr(), W.data_ptr(), None, r.data_ptr(), T, 64, 40, 0, r.data_ptr(), None, status.data_ptr(),
                                      torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
        assert torch.equal(r, want) and int(status) == 0


def test_another_stream_and_a_graph():
    from paper_2603_06626_b200 import binding as B
    rng = np.random.default_rng(8)
    x, W, b = _bf(rng, 600, 512), _bf(rng, 768, 512, std=0.05), _bf(rng, 768)
    want, z = B.linear(x, W, bias=b, act=B.ACT_SILU, save_pre=True)
    grads = B.linear_backward(want, x, W, pre=z, act=B.ACT_SILU, want_bias=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y, z2 = B.linear(x, W, bias=b, act=B.ACT_SILU, save_pre=True)
        g2 = B.linear_backward(y, x, W, pre=z2, act=B.ACT_SILU, want_bias=True)
    torch.cuda.synchronize()
    assert torch.equal(y, want) and all(torch.equal(p, q) for p, q in zip(grads, g2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y3, z3 = B.linear(x, W, bias=b, act=B.ACT_SILU, save_pre=True)
        g3 = B.linear_backward(y3, x, W, pre=z3, act=B.ACT_SILU, want_bias=True)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y3, want) and all(torch.equal(p, q) for p, q in zip(grads, g3))
    B.check_status()
