"""Expert counts, balance and z losses and the gradient of the scores against the fp64 oracle.

Counts are whole numbers: equal.  Bounds for the gradient, per element: p of a row is off by a few times 2^-22 relative (fast
exponential of a difference, a sum of at most 1024 terms in a tree), the sum a = sum f p by the same share of itself, and a
gate's term by 2^-20 of the magnitudes in it; 2^-19 of (ca/n) p (f + a) + (2 cz/n) |lse| p + |gate terms| covers the whole, on top comes
the rounding of the output to bf16 (2^-8).  Differences s - top of the scores are exact to 2^-24 of their size, which enters p as an
absolute error of the exponent: 2^-23 (|s| + |top|) p on top.  Losses: 2^-18 of their value (all terms are positive).
"""
import numpy as np
import pytest
import torch

from oracle import block_oracle as orc
from tests.gpu_util import bf16_to_f64 as f64

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
CA, CZ = 0.37, 0.021


def _inputs(T, E, k, ty, idx, seed=0, pad=0, mask=None):
    rng = np.random.default_rng(seed + 31 * T + E)
    s = torch.from_numpy(rng.normal(size=(T, E + pad)).astype(np.float32) * 2).to("cuda:0").to(TYPES[ty])[:, :E]
    order = np.argsort(-f64(s), 1, kind="stable")[:, :k]
    i = torch.from_numpy(np.ascontiguousarray(order.astype(np.uint8 if idx == "u8" else np.int32))).to("cuda:0")
    m = None
    if mask == "some":
        m = torch.from_numpy((rng.random(T) < 0.6).astype(np.uint8)).to("cuda:0")
    elif mask == "none":
        m = torch.zeros(T, dtype=torch.bool, device="cuda:0")
    dg = torch.from_numpy(rng.normal(size=(T, k)).astype(np.float32)).to("cuda:0")
    return s, i, m, dg


def _check(s, i, m, dg, norm, ca=CA, cz=CZ, dloss=None):
    from paper_2603_06626_b200 import binding as B
    T, E = s.shape
    ty = "bf16" if s.dtype == torch.bfloat16 else "f32"
    counts, n = B.expert_counts(i, E, mask=m)
    ir, mr = i.cpu().numpy(), None if m is None else m.cpu().numpy()
    cr, nr = orc.expert_counts(ir, E, mr)
    assert np.array_equal(counts.cpu().numpy(), cr) and int(n) == nr
    up = None if dloss is None else torch.tensor([dloss], device="cuda:0")
    nm = B.NORM_SOFTMAX if norm == "softmax" else B.NORM_SIGMOID
    loss, d = B.balance_loss(s, i, counts, n, mask=m, balance_coef=ca, z_coef=cz, dgates=dg, norm=nm, dloss=up)
    alone, none = B.balance_loss(s, i, counts, n, mask=m, balance_coef=ca, z_coef=cz, norm=nm, want_grad=False)
    none2, d2 = B.balance_loss(s, i, counts, n, mask=m, balance_coef=ca, z_coef=cz, dgates=dg, norm=nm, want_loss=False, dloss=up)
    B.check_status()
    assert none is None and none2 is None and torch.equal(loss, alone) and torch.equal(d, d2)
    sr, scale = f64(s), 1.0 if dloss is None else dloss
    want = orc.balance_loss(sr, cr, nr, ca, cz, mr)
    assert np.allclose(f64(loss), want, rtol=2.0 ** -18, atol=1e-30)
    dr = scale * orc.balance_gradient(sr, cr, nr, ca, cz, mr)
    live = np.ones(T, bool) if mr is None else mr != 0
    p, lse = orc._softmax(sr)
    f = cr * (E / cr.sum()) if cr.sum() else np.zeros(E)
    mag = abs(scale) / max(nr, 1) * p * (ca * (f + (p @ f)[:, None]) + 2 * cz * np.abs(lse)[:, None])
    top = np.abs(sr).max(1, keepdims=True)
    bound = mag * (2.0 ** -19 + 2.0 ** -23 * (np.abs(sr) + top))
    if dg is not None:
        g = f64(dg)
        dr = dr + orc.balance_gradient(sr, cr, 0, 0, 0, mr, ir, g, norm)
        q = orc.gates(np.take_along_axis(sr, ir.astype(np.int64), 1), norm)
        each = q * (np.abs(g) + ((q * np.abs(g)).sum(1, keepdims=True) if norm == "softmax" else 0))
        add = np.zeros((T, E))
        np.put_along_axis(add, ir.astype(np.int64), each, 1)
        bound = bound + add * (2.0 ** -19 + 2.0 ** -22 * top)
    got = f64(d)
    assert (got[~live] == 0).all()
    err = np.abs(got - dr)[live]
    lim = (bound + (2.0 ** -8 * np.abs(dr) if ty == "bf16" else 0) + 1e-30)[live]
    assert (err <= lim).all(), (err / lim).max()


CASES = [(1, 8, 2, "f32", "u8", 0), (1, 1, 1, "f32", "i32", 0), (5, 3, 3, "bf16", "u8", 0), (64, 8, 8, "bf16", "u8", 0), (77, 8, 1, "f32", "i32", 0),
         (500, 16, 2, "bf16", "i32", 0), (333, 60, 6, "bf16", "u8", 0), (333, 60, 6, "f32", "u8", 0), (1000, 64, 8, "f32", "u8", 4),
         (1000, 64, 8, "bf16", "u8", 3), (2049, 128, 8, "f32", "u8", 0), (700, 160, 6, "bf16", "i32", 0), (513, 256, 8, "bf16", "u8", 0),
         (99, 256, 32, "f32", "u8", 0), (40, 257, 4, "f32", "i32", 0), (50, 512, 8, "bf16", "i32", 0), (31, 777, 12, "f32", "i32", 0),
         (20, 1000, 8, "bf16", "i32", 0), (30, 1024, 16, "f32", "i32", 0), (12, 1023, 32, "bf16", "i32", 0), (30, 1024, 8, "bf16", "i32", 0)]


@pytest.mark.parametrize("T,E,k,ty,idx,pad", CASES)
@pytest.mark.parametrize("norm", ["softmax", "sigmoid"])
def test_sizes(T, E, k, ty, idx, pad, norm):
    s, i, m, dg = _inputs(T, E, k, ty, idx, pad=pad, mask="some" if (T + E) % 2 else None)
    _check(s, i, m, dg, norm)
    if norm == "softmax":
        _check(s, i, m, None, norm)


def test_many_tokens():
    # more tokens than one round of the grid, with the partial sums of many blocks
    s, i, m, dg = _inputs(40000, 16, 2, "f32", "u8", mask="some")
    _check(s, i, m, None, "softmax")


@pytest.mark.parametrize("dloss", [0.0, 1.0, -3.5])
def test_upstream_gradient_scales_the_losses_only(dloss):
    s, i, m, dg = _inputs(50, 24, 3, "f32", "u8")
    _check(s, i, m, dg, "softmax", dloss=dloss)


def test_nothing_counts():
    from paper_2603_06626_b200 import binding as B
    for T in (7, 3000):
        s, i, m, dg = _inputs(T, 32, 4, "f32", "u8", mask="none")
        counts, n = B.expert_counts(i, 32, mask=m)
        loss, d = B.balance_loss(s, i, counts, n, mask=m, balance_coef=CA, z_coef=CZ, dgates=dg)
        assert int(n) == 0 and (counts == 0).all() and (loss == 0).all() and (d == 0).all()
    e = torch.empty(0, 4, dtype=torch.uint8, device="cuda:0")
    counts, n = B.expert_counts(e, 32)
    loss, d = B.balance_loss(torch.empty(0, 32, device="cuda:0"), e, counts, n)
    assert int(n) == 0 and (counts == 0).all() and (loss == 0).all() and d.shape == (0, 32)


@pytest.mark.parametrize("E", [8, 40, 128, 300])
def test_scores_that_take_experts_out(E):
    """-inf and the type's lowest value in some places, in all but one, in a whole row; finite results that follow the formula."""
    from paper_2603_06626_b200 import binding as B
    low = torch.finfo(torch.float32).min
    s, i, m, dg = _inputs(6, E, 2, "f32", "i32")
    s = s.contiguous()
    s[0, 1::2] = -float("inf")
    s[1, 1:] = -float("inf")
    s[2] = -float("inf")
    s[3, 1::2] = low
    s[4, 1:] = low
    order = np.argsort(-f64(s), 1, kind="stable")[:, :2].astype(np.int32)
    i = torch.from_numpy(np.ascontiguousarray(order)).to("cuda:0")
    counts, n = B.expert_counts(i, E)
    loss, d = B.balance_loss(s, i, counts, n, balance_coef=CA, z_coef=CZ, dgates=dg)
    cr, nr = orc.expert_counts(order, E)
    with np.errstate(invalid="ignore"):
        want = orc.balance_gradient(f64(s), cr, nr, CA, CZ, None, order, f64(dg), "softmax")
    assert torch.isfinite(d).all() and torch.isfinite(loss).all()
    assert (d[2] == 0).all() and (d[0, 1::2] == 0).all() and (d[1, 1:] == 0).all()
    assert np.allclose(f64(d), want, rtol=1e-5, atol=1e-6)
    assert np.allclose(f64(loss), orc.balance_loss(f64(s), cr, nr, CA, CZ), rtol=1e-5)


def test_a_row_of_the_lowest_value():
    """Every score the lowest value: p is even, lse^2 overflows; with a zero coefficient the z term is left out of the sum."""
    from paper_2603_06626_b200 import binding as B
    s = torch.full((3, 16), torch.finfo(torch.float32).min, device="cuda:0")
    i = torch.zeros(3, 1, dtype=torch.uint8, device="cuda:0")
    counts, n = B.expert_counts(i, 16)
    loss, d = B.balance_loss(s, i, counts, n, balance_coef=1.0, z_coef=0.0)
    assert abs(float(loss[0]) - 1.0) < 1e-5 and float(loss[2]) == float("inf") and torch.isfinite(d).all()


def test_masked_rows_may_hold_anything():
    from paper_2603_06626_b200 import binding as B
    s, i, m, dg = _inputs(200, 48, 4, "bf16", "u8")
    m = torch.ones(200, dtype=torch.uint8, device="cuda:0")
    m[10], m[77] = 0, 0
    counts, n = B.expert_counts(i, 48, mask=m)
    want = B.balance_loss(s, i, counts, n, mask=m, dgates=dg)
    s2, i2, dg2 = s.clone(), i.clone(), dg.clone()
    s2[10], s2[77], i2[10], dg2[10] = float("nan"), float("inf"), 255, float("nan")
    c2, n2 = B.expert_counts(i2, 48, mask=m)
    got = B.balance_loss(s2, i2, c2, n2, mask=m, dgates=dg2)
    B.check_status()
    assert torch.equal(c2, counts) and torch.equal(n2, n) and all(torch.equal(p, q) for p, q in zip(want, got))
    assert (got[1][10] == 0).all()


def test_an_id_out_of_range_is_reported_and_skipped():
    from paper_2603_06626_b200 import binding as B
    status = torch.zeros(1, dtype=torch.int32, device="cuda:0")
    s, i, m, dg = _inputs(300, 20, 3, "f32", "i32")
    bad = i.clone()
    bad[5, 1], bad[299, 2] = 20, -1
    counts, n = B.expert_counts(bad, 20, status=status)
    assert int(status) == 1 and int(n) == 300 and int(counts.sum()) == 898
    status.zero_()
    good, _ = B.balance_loss(s, i, counts, n, dgates=dg, status=status)
    assert int(status) == 0
    _, d = B.balance_loss(s, bad, counts, n, dgates=dg, status=status)
    assert int(status) == 1 and torch.isfinite(d).all()
    B.expert_counts(bad, 20)
    with pytest.raises(B.GrouterError):
        B.check_status()
    B.check_status()                      # cleared


def test_an_expert_twice_in_a_token():
    """After a fold of the ids a token may name one expert twice: both slots' gradients land on its score."""
    s, i, m, dg = _inputs(64, 12, 4, "f32", "u8")
    i[:, 2] = i[:, 0]
    from paper_2603_06626_b200 import binding as B
    counts, n = B.expert_counts(i, 12)
    _, d = B.balance_loss(s, i, counts, n, balance_coef=CA, z_coef=CZ, dgates=dg)
    cr, nr = orc.expert_counts(i.cpu().numpy(), 12)
    want = orc.balance_gradient(f64(s), cr, nr, CA, CZ, None, i.cpu().numpy(), f64(dg), "softmax")
    assert np.allclose(f64(d), want, rtol=1e-5, atol=2e-6)


def test_counts_of_other_ranks_and_a_graph():
    """Counts summed over ranks change the shares; a whole pass captured and replayed gives the same."""
    from paper_2603_06626_b200 import binding as B
    s, i, m, dg = _inputs(257, 32, 4, "f32", "u8")
    counts, n = B.expert_counts(i, 32)
    far = counts * 3 + 1000000000 // 16
    loss, d = B.balance_loss(s, i, far, n, balance_coef=CA, z_coef=CZ)
    cr = far.cpu().numpy().astype(np.int64)
    assert np.allclose(f64(d), orc.balance_gradient(f64(s), cr, 257, CA, CZ), rtol=2e-5, atol=1e-9)
    assert np.allclose(f64(loss), orc.balance_loss(f64(s), cr, 257, CA, CZ), rtol=1e-5)
    graph = torch.cuda.CUDAGraph()
    B.balance_loss(s, i, counts, n, dgates=dg)
    with torch.cuda.graph(graph):
        c2, n2 = B.expert_counts(i, 32)
        held = B.balance_loss(s, i, c2, n2, dgates=dg)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    want = B.balance_loss(s, i, counts, n, dgates=dg)
    assert torch.equal(c2, counts) and all(torch.equal(p, q) for p, q in zip(held, want))


def test_gradient_against_differences_of_the_kernel():
    """Central differences of the f32 loss, along the gradient: loss values are good to 2^-22, the step moves them by 1e-3 of it."""
    from paper_2603_06626_b200 import binding as B
    s, i, m, dg = _inputs(40, 16, 2, "f32", "u8")
    counts, n = B.expert_counts(i, 16)
    f = lambda v: float(B.balance_loss(v, i, counts, n, balance_coef=1.0, z_coef=0.1, want_grad=False)[0][0].double())  # noqa: E731
    _, d = B.balance_loss(s, i, counts, n, balance_coef=1.0, z_coef=0.1)
    u = d / d.norm()
    h = 0.25
    num = (f(s + h * u) - f(s - h * u)) / (2 * h)
    assert abs(num - float(d.norm())) <= 2e-2 * float(d.norm())
