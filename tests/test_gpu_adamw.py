"""AdamW over many tensors against the fp64 oracle, in 32 and in 8 bits.

Bounds: m and v are two products and a sum, each rounded to f32: 4 * 2^-24 of |b1 m| + |(1-b1) g| (and of v's two positive terms),
plus 2^-23 relative for the rounded coefficients.  The step is a handful of roundings of lr/c1 m / (sqrt(v)/sqrt(c2) + eps): 16 * 2^-24
of it and of |p|, plus what the error of m brings.  8-bit moments: from the oracle's own codes of the kernel's f32 results.
"""
import numpy as np
import pytest
import torch

from oracle import block_oracle as orc
from tests.gpu_util import bf16_to_f64 as f64

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HY = dict(lr=2e-3, betas=(0.9, 0.95), eps=1e-8)
SIZES = [1, 2, 3, 31, 32, 33, 100, 255, 1024, 4097, 8192, 8193, 30000]


def _tensors(sizes, ptype, gtype, seed=0, shift=0):
    """Parameters and gradients, each `shift` elements into an allocation of its own."""
    g = torch.Generator().manual_seed(seed)
    P, G = [], []
    for n in sizes:
        P.append(torch.randn(n + shift, generator=g).to("cuda:0").to(ptype)[shift:])
        G.append((torch.randn(n + shift, generator=g) * 0.01).to("cuda:0").to(gtype)[shift:])
    return P, G


def _step_reference(opt, p, g, m, v, wd, t, scale):
    return orc.adamw(p, g, m, v, HY["lr"], *HY["betas"], HY["eps"], wd, t, scale)


@pytest.mark.parametrize("ptype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("gtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("shift", [0, 1])
def test_three_steps(ptype, gtype, bits, shift):
    from paper_2603_06626_b200 import binding as B
    P, G = _tensors(SIZES, ptype, gtype, shift=shift)
    wd = [0.1 if i % 2 else 0.0 for i in range(len(P))]
    opt = B.AdamW(P, G, weight_decay=wd, state_bits=bits, **HY)
    scale = torch.tensor([0.7], device="cuda:0")
    sc = float(scale)
    for t in range(1, 4):
        src = [opt.master[o:o + p.numel()] if ptype == torch.bfloat16 else p for p, o in zip(P, opt.offsets)]
        before = [f64(s.clone()) for s in src]
        m0, v0 = [f64(x.clone()) for x in opt.moments()]
        opt.step(grad_scale=scale)
        m1, v1 = [f64(x) for x in opt.moments()]
        for i, (p, g, o) in enumerate(zip(P, G, opt.offsets)):
            n = p.numel()
            s = slice(o, o + n)
            pr, mr, vr = _step_reference(opt, before[i], f64(g), m0[s], v0[s], wd[i], t, sc)
            gm = np.abs(f64(g)) * sc
            moff = 8 * U * (0.9 * np.abs(m0[s]) + 0.1 * gm)
            rate = HY["lr"] / (1 - 0.9 ** t) / (np.sqrt(vr) / np.sqrt(1 - 0.95 ** t) + HY["eps"])
            tol = 16 * U * (np.abs(before[i]) + rate * np.abs(mr)) + rate * moff * 2
            assert (np.abs(f64(src[i]) - pr) <= tol).all()
            if ptype == torch.bfloat16:
                assert torch.equal(p, src[i].bfloat16())
            if bits == 32:
                assert (np.abs(m1[s] - mr) <= moff + 1e-45).all()
                assert (np.abs(v1[s] - vr) <= 12 * U * vr + 1e-45).all()
            else:
                # within the codes' rounding of the exact moments: half a step of 3 mantissa bits, the smallest code at the low end
                for got, ref in ((m1[s], mr), (np.sqrt(v1[s]), np.sqrt(vr))):
                    pad = np.zeros((n + 31) // 32 * 32)
                    pad[:n] = np.abs(ref)
                    top = np.repeat(pad.reshape(-1, 32).max(1), 32)[:n]
                    assert (np.abs(got - ref) <= np.maximum(np.abs(ref) / 16, top / 448 * 2 * 2.0 ** -9) * (1 + 1e-5)).all()
                assert (v1[s][vr > 0] > 0).all()           # a root that is there stays there
        if bits == 32:                                     # nothing between the tensors is written
            hole = np.ones(len(m1), bool)
            for p, o in zip(P, opt.offsets):
                hole[o:o + p.numel()] = False
            assert (m1[hole] == 0).all() and (v1[hole] == 0).all()
    assert opt.steps_done == 3


def test_codes_are_the_oracles():
    """beta1 = beta2 = 0: the new moments are g and g^2 exactly, so the codes can be compared byte for byte."""
    from paper_2603_06626_b200 import binding as B
    rng = np.random.default_rng(0)
    x = rng.normal(size=32 * 40) * np.exp(rng.normal(size=32 * 40) * 2)
    x[:32] = 0                                             # an empty group
    x[32:64] = np.r_[1.0, 1e-9, -1e-9, np.zeros(29)]       # below the smallest code
    x[64:96] = 448.0 * 2.0 ** -np.arange(32)
    x[96:128] = -449.0 * 2.0 ** -np.arange(32)
    x[128:160] = np.r_[17.0, 18.0, 19.0, 34.0, 448.0, np.arange(27) / 3]      # ties between codes
    x[160:192] = np.float32(1e-20)                         # a root of 1e-20, squares far below the normal range of f32
    x[192:224] = np.r_[np.float32(1e18), np.ones(31)]      # wider than a group's codes reach
    x = x.astype(np.float32)
    p, g = torch.zeros(len(x), device="cuda:0"), torch.from_numpy(x).to("cuda:0")
    opt = B.AdamW([p], [g], lr=0.0, betas=(0.0, 0.0), eps=1e-3, weight_decay=0.0, state_bits=8)
    opt.step()
    codes, exps = orc.encode8(x.astype(np.float64), False)
    assert np.array_equal(opt.m.cpu().numpy(), codes) and np.array_equal(opt.m_exp.cpu().numpy(), exps)
    root = np.sqrt((x * x).astype(np.float32))             # f32, correctly rounded, as the kernel computes it
    codes, exps = orc.encode8(root.astype(np.float64), True)
    assert np.array_equal(opt.v.cpu().numpy(), codes) and np.array_equal(opt.v_exp.cpu().numpy(), exps)
    m, v = opt.moments()
    assert np.array_equal(f64(m), orc.decode8(opt.m.cpu().numpy(), opt.m_exp.cpu().numpy()).astype(np.float32))
    r = orc.decode8(codes, exps).astype(np.float32)
    assert np.array_equal(v.cpu().numpy(), r * r)


def test_a_lost_spike_does_not_blow_up_the_step():
    """An old spike leaves a large root beside small ones in its group: the small ones' steps stay bounded."""
    from paper_2603_06626_b200 import binding as B
    p, g = torch.zeros(32, device="cuda:0"), torch.full((32,), 1e-6, device="cuda:0")
    g[0] = 100.0
    opt = B.AdamW([p], [g], lr=1e-3, betas=(0.9, 0.999), eps=1e-12, weight_decay=0.0, state_bits=8)
    opt.step()
    g[0] = 0.0
    for _ in range(40):
        opt.step()
    assert torch.isfinite(p).all() and p.abs().max() < 1.0


def test_a_gradient_that_is_not_finite_stays_alone():
    from paper_2603_06626_b200 import binding as B
    for bits in (32, 8):
        p, g = torch.ones(96, device="cuda:0"), torch.ones(96, device="cuda:0")
        g[40] = float("nan")
        g[41] = float("inf")
        opt = B.AdamW([p], [g], state_bits=bits, **HY)
        opt.step()
        ok = torch.ones(96, dtype=torch.bool, device="cuda:0")
        ok[40] = ok[41] = False
        assert torch.isfinite(p[ok]).all() and not torch.isfinite(p[~ok]).any()
        if bits == 8:
            m, v = opt.moments()
            assert not torch.isfinite(m[40:42]).any() and not torch.isfinite(v[40:42]).any() and torch.isfinite(m[:32]).all() and torch.isfinite(m[64:]).all()
            assert torch.isfinite(m[32:64][ok[32:64]]).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_a_run_continued_from_its_state_is_the_same_run(bits):
    from paper_2603_06626_b200 import binding as B
    P, G = _tensors([50, 3000], torch.bfloat16, torch.float32)
    opt = B.AdamW(P, G, state_bits=bits, **HY)
    for _ in range(2):
        opt.step()
    keys = ["m", "v", "master"] + (["m_exp", "v_exp"] if bits == 8 else [])
    Q = [p.clone() for p in P]
    two = B.AdamW(Q, G, state_bits=bits, state={k: getattr(opt, k).clone() for k in keys}, steps_done=2, **HY)
    opt.step()
    two.step()
    assert all(torch.equal(p, q) for p, q in zip(P, Q)) and all(torch.equal(getattr(opt, k), getattr(two, k)) for k in keys)


def test_empty_tensors_shapes_and_mixed_types():
    from paper_2603_06626_b200 import binding as B
    a, b, c = torch.randn(7, 9, device="cuda:0"), torch.empty(0, 5, device="cuda:0"), torch.randn(4, 33, device="cuda:0").bfloat16()
    g = [torch.randn_like(a).bfloat16(), torch.empty_like(b), torch.randn(4, 33, device="cuda:0")]
    a0, c0 = f64(a.clone()), f64(c.clone())
    opt = B.AdamW([a, b, c], g, weight_decay=0.05, **HY)
    opt.step()
    pr, _, _ = orc.adamw(a0, f64(g[0]), 0 * a0, 0 * a0, HY["lr"], *HY["betas"], HY["eps"], 0.05, 1)
    assert np.abs(f64(a) - pr).max() < 1e-6
    pr, _, _ = orc.adamw(c0, f64(g[2]), 0 * c0, 0 * c0, HY["lr"], *HY["betas"], HY["eps"], 0.05, 1)
    assert (np.abs(f64(c) - pr) <= 2.0 ** -8 * np.abs(pr) + 1e-6).all()
    B.AdamW([b], [g[1]], **HY).step()                       # nothing to do


def test_many_tensors_on_another_stream():
    from paper_2603_06626_b200 import binding as B
    P, G = _tensors([17 + 13 * i for i in range(700)], torch.float32, torch.float32)
    Q = [p.clone() for p in P]
    one = B.AdamW(P, G, **HY)
    one.step()
    two = B.AdamW(Q, G, **HY)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        two.step()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(P, Q))
