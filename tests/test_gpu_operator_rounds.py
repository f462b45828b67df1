"""The operators around the expert layer where their kernels come round: sizes past the first round of resident blocks, the last round
not full, derived from the launch rules and this GPU's number of SMs.  Bounds as in the operators' own tests."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as orc
from oracle.grouter_oracle import rel_frobenius
from tests.gpu_util import bf16_to_f64 as f64

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24


def _sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


def _normal(shape, std=1.0, mean=0.0, ty="f32", seed=0):
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    return torch.empty(shape, device="cuda:0").normal_(mean, std, generator=g).to(TYPES[ty])


# ---------------------------------------------------------------- balance loss
def _tokens_of_a_round(E, k):
    """Tokens that eight blocks an SM (1184 at most) take in one round: more than any form of the kernel holds."""
    lanes = 1
    while lanes < 32 and (lanes * 16 < E or lanes < k):
        lanes *= 2
    return min(8 * _sms(), 1184) * 8 * (32 // lanes)


# E, k, type of the scores, row padding, rounds: rings of 16-byte (bf16, f32) and 8-byte copies, and none; a token to a lane up to a
# token to a warp with 32 elements a lane.  `rounds` full grids of eight blocks an SM (no form holds so many: every one goes round more
# often) are more than the deepest ring's six slots for the narrow forms and more than the two or three slots of the wide ones.
ROUNDS = [(256, 8, "bf16", 0, 3), (256, 8, "f32", 0, 3), (333, 5, "bf16", 0, 2), (333, 5, "f32", 0, 2), (60, 6, "bf16", 0, 7),
          (60, 6, "f32", 0, 4), (64, 8, "f32", 4, 4), (64, 8, "bf16", 3, 3), (128, 8, "bf16", 0, 5), (8, 2, "bf16", 0, 7), (16, 1, "f32", 0, 5),
          (7, 3, "f32", 0, 3), (1000, 4, "bf16", 0, 3), (1024, 32, "f32", 0, 2)]


def _balance_reference(s, i, mask, dg, norm, counts, n, ca, cz):
    """Losses, gradient and the gradient's bound in float64, on the GPU; written from the formulas."""
    x, ix = s.double(), i.long()
    T, E = x.shape
    live = torch.ones(T, dtype=torch.bool, device=x.device) if mask is None else mask != 0
    n = max(n, 1)
    f = counts.double() * (E / max(int(counts.sum()), 1))
    lse = torch.logsumexp(x, 1)
    p = torch.exp(x - lse[:, None])
    a = p @ f
    balance, z = a[live].sum() / n, lse[live].square().sum() / n
    d = ca / n * p * (f - a[:, None]) + 2 * cz / n * lse[:, None] * p
    top = x.abs().max(1, keepdim=True).values
    bound = 1 / n * p * (ca * (f + a[:, None]) + 2 * cz * lse.abs()[:, None]) * (2.0 ** -19 + 2.0 ** -23 * (x.abs() + top))
    if dg is not None:
        kept, g = x.gather(1, ix), dg.double()
        if norm == "softmax":
            q = torch.softmax(kept, 1)
            back = q * (g - (q * g).sum(1, keepdim=True))
            each = q * (g.abs() + (q * g.abs()).sum(1, keepdim=True))
        else:
            q = torch.sigmoid(kept)
            back = q * torch.sigmoid(-kept) * g
            each = q * g.abs()
        d = d.scatter_add(1, ix, back)
        bound = bound + torch.zeros_like(x).scatter_add(1, ix, each) * (2.0 ** -19 + 2.0 ** -22 * top)
    d = d * live[:, None]
    return torch.stack([ca * balance + cz * z, balance, z]), d, bound


@pytest.mark.parametrize("E,k,ty,pad,rounds", ROUNDS)
@pytest.mark.parametrize("gates", ["none", "softmax", "sigmoid"])
def test_balance_loss_goes_round(E, k, ty, pad, rounds, gates):
    from paper_2603_06626_b200 import binding as B
    T = rounds * _tokens_of_a_round(E, k) + 77
    s = _normal((T, E + pad), 2.0, ty=ty, seed=E + T)[:, :E]
    i = torch.cat([c.topk(k, dim=1).indices for c in s.float().split(65536)]).to(torch.int32)
    if k > 1:
        i[1::3, k - 1] = i[1::3, 0]                       # an expert twice in a token: in every round
    g = torch.Generator(device="cuda:0").manual_seed(T)
    mask = (torch.rand(T, generator=g, device="cuda:0") < 0.8).to(torch.uint8) if gates != "sigmoid" else None
    dg = None if gates == "none" else _normal((T, k), seed=5)
    ca, cz = 0.37, 0.021
    counts, n = B.expert_counts(i, E, mask=mask)
    live = torch.ones(T, dtype=torch.bool, device="cuda:0") if mask is None else mask != 0
    assert int(n) == int(live.sum()) and torch.equal(counts.long(), torch.bincount(i[live].reshape(-1).long(), minlength=E))
    nm = B.NORM_SIGMOID if gates == "sigmoid" else B.NORM_SOFTMAX
    loss, d = B.balance_loss(s, i, counts, n, mask=mask, balance_coef=ca, z_coef=cz, dgates=dg, norm=nm)
    again = B.balance_loss(s, i, counts, n, mask=mask, balance_coef=ca, z_coef=cz, dgates=dg, norm=nm)
    alone, _ = B.balance_loss(s, i, counts, n, mask=mask, balance_coef=ca, z_coef=cz, norm=nm, want_grad=False)
    B.check_status()
    assert torch.equal(loss, again[0]) and torch.equal(d, again[1])
    want, dr, bound = _balance_reference(s, i, mask, dg, gates, counts, int(n), ca, cz)
    assert np.allclose(f64(loss), f64(want), rtol=2.0 ** -18, atol=1e-30) and np.allclose(f64(alone), f64(want), rtol=2.0 ** -18, atol=1e-30)
    err = (d.double() - dr).abs()
    lim = bound + (2.0 ** -8 * dr.abs() if ty == "bf16" else 0) + 1e-30
    assert (err <= lim)[live].all(), float((err / lim)[live].max())
    assert (d[~live] == 0).all()


def test_the_reference_of_the_rounds_is_the_oracle():
    s, k = _normal((300, 24), 2.0, seed=1), 3
    i = s.topk(k, dim=1).indices.to(torch.int32)
    i[::5, 2] = i[::5, 0]
    mask, dg = (torch.arange(300, device="cuda:0") % 4 != 1).to(torch.uint8), _normal((300, k), seed=2)
    cr, nr = orc.expert_counts(i.cpu().numpy(), 24, mask.cpu().numpy())
    for norm in ("softmax", "sigmoid"):
        want, dr, _ = _balance_reference(s, i, mask, dg, norm, torch.from_numpy(cr).to("cuda:0"), nr, 0.37, 0.021)
        assert np.allclose(f64(want), orc.balance_loss(f64(s), cr, nr, 0.37, 0.021, mask.cpu().numpy()), rtol=1e-12)
        ref = orc.balance_gradient(f64(s), cr, nr, 0.37, 0.021, mask.cpu().numpy(), i.cpu().numpy(), f64(dg), norm)
        assert np.abs(f64(dr) - ref).max() < 1e-12


# ---------------------------------------------------------------- counts
# One cluster of eight blocks counts up to 2^19 ids, in trips of 131072 8-bit or 32768 32-bit ones; above that blocks on all SMs add
# to zeroed outputs, two blocks an SM, coming round from 2 * 148 * 16384 = 4.8 M 8-bit (1.2 M 32-bit) ids on.
@pytest.mark.parametrize("ty", [torch.uint8, torch.int32])
@pytest.mark.parametrize("T,k,E", [(1 << 16, 8, 64), ((1 << 16) + 1, 8, 64), (174763, 3, 60), (74899, 7, 256), (300001, 7, 250), (1048575, 8, 256),
                                   (1400003, 6, 9)])
@pytest.mark.parametrize("masked", [False, True])
def test_counts_of_many_ids(ty, T, k, E, masked):
    from paper_2603_06626_b200 import binding as B
    g = torch.Generator(device="cuda:0").manual_seed(T + k)
    i = torch.randint(0, E, (T, k), generator=g, device="cuda:0").to(ty)
    mask = (torch.rand(T, generator=g, device="cuda:0") < 0.7).to(torch.uint8) if masked else None
    live = torch.ones(T, dtype=torch.bool, device="cuda:0") if mask is None else mask != 0
    status = torch.zeros(1, dtype=torch.int32, device="cuda:0")
    counts, n = B.expert_counts(i, E, mask=mask, status=status)
    want = torch.bincount(i[live].reshape(-1).long(), minlength=E)
    assert torch.equal(counts.long(), want) and int(n) == int(live.sum()) and int(status) == 0
    if E < 256 or ty == torch.int32:
        t = T - 2                                         # out of range near the end: left out and reported; of a masked token: neither
        if masked:
            mask[t], live[t] = 0, False
            i[t] = E
            counts, n = B.expert_counts(i, E, mask=mask, status=status)
            assert torch.equal(counts.long(), torch.bincount(i[live].reshape(-1).long(), minlength=E)) and int(status) == 0
            mask[t] = 1
        else:
            i[t, 0] = E
        gone = i[t].long()
        live[t] = False
        counts, n = B.expert_counts(i, E, mask=mask, status=status)
        rest = torch.bincount(i[live].reshape(-1).long(), minlength=E) + torch.bincount(gone[gone < E], minlength=E)
        assert torch.equal(counts.long(), rest) and int(n) == int(live.sum()) + 1 and int(status) == 1


# ---------------------------------------------------------------- layer norm, backward
def _norm_tokens(d, rounds):
    """Rows that make every resident block of the backward pass go round `rounds` times and a bit: 16 elements a thread, 512 threads an SM
    (1024 for the widest rows)."""
    lanes = 8
    while lanes * 16 < d:
        lanes *= 2
    return rounds * _sms() * max(512 // lanes, 1) + 3


# width, activations, weights, row padding, rounds.  The ring has 4 slots (bf16) or 3 (f32), 3 or 1 in rows of 1024 threads: nine rounds
# refill and wrap it; from width 1024 on eight rounds join neighbouring blocks' columns in clusters of two.  Odd widths: no ring.
NORM = [(64, "bf16", "bf16", 0, 9), (128, "f32", "bf16", 0, 9), (256, "bf16", "f32", 8, 9), (512, "bf16", "bf16", 0, 9), (1024, "f32", "f32", 0, 9),
        (1000, "bf16", "bf16", 0, 9), (2048, "bf16", "f32", 0, 9), (2048, "f32", "f32", 4, 9), (4096, "bf16", "bf16", 0, 9), (8192, "f32", "bf16", 0, 9),
        (8192, "bf16", "bf16", 0, 9), (16384, "bf16", "f32", 0, 9), (16384, "f32", "bf16", 0, 9), (2047, "bf16", "bf16", 0, 9),
        (2046, "f32", "f32", 0, 9), (8191, "f32", "f32", 1, 9), (16383, "bf16", "bf16", 0, 9), (100, "bf16", "bf16", 2, 9)]


@pytest.mark.parametrize("d,ty,wt,pad,rounds", NORM)
def test_norm_backward_goes_round(d, ty, wt, pad, rounds):
    from paper_2603_06626_b200 import binding as B
    T = _norm_tokens(d, rounds)
    x, dy = _normal((T, d + pad), 1.5, 0.3, ty, seed=d)[:, :d], _normal((T, d), ty=ty, seed=d + 1)
    w = _normal((d,), 0.3, 1.0, wt, seed=2)
    _, mean, rstd = B.layer_norm(x, w, None)
    dx, dw, db = B.layer_norm_backward(dy, x, w, mean, rstd)
    again = B.layer_norm_backward(dy, x, w, mean, rstd)
    assert all(torch.equal(p, q) for p, q in zip((dx, dw, db), again))
    dw_sum, db_sum, dw_mag, db_mag = (torch.zeros(d, dtype=torch.float64, device="cuda:0") for _ in range(4))
    for r in range(0, T, 4096):                            # in pieces: whole matrices in 64 bits would take some GB
        s = slice(r, r + 4096)
        g, xr, wr, mr, rr = dy[s].double(), x[s].double(), w.double(), mean[s].double()[:, None], rstd[s].double()[:, None]
        h, gw = (xr - mr) * rr, g * wr
        dxr = rr * (gw - gw.mean(1, keepdim=True) - h * (gw * h).mean(1, keepdim=True))
        ha = (xr.abs() + mr.abs()) * rr
        mags = rr * (gw.abs() + gw.abs().mean(1, keepdim=True) + ha * (gw.abs() * ha).mean(1, keepdim=True))
        assert ((dx[s].double() - dxr).abs() <= (2.0 ** -8 * dxr.abs() if ty == "bf16" else 0) + 128 * U * mags + 1e-30).all()
        dw_sum += (g * h).sum(0)
        db_sum += g.sum(0)
        dw_mag += (g.abs() * ha).sum(0)
        db_mag += g.abs().sum(0)
    assert ((dw.double() - dw_sum).abs() <= (T + 64) * U * dw_mag + 1e-30).all()
    assert ((db.double() - db_sum).abs() <= (T + 64) * U * db_mag + 1e-30).all()
    # the worst case over T rows is wide: sums of T random signs lose far less
    assert float((dw.double() - dw_sum).norm() / dw_sum.norm()) < 1e-4 and float((db.double() - db_sum).norm() / db_sum.norm()) < 1e-4


# ---------------------------------------------------------------- linear layer
KINDS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}


def _act(z, kind):
    if kind == "relu":
        return torch.relu(z)
    if kind == "silu":
        return z * torch.sigmoid(z)
    if kind == "gelu":
        return 0.5 * z * (1 + torch.tanh((2 / np.pi) ** 0.5 * (z + 0.044715 * z ** 3)))
    return z


# More than two 256 x 256 tiles for each of the SMs' pairs (74: 256 tiles are three and a half rounds), so that both accumulators
# come round and a residual is fetched while the tile before is still being written; ragged in every dimension.
@pytest.mark.parametrize("kind,bias,residual,pre", [("silu", True, True, True), ("gelu", True, True, False), ("none", False, True, False),
                                                    ("relu", False, False, True)])
def test_linear_forward_takes_several_tiles_a_pair(kind, bias, residual, pre):
    from paper_2603_06626_b200 import binding as B
    T, K, N = 3 * 256 * (_sms() // 2) // 8 + 256 + 13, 200, 8 * 256 + 72
    x, W = _normal((T, K), ty="bf16", seed=1), _normal((N, K), K ** -0.5, ty="bf16", seed=2)
    b = _normal((N,), ty="bf16", seed=3) if bias else None
    r = _normal((T, N), ty="bf16", seed=4) if residual else None
    y, z = B.linear(x, W, bias=b, act=KINDS[kind], residual=r, save_pre=pre)
    y2, _ = B.linear(x, W, bias=b, act=KINDS[kind], residual=r, save_pre=pre)
    B.check_status()
    assert torch.equal(y, y2)
    zr = x.double() @ W.double().t() + (0 if b is None else b.double())
    off = (K / 16 + 32) * 2 * U * (x.double().abs() @ W.double().abs().t() + (0 if b is None else b.double().abs()))
    yr = _act(zr, kind) + (0 if r is None else r.double())
    bound = 1.2 * off + 2.0 ** -18 * zr.abs() + 2.0 ** -8 * yr.abs() + (0 if r is None else 8 * U * r.double().abs())
    assert ((y.double() - yr).abs() <= bound).all()
    if pre:
        assert ((z.double() - zr).abs() <= off + 2.0 ** -8 * zr.abs()).all()


# The pass over dy and z: a thread takes four rows a trip, about six blocks an SM over all columns.  6000 x 1408: six column blocks, 148
# row blocks of 8 rows each: 6000 / (148 * 8 * 4) = two trips, the second one short; 100003 x 136: one column block, 888 row blocks, four.
@pytest.mark.parametrize("T,K,N,kind", [(6000, 264, 1408, "gelu"), (6001, 136, 1400, "silu"), (100003, 64, 136, "relu"), (100000, 72, 136, "none")])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_linear_backward_goes_round(T, K, N, kind, dtype):
    from paper_2603_06626_b200 import binding as B
    x, W, dy = _normal((T, K), ty="bf16", seed=1), _normal((N, K), K ** -0.5, ty="bf16", seed=2), _normal((T, N), ty="bf16", seed=3)
    z = None if kind == "none" else _normal((T, N), 2.0, ty="bf16", seed=4)
    args = dict(pre=z, act=KINDS[kind], want_bias=True, dW_dtype=dtype)
    dx, dW, db = B.linear_backward(dy, x, W, **args)
    assert all(torch.equal(p, q) for p, q in zip((dx, dW, db), B.linear_backward(dy, x, W, **args)))
    B.check_status()
    zz = torch.zeros((), dtype=torch.float64, device="cuda:0") if z is None else z.double().requires_grad_()
    g = dy.double()
    if z is not None:
        g = torch.autograd.grad(_act(zz, kind), zz, g)[0]
    dxr, dWr, dbr = g @ W.double(), g.t() @ x.double(), g.sum(0)
    r = 0.0 if kind == "none" else 2.0 ** -8 + 2.0 ** -17
    assert ((dx.double() - dxr).abs() <= ((N / 16 + 32) * 2 * U + r) * (g.abs() @ W.double().abs()) + 2.0 ** -8 * dxr.abs()).all()
    last = 2.0 ** -8 * dWr.abs() if dtype == torch.bfloat16 else 0
    assert ((dW.double() - dWr).abs() <= ((T / 16 + 32) * 2 * U + r) * (g.abs().t() @ x.double().abs()) + last).all()
    assert rel_frobenius(f64(dx), f64(dxr)) < 5e-3 and rel_frobenius(f64(dW), f64(dWr)) < 5e-3
    assert ((db.double() - dbr).abs() <= ((T + 64) * U + 2.0 ** -17) * dy.double().abs().sum(0) * 1.2 + 1e-30).all()
