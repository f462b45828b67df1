"""What the operators around the expert layer refuse: through the C ABI (codes, before anything is launched) and in the binding."""
import ctypes

import pytest
import torch

from paper_2603_06626_b200 import binding as B

OK, INVALID, MISALIGNED, UNSUPPORTED = 0, -1, -2, -3
A = 1 << 20           # stands for a 256-byte-aligned device address: every call below returns before it is used


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


def test_layer_norm(lib):
    def fwd(x=A, ldx=64, w=A, b=A, rows=4, d=64, dt=0, wt=0, eps=1e-5, y=A, mean=A, rstd=A):
        return lib.grouter_layernorm_fwd(x, ldx, w, b, rows, d, dt, wt, eps, y, mean, rstd, None)
    assert fwd(x=None) == fwd(w=None) == fwd(y=None) == fwd(d=0) == fwd(rows=-1) == fwd(ldx=63) == fwd(dt=2) == fwd(wt=-1) == INVALID
    assert fwd(eps=-1.0) == fwd(eps=float("nan")) == INVALID
    assert fwd(d=16385, ldx=16385) == fwd(rows=2 ** 31 - 1) == UNSUPPORTED
    assert fwd(x=A + 1) == fwd(y=A + 1) == fwd(mean=A + 2) == fwd(w=A + 2, wt=1) == MISALIGNED
    assert fwd(rows=0, x=None, y=None) == OK

    def bwd(dy=A, x=A, ldx=64, w=A, mean=A, rstd=A, rows=4, d=64, dt=0, wt=0, dx=A, dw=A, db=A, ws=A):
        return lib.grouter_layernorm_bwd(dy, x, ldx, w, mean, rstd, rows, d, dt, wt, dx, dw, db, ws, None)
    for name in ("dy", "x", "w", "mean", "rstd", "dx", "dw", "ws"):
        assert bwd(**{name: None}) == INVALID, name
    assert bwd(dw=A + 1) == bwd(ws=A + 4) == bwd(dx=A + 1) == MISALIGNED
    assert lib.grouter_layernorm_bwd_workspace_bytes(4, 16385) == 0


def test_linear(lib):
    def fwd(x=A, W=A, b=None, r=None, T=4, K=64, N=64, act=0, y=A, pre=None, status=A):
        return lib.grouter_linear_fwd(x, W, b, r, T, K, N, act, y, pre, status, None)
    assert fwd(x=None) == fwd(W=None) == fwd(y=None) == fwd(status=None) == fwd(T=-1) == fwd(K=0) == fwd(act=4) == fwd(act=-1) == INVALID
    assert fwd(K=60) == fwd(N=4) == UNSUPPORTED
    assert fwd(x=A + 8) == fwd(b=A + 2) == fwd(r=A + 2) == fwd(pre=A + 2) == MISALIGNED
    assert fwd(T=0, x=None, y=None) == OK

    def bwd(dy=A, x=A, W=A, pre=A, T=4, K=64, N=64, act=2, dx=A, dW=A, dt=0, db=A, ws=A, status=A):
        return lib.grouter_linear_bwd(dy, x, W, pre, T, K, N, act, dx, dW, dt, db, ws, status, None)
    for name in ("dy", "x", "W", "pre", "ws", "status"):
        assert bwd(**{name: None}) == INVALID, name
    assert bwd(dx=None, dW=None, db=None) == bwd(dt=2) == INVALID
    assert bwd(K=12) == UNSUPPORTED and bwd(ws=A + 16) == bwd(dx=A + 2) == MISALIGNED
    assert lib.grouter_linear_bwd_workspace_bytes(4, 60, 64, 0) == 0


def test_counts_and_balance(lib):
    def counts(idx=A, dt=0, mask=None, T=4, k=2, E=8, c=A, n=A, status=None):
        return lib.grouter_expert_counts(idx, dt, mask, T, k, E, c, n, status, None)
    assert counts(idx=None) == counts(c=None) == counts(n=None) == counts(dt=2) == counts(k=0) == counts(E=0) == counts(T=-1) == INVALID
    assert counts(E=257) == counts(E=1025, dt=1) == counts(k=33) == counts(T=2 ** 30, k=4) == UNSUPPORTED
    assert counts(idx=A + 1) == counts(c=A + 2) == MISALIGNED

    def bal(x=A, ld=8, dt=0, idx=A, it=0, mask=None, c=A, n=A, dg=A, norm=0, T=4, E=8, k=2, dl=None, loss=A, d=A, ws=A, status=None):
        return lib.grouter_balance_loss(x, ld, dt, idx, it, mask, c, n, dg, norm, T, E, k, 0.1, 0.1, dl, loss, d, ws, status, None)
    assert bal(x=None) == bal(c=None) == bal(n=None) == bal(idx=None) == bal(loss=None, d=None) == bal(ws=None, T=100000) == INVALID
    assert bal(d=None) == INVALID                       # a gradient of the gates has nowhere to go
    assert bal(ld=7) == bal(norm=2) == bal(dt=3) == bal(it=2) == bal(k=0) == INVALID
    assert bal(E=257, ld=257) == bal(E=1025, ld=1025, it=1) == bal(k=33) == UNSUPPORTED
    assert bal(x=A + 1) == bal(d=A + 1) == bal(loss=A + 2) == bal(idx=A + 2, it=1) == MISALIGNED


def test_adamw(lib):
    def layout(p=A, g=A, n=100, wd=0.1, pt=0, gt=1, count=1):
        t = (B.AdamwTensor * 1)(B.AdamwTensor(p, g, n, wd, pt, gt))
        out = B.AdamwLayout()
        return lib.grouter_adamw_layout_host(t, count, ctypes.byref(out), None), out
    assert layout(p=None)[0] == layout(g=None)[0] == layout(n=-1)[0] == layout(pt=2)[0] == layout(gt=-1)[0] == layout(count=0)[0] == INVALID
    assert layout(wd=float("inf"))[0] == INVALID and layout(p=A + 1)[0] == layout(g=A + 2)[0] == MISALIGNED
    code, lay = layout()
    assert code == OK and lay.state_elements == 128 and lay.n_chunks == 1 and lay.needs_master == 1 and lay.table_bytes % 8 == 0
    code, empty = layout(p=None, g=None, n=0)
    assert code == OK and empty.state_elements == 0 and empty.n_chunks == 0

    def step(lay=lay, table=A, bits=32, master=A, m=A, v=A, mx=A, vx=A, lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, t=1, scale=None):
        return lib.grouter_adamw_step(ctypes.byref(lay), table, bits, master, m, v, mx, vx, lr, b1, b2, eps, t, scale, None)
    assert step(table=None) == step(m=None) == step(v=None) == step(master=None) == step(bits=16) == step(t=0) == INVALID
    assert step(bits=8, mx=None) == step(b1=1.0) == step(b2=-0.1) == step(eps=-1.0) == step(lr=float("nan")) == INVALID
    assert step(m=A + 4) == step(table=A + 8) == step(scale=A + 2) == MISALIGNED
    assert step(lay=empty, table=None, m=None, v=None) == OK
    assert lib.grouter_adamw_moments(A, A, A, A, 33, A, A, None) == INVALID


def _raises(kind, call):
    with pytest.raises(kind):
        call()


def test_the_binding_checks_shapes_types_and_layouts():
    f, b16 = torch.zeros(4, 64), torch.zeros(4, 64, dtype=torch.bfloat16)
    w = torch.ones(64)
    _raises(ValueError, lambda: B.layer_norm(f[0], w))
    _raises(ValueError, lambda: B.layer_norm(f.t(), torch.ones(4)))
    _raises(ValueError, lambda: B.layer_norm(f, w[:32]))
    _raises(TypeError, lambda: B.layer_norm(f, w, w.bfloat16()))
    _raises(TypeError, lambda: B.layer_norm(f.half(), w))
    _raises(ValueError, lambda: B.layer_norm(torch.zeros(64).as_strided((4, 8), (4, 1)), torch.ones(8)))       # rows that overlap
    _raises(TypeError, lambda: B.layer_norm_backward(b16, f, w, torch.zeros(4), torch.zeros(4)))
    _raises(ValueError, lambda: B.layer_norm_backward(f, f, w, torch.zeros(3), torch.zeros(4)))
    W = torch.zeros(8, 64, dtype=torch.bfloat16)
    _raises(TypeError, lambda: B.linear(f, W))
    _raises(ValueError, lambda: B.linear(b16, W[:, :32]))
    _raises(ValueError, lambda: B.linear(b16, W, bias=torch.zeros(9, dtype=torch.bfloat16)))
    _raises(ValueError, lambda: B.linear(b16, W, residual=b16))
    _raises(ValueError, lambda: B.linear(torch.zeros(64, 4, dtype=torch.bfloat16).t(), W))
    dy = torch.zeros(4, 8, dtype=torch.bfloat16)
    _raises(ValueError, lambda: B.linear_backward(dy, b16, W, act=B.ACT_SILU))
    _raises(TypeError, lambda: B.linear_backward(dy, b16, W, dW_dtype=torch.float16))
    idx = torch.zeros(4, 2, dtype=torch.uint8)
    _raises(TypeError, lambda: B.expert_counts(idx.long(), 8))
    _raises(ValueError, lambda: B.expert_counts(idx, 8, mask=torch.ones(3, dtype=torch.uint8)))
    _raises(TypeError, lambda: B.expert_counts(idx, 8, mask=torch.ones(4)))
    c, n = torch.zeros(64, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    _raises(ValueError, lambda: B.balance_loss(f, None, c, n, dgates=torch.zeros(4, 2)))
    _raises(ValueError, lambda: B.balance_loss(f, idx, c[:8], n))
    _raises(TypeError, lambda: B.balance_loss(f, idx, c.float(), n))
    _raises(ValueError, lambda: B.balance_loss(f, idx, c, n, dgates=torch.zeros(4, 3)))
    p = torch.zeros(10)
    _raises(ValueError, lambda: B.AdamW([p], []))
    _raises(ValueError, lambda: B.AdamW([p], [p], state_bits=16))
    _raises(ValueError, lambda: B.AdamW([p], [p[:5]]))
    _raises(TypeError, lambda: B.AdamW([p.half()], [p]))
    _raises(ValueError, lambda: B.AdamW([p], [p], weight_decay=[0.1, 0.2]))
    _raises(ValueError, lambda: B.AdamW([p], [p], state=dict(m=torch.zeros(10), v=torch.zeros(32))))
    _raises(ValueError, lambda: B.AdamW([p], [p], state=dict(master=torch.zeros(32))))
