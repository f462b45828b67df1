"""What the operators of the dense gated branch refuse: through the C ABI (codes, before anything is launched) and in the binding."""
import pytest
import torch

from paper_2603_06626_b200 import binding as B

OK, INVALID, MISALIGNED, UNSUPPORTED = 0, -1, -2, -3
A = 1 << 20           # stands for a 256-byte-aligned device address: every call below returns before it is used
MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


def test_rms_norm(lib):
    def fwd(x=A, ldx=64, r=A, ldr=64, w=A, rows=4, d=64, dt=0, wt=0, eps=1e-5, h=A, y=A, s=None, rstd=A):
        return lib.grouter_rmsnorm_fwd(x, ldx, r, ldr, w, rows, d, dt, wt, eps, h, y, s, rstd, None)
    assert fwd(x=None) == fwd(w=None) == fwd(y=None) == fwd(h=None) == fwd(d=0) == fwd(rows=-1) == fwd(ldx=63) == fwd(ldr=63) == INVALID
    assert fwd(dt=2) == fwd(wt=-1) == fwd(eps=-1.0) == fwd(eps=float("nan")) == INVALID
    assert fwd(d=16385, ldx=16385, ldr=16385) == fwd(rows=MOST) == UNSUPPORTED
    assert fwd(x=A + 1) == fwd(y=A + 1) == fwd(r=A + 1) == fwd(h=A + 1) == fwd(rstd=A + 2) == fwd(w=A + 2, wt=1) == MISALIGNED
    assert fwd(s=A, d=72, ldx=72, ldr=72) == UNSUPPORTED
    assert fwd(s=A + 8) == fwd(s=A, x=A + 8) == fwd(s=A, y=A + 8) == fwd(s=A, w=A + 8) == fwd(s=A, ldx=68) == fwd(s=A, ldr=68) == MISALIGNED
    assert fwd(rows=0, x=None, y=None, r=None, h=None) == OK

    def bwd(dy=A, h=A, ldh=64, dh=A, w=A, rstd=A, rows=4, d=64, dt=0, wt=0, dx=A, dw=A, ws=A):
        return lib.grouter_rmsnorm_bwd(dy, h, ldh, dh, w, rstd, rows, d, dt, wt, dx, dw, ws, None)
    for name in ("dy", "h", "w", "rstd", "dx", "dw", "ws"):
        assert bwd(**{name: None}) == INVALID, name
    assert bwd(ldh=60) == bwd(dt=3) == INVALID and bwd(d=16385, ldh=16385) == UNSUPPORTED
    assert bwd(dw=A + 1) == bwd(ws=A + 4) == bwd(dx=A + 1) == bwd(dh=A + 1) == MISALIGNED
    assert lib.grouter_rmsnorm_bwd_workspace_bytes(4, 16385) == 0


def test_eight_bits(lib):
    assert [lib.grouter_fp8_pitch(c) for c in (0, 1, 16, 17)] == [0, 16, 16, 32]
    assert lib.grouter_fp8_scale_bytes(1, 1) == 512 and lib.grouter_fp8_scale_bytes(129, 513) == 2048 and lib.grouter_fp8_scale_bytes(0, 9) == 0

    def quant(x=A, ld=64, dt=0, rows=4, cols=64, square=0, q=A, s=A, qt=A, st=A):
        return lib.grouter_quantize_fp8(x, ld, dt, rows, cols, square, q, s, qt, st, None)
    assert quant(x=None) == quant(ld=63) == quant(dt=2) == quant(rows=-1) == quant(q=None, qt=None) == quant(s=None) == quant(st=None) == INVALID
    assert quant(x=A + 1) == quant(q=A + 8) == quant(s=A + 4) == quant(qt=A + 8) == quant(st=A + 4) == MISALIGNED
    assert quant(rows=MOST) == UNSUPPORTED and quant(rows=0, x=None, q=None, qt=None) == OK

    def back(q=A, s=A, rows=4, cols=64, ld=64, dt=0, y=A):
        return lib.grouter_dequantize_fp8(q, s, rows, cols, ld, dt, y, None)
    assert back(q=None) == back(s=None) == back(y=None) == back(ld=63) == back(dt=2) == INVALID
    assert back(q=A + 8) == back(y=A + 1) == MISALIGNED and back(rows=0, q=None, s=None, y=None) == OK

    def fwd(x=A, xs=A, ld=0, W=A, Ws=A, b=A, r=A, T=4, K=64, N=64, y=A, ws=None, status=A):
        return lib.grouter_linear_fp8_fwd(x, xs, ld, W, Ws, b, r, T, K, N, y, ws, status, None)
    for name in ("x", "W", "Ws", "y", "status"):
        assert fwd(**{name: None}) == INVALID, name
    assert fwd(xs=None, ld=64) == fwd(xs=None, ld=63, ws=A) == INVALID and fwd(xs=None, ld=64, ws=A + 16) == fwd(xs=None, ld=64, ws=A, x=A + 1) == MISALIGNED
    assert lib.grouter_linear_fp8_fwd_workspace_bytes(4, 64) >= 4 * 64 + 512 and lib.grouter_linear_fp8_fwd_workspace_bytes(-1, 64) == 0
    assert fwd(T=-1) == fwd(K=0) == fwd(N=0) == INVALID and fwd(N=12) == fwd(T=MOST) == UNSUPPORTED
    assert fwd(x=A + 8) == fwd(xs=A + 8) == fwd(b=A + 8) == fwd(r=A + 8) == fwd(y=A + 8) == MISALIGNED
    assert fwd(T=0, x=None, xs=None, y=None) == OK

    def bwd(dy=A, xt=A, xs=A, Wt=A, Ws=A, T=4, K=64, N=64, dx=A, dW=A, dt=0, db=A, ws=A, status=A):
        return lib.grouter_linear_fp8_bwd(dy, xt, xs, Wt, Ws, T, K, N, dx, dW, dt, db, ws, status, None)
    for name in ("dy", "xt", "xs", "Wt", "Ws", "ws", "status"):
        assert bwd(**{name: None}) == INVALID, name
    assert bwd(dx=None, dW=None, db=None) == bwd(dt=2) == INVALID and bwd(K=12) == bwd(N=12) == UNSUPPORTED
    assert bwd(ws=A + 16) == bwd(dx=A + 8) == bwd(dW=A + 8) == MISALIGNED
    assert lib.grouter_linear_fp8_bwd_workspace_bytes(4, 64, 12) == 0


def test_gated(lib):
    def fwd(x=A, Wgu=A, Wd=A, r=A, T=4, d=64, H=64, act=2, h=A, y=A, pre=A, status=A):
        return lib.grouter_gated_ffn_fwd(x, Wgu, Wd, r, T, d, H, act, h, y, pre, status, None)
    for name in ("x", "Wgu", "Wd", "h", "y", "status"):
        assert fwd(**{name: None}) == INVALID, name
    assert fwd(T=-1) == fwd(d=0) == fwd(H=0) == fwd(act=4) == fwd(act=-1) == INVALID
    assert fwd(d=60) == fwd(H=12) == fwd(H=2 ** 30) == UNSUPPORTED
    assert fwd(x=A + 8) == fwd(pre=A + 8) == fwd(h=A + 8) == fwd(r=A + 8) == fwd(status=A + 2) == MISALIGNED
    assert fwd(T=0, x=None, h=None, y=None) == OK

    def bwd(dy=A, x=A, Wgu=A, Wd=A, pre=A, T=4, d=64, H=64, act=2, dx=A, dgu=A, dd=A, dt=0, ws=A, status=A):
        return lib.grouter_gated_ffn_bwd(dy, x, Wgu, Wd, pre, T, d, H, act, dx, dgu, dd, dt, ws, status, None)
    for name in ("dy", "x", "Wgu", "Wd", "pre", "ws", "status"):
        assert bwd(**{name: None}) == INVALID, name
    assert bwd(dx=None, dgu=None, dd=None) == bwd(dt=2) == INVALID and bwd(d=12) == UNSUPPORTED
    assert bwd(ws=A + 16) == bwd(dd=A + 8) == MISALIGNED
    assert lib.grouter_gated_ffn_bwd_workspace_bytes(4, 64, 12) == 0

    def eight(x=A, xs=A, ld=0, g=A, gs=A, u=A, us=A, dn=A, ds=A, r=A, T=4, d=64, H=64, act=2, y=A, ws=A, status=A):
        return lib.grouter_gated_ffn_fp8_fwd(x, xs, ld, g, gs, u, us, dn, ds, r, T, d, H, act, y, ws, status, None)
    for name in ("x", "g", "gs", "u", "us", "dn", "ds", "y", "ws", "status"):
        assert eight(**{name: None}) == INVALID, name
    assert eight(act=9) == eight(xs=None, ld=63) == INVALID and eight(d=12) == UNSUPPORTED
    assert eight(ws=A + 16) == eight(y=A + 8) == eight(us=A + 1) == eight(xs=A + 8) == eight(xs=None, ld=64, x=A + 1) == MISALIGNED
    assert eight(T=0, x=None, xs=None, ws=None, y=None) == OK
    assert lib.grouter_gated_ffn_fp8_fwd_workspace_bytes(4, 64, 128) >= 4 * 192 + 1024


def _raises(kind, call):
    with pytest.raises(kind):
        call()


def _blocks(rows, columns, **kw):
    q = B.Fp8Blocks.empty(rows, columns, "cpu")
    for name, v in kw.items():
        setattr(q, name, v)
    return q


def test_the_binding_checks_the_norms_arguments():
    f, b16, w = torch.zeros(4, 64), torch.zeros(4, 64, dtype=torch.bfloat16), torch.ones(64)
    _raises(ValueError, lambda: B.rms_norm(f[0], w))
    _raises(ValueError, lambda: B.rms_norm(f, w[:32]))
    _raises(ValueError, lambda: B.rms_norm(f, w, residual=f[:2]))
    _raises(ValueError, lambda: B.rms_norm(f, w, residual=b16))
    _raises(ValueError, lambda: B.rms_norm(f, w, residual=f.t()))
    _raises(TypeError, lambda: B.rms_norm(f.half(), w))
    _raises(TypeError, lambda: B.rms_norm(f, w.half()))
    _raises(ValueError, lambda: B.rms_norm(f, w))                                    # not on a GPU
    _raises(TypeError, lambda: B.rms_norm_backward(b16, f, w, torch.zeros(4)))
    _raises(TypeError, lambda: B.rms_norm_backward(f, f, w, torch.zeros(4), dh=b16))
    _raises(ValueError, lambda: B.rms_norm_backward(f, f, w, torch.zeros(3)))
    _raises(ValueError, lambda: B.rms_norm_backward(f, f, w, torch.zeros(4), dw=torch.zeros(63)))


def test_the_binding_checks_matrices_in_8_bits():
    b16, W = torch.zeros(4, 64, dtype=torch.bfloat16), _blocks(8, 64)
    _raises(TypeError, lambda: B.quantize_fp8(b16.half()))
    _raises(ValueError, lambda: B.quantize_fp8(b16[0]))
    _raises(ValueError, lambda: B.quantize_fp8(b16, rows=False))
    _raises(TypeError, lambda: B.dequantize_fp8(b16))
    _raises(ValueError, lambda: B.dequantize_fp8(_blocks(8, 64, cols=40)))
    _raises(TypeError, lambda: B.linear_fp8(b16, b16))
    _raises(ValueError, lambda: B.linear_fp8(b16[:, :32], W))
    _raises(TypeError, lambda: B.linear_fp8([1.0], W))
    _raises(ValueError, lambda: B.linear_fp8(_blocks(4, 72), W))
    _raises(ValueError, lambda: B.linear_fp8(_blocks(4, 64, scales=torch.zeros(2, 1, 32, 4, 4, dtype=torch.uint8)), W))
    _raises(TypeError, lambda: B.linear_fp8(_blocks(4, 64, codes=torch.zeros(4, 64, dtype=torch.uint8)), W))
    _raises(ValueError, lambda: B.linear_fp8(_blocks(4, 64, codes=torch.zeros(64, 4).to(torch.float8_e4m3fn).t()), W))
    _raises(ValueError, lambda: B.linear_fp8(b16, W, bias=torch.zeros(9, dtype=torch.bfloat16)))
    _raises(TypeError, lambda: B.linear_fp8(b16, W, bias=torch.zeros(8)))
    _raises(ValueError, lambda: B.linear_fp8(b16, W, residual=b16))
    dy, xt, Wt = torch.zeros(4, 8, dtype=torch.bfloat16), _blocks(64, 4), _blocks(64, 8)
    _raises(ValueError, lambda: B.linear_fp8_backward(dy, None, Wt))
    _raises(ValueError, lambda: B.linear_fp8_backward(dy, xt, None))
    _raises(ValueError, lambda: B.linear_fp8_backward(dy, None, None, want_dx=False, want_dW=False))
    _raises(ValueError, lambda: B.linear_fp8_backward(dy, _blocks(64, 5), Wt))
    _raises(ValueError, lambda: B.linear_fp8_backward(dy, _blocks(72, 4), Wt))
    _raises(TypeError, lambda: B.linear_fp8_backward(dy, b16, Wt))
    _raises(TypeError, lambda: B.linear_fp8_backward(dy.float(), xt, Wt))
    _raises(TypeError, lambda: B.linear_fp8_backward(dy, xt, Wt, dW_dtype=torch.float16))
    _raises(ValueError, lambda: B.linear_fp8_backward(dy, xt, Wt, db=torch.zeros(9)))


def test_the_binding_checks_the_gated_blocks_arguments():
    bf = torch.bfloat16
    x, Wgu, Wd = torch.zeros(4, 64, dtype=bf), torch.zeros(48, 64, dtype=bf), torch.zeros(64, 24, dtype=bf)
    _raises(TypeError, lambda: B.gated_ffn(x.float(), Wgu, Wd))
    _raises(ValueError, lambda: B.gated_ffn(x, Wgu[:40], Wd))
    _raises(ValueError, lambda: B.gated_ffn(x, Wgu, Wd[:32]))
    _raises(ValueError, lambda: B.gated_ffn(x, Wgu, Wd, residual=x[:3]))
    _raises(ValueError, lambda: B.gated_ffn(x[0], Wgu, Wd))
    pre = torch.zeros(4, 48, dtype=bf)
    _raises(ValueError, lambda: B.gated_ffn_backward(x, x, Wgu, Wd, pre[:, :24]))
    _raises(ValueError, lambda: B.gated_ffn_backward(x[:2], x, Wgu, Wd, pre))
    _raises(ValueError, lambda: B.gated_ffn_backward(x, x, Wgu, Wd, pre, want_dx=False, want_dW=False))
    _raises(TypeError, lambda: B.gated_ffn_backward(x, x, Wgu, Wd, pre, dW_dtype=torch.float16))
    _raises(TypeError, lambda: B.gated_ffn_backward(x, x, Wgu, Wd, pre, dW_gu=torch.zeros(48, 64), dW_d=torch.zeros(64, 24, dtype=bf)))
    g, u, dn = _blocks(24, 64), _blocks(24, 64), _blocks(64, 24)
    _raises(TypeError, lambda: B.gated_ffn_fp8(x, g, u, Wd))
    _raises(TypeError, lambda: B.gated_ffn_fp8(x, None, u, dn))
    _raises(ValueError, lambda: B.gated_ffn_fp8(x, _blocks(32, 64), u, dn))
    _raises(ValueError, lambda: B.gated_ffn_fp8(x[:, :32], g, u, dn))
    _raises(TypeError, lambda: B.gated_ffn_fp8(x.float(), g, u, dn))
    _raises(ValueError, lambda: B.gated_ffn_fp8(x, g, u, dn, residual=x[:3]))


def test_the_dense_block_names_the_size_it_refuses():
    from paper_2603_06626_b200.dense import DenseBlock, Projection8
    with pytest.raises(ValueError, match="hidden"):
        DenseBlock(256, 200, device="cpu")
    with pytest.raises(ValueError, match="n:"):
        Projection8(256, 8, device="cpu")


def test_a_matrix_in_8_bits_is_looked_at_whenever_a_part_of_it_is_set():
    on, q = torch.device("cpu"), _blocks(3, 40)
    assert q.shape == (3, 40) and q.rows == 3 and q.cols == 40 and q.codes.shape == (3, 48)
    for good in (q, B.Fp8Blocks(q.codes, q.scales, 40), _blocks(3, 40, codes=q.codes.clone(), scales=q.scales.clone())):
        B._expect_fp8("q", good, 3, 40, on)
        _raises(ValueError, lambda: B._expect_fp8("q", good, 4, 40, on))
        _raises(ValueError, lambda: B._expect_fp8("q", good, 3, 41, on))
    wide = torch.empty(3, 96, dtype=torch.float8_e4m3fn)
    for parts in (dict(codes=q.codes[:2]), dict(codes=wide[:, :48]), dict(codes=q.codes.view(torch.uint8)), dict(codes=q.codes[0]), dict(cols=41),
                  dict(scales=q.scales[..., :2]), dict(scales=q.scales.transpose(3, 4)), dict(scales=q.scales.int()), dict(scales=q.scales[0])):
        made = B.Fp8Blocks(**{"codes": q.codes, "scales": q.scales, "cols": 40, **parts})
        for bad in (made, _blocks(3, 40, **parts)):
            _raises((ValueError, TypeError), lambda: B._expect_fp8("q", bad, 3, 40, on))
    back = _blocks(3, 40, cols=41)
    back.cols = 40
    B._expect_fp8("q", back, 3, 40, on)
