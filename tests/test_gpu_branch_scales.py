"""Scales at the ends of their range, and rows further apart than they are long: calls that the header allows and the other tests leave out."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def _bf(seed, *shape, std=1.0):
    return torch.from_numpy((np.random.default_rng(seed).normal(size=shape) * std).astype(np.float32)).to("cuda:0").bfloat16()


def _shifted(q, by):
    """The same codes with every scale multiplied by 2^by."""
    from paper_2603_06626_b200 import binding as B
    e = q.scales.int() + by
    used = q.scale_exponents().int() + by
    assert int(used.min()) >= 1 and int(used.max()) <= 254
    return B.Fp8Blocks(q.codes, e.clamp(0, 255).to(torch.uint8), q.cols)


@pytest.mark.parametrize("T", [1, 40, 500])
@pytest.mark.parametrize("up", [100, 60, -60, -110])
def test_scales_that_cancel(T, up):
    """x 2^up and W 2^-up have the products of x and W, bit for bit: powers of two are applied exactly, also far apart."""
    from paper_2603_06626_b200 import binding as B
    K, N = 520, 264
    x, W = B.quantize_fp8(_bf(T, T, K))[0], B.quantize_fp8(_bf(1, N, K, std=K ** -0.5), square=True)[0]
    r, b = _bf(2, T, N), _bf(3, N)
    want = B.linear_fp8(x, W, bias=b, residual=r)
    assert torch.equal(B.linear_fp8(_shifted(x, up), _shifted(W, -up), bias=b, residual=r), want)
    if T > 1:
        dy = _bf(4, T, N)
        xt, Wt = B.quantize_fp8(_bf(T, T, K), rows=False, transposed=True)[1], B.quantize_fp8(_bf(1, N, K, std=K ** -0.5), square=True, transposed=True)[1]
        dx, dW, _ = B.linear_fp8_backward(dy, xt, Wt, dW_dtype=torch.float32)
        s = 2.0 ** (up / 2)
        dx2, dW2, _ = B.linear_fp8_backward((dy.float() * s).bfloat16(), _shifted(xt, -up // 2), _shifted(Wt, -up // 2), dW_dtype=torch.float32)
        assert torch.equal(dx2, dx) and torch.equal(dW2, dW)
    B.check_status()


@pytest.mark.parametrize("T", [1, 12, 40, 500])
@pytest.mark.parametrize("up", [80, -80])
def test_a_gated_block_whose_scales_cancel(T, up):
    """Without an activation the block is linear in each of its matrices, and what one is larger by another is smaller by."""
    from paper_2603_06626_b200 import binding as B
    d, H = 264, 392
    x = _bf(T, T, d)
    W = [B.quantize_fp8(_bf(k, *s, std=s[1] ** -0.5), square=True)[0] for k, s in ((1, (H, d)), (2, (H, d)), (3, (d, H)))]
    want = B.gated_ffn_fp8(x, *W, act=B.ACT_NONE)
    assert torch.equal(B.gated_ffn_fp8(x, _shifted(W[0], up // 2), _shifted(W[1], up // 2), _shifted(W[2], -up), act=B.ACT_NONE), want)
    big = (x.float() * 2.0 ** (up // 2)).bfloat16()
    assert torch.equal(B.gated_ffn_fp8(big, _shifted(W[0], -up // 2), _shifted(W[1], -up // 2), W[2], act=B.ACT_NONE), want)
    assert torch.equal(B.gated_ffn_fp8(B.quantize_fp8(big)[0], _shifted(W[0], -up // 2), _shifted(W[1], -up // 2), W[2], act=B.ACT_NONE), want)
    B.check_status()


@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("rows,cols,ldy", [(5, 130, 131), (129, 517, 528), (300, 96, 104), (3, 1, 9), (64, 1024, 1500)])
def test_values_into_rows_that_are_further_apart(rows, cols, ldy, dtype):
    """grouter_dequantize_fp8 with a row stride: the places between the rows and behind the last one keep what they held."""
    from paper_2603_06626_b200 import binding as B
    lib = B.load_library()
    q = B.quantize_fp8(_bf(rows, rows, cols))[0]
    for shift in (0, 1):
        room = torch.full((rows * ldy + 8 + shift,), 7.0, dtype=dtype, device="cuda:0")
        y = room[shift:]
        assert lib.grouter_dequantize_fp8(q.codes.data_ptr(), q.scales.data_ptr(), rows, cols, ldy, B.F32 if dtype == torch.float32 else B.BF16,
                                          y.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
        m = y[:rows * ldy].view(rows, ldy)
        assert torch.equal(m[:, :cols], B.dequantize_fp8(q, dtype)) and (m[:, cols:] == 7).all() and (y[rows * ldy:] == 7).all()
        assert (room[:shift] == 7).all()


@pytest.mark.parametrize("T", [1, 70, 333])
def test_outputs_end_where_they_end(T):
    """Every output of the C calls in the middle of a larger buffer: what lies around it stays."""
    from paper_2603_06626_b200 import binding as B
    lib, st = B.load_library(), torch.cuda.current_stream().cuda_stream
    d, H = 136, 200
    around = 512

    def room(n, dtype):
        r = torch.full((n + 2 * around,), 7, dtype=dtype, device="cuda:0")
        return r, r[around:].data_ptr()

    def kept(r, n):
        return bool((r[:around] == 7).all() and (r[around + n:] == 7).all())

    x, dy, Wgu, Wd, p = _bf(T, T, d), _bf(T + 1, T, d), _bf(1, 2 * H, d), _bf(2, d, H), _bf(3, T, 2 * H)
    status = torch.zeros(1, dtype=torch.int32, device="cuda:0")
    h, y, pre = room(T * H, BF), room(T * d, BF), room(T * 2 * H, BF)
    assert lib.grouter_gated_ffn_fwd(x.data_ptr(), Wgu.data_ptr(), Wd.data_ptr(), None, T, d, H, B.ACT_SILU, h[1], y[1], pre[1], status.data_ptr(), st) == 0
    assert kept(h[0], T * H) and kept(y[0], T * d) and kept(pre[0], T * 2 * H)
    size = lib.grouter_gated_ffn_bwd_workspace_bytes(T, d, H)
    dx, dgu, dd, ws = room(T * d, BF), room(2 * H * d, torch.float32), room(d * H, torch.float32), room(size, torch.uint8)
    assert lib.grouter_gated_ffn_bwd(dy.data_ptr(), x.data_ptr(), Wgu.data_ptr(), Wd.data_ptr(), p.data_ptr(), T, d, H, B.ACT_SILU, dx[1], dgu[1], dd[1],
                                     B.F32, ws[1], status.data_ptr(), st) == 0
    assert kept(dx[0], T * d) and kept(dgu[0], 2 * H * d) and kept(dd[0], d * H) and kept(ws[0], size)
    q, t = B.quantize_fp8(x, transposed=True)
    W, Wt = B.quantize_fp8(Wgu[:H].contiguous(), square=True, transposed=True)
    z, dz = room(T * H, BF), _bf(4, T, H)
    assert lib.grouter_linear_fp8_fwd(q.codes.data_ptr(), q.scales.data_ptr(), 0, W.codes.data_ptr(), W.scales.data_ptr(), None, None, T, d, H, z[1], None,
                                      status.data_ptr(), st) == 0
    assert kept(z[0], T * H)
    size = lib.grouter_linear_fp8_bwd_workspace_bytes(T, d, H)
    dx, dW, db, ws = room(T * d, BF), room(H * d, torch.float32), room(H, torch.float32), room(size, torch.uint8)
    assert lib.grouter_linear_fp8_bwd(dz.data_ptr(), t.codes.data_ptr(), t.scales.data_ptr(), Wt.codes.data_ptr(), Wt.scales.data_ptr(), T, d, H, dx[1],
                                      dW[1], B.F32, db[1], ws[1], status.data_ptr(), st) == 0
    assert kept(dx[0], T * d) and kept(dW[0], H * d) and kept(db[0], H) and kept(ws[0], size)
    codes, codes_t = T * int(lib.grouter_fp8_pitch(d)), d * int(lib.grouter_fp8_pitch(T))
    sizes = [codes, int(lib.grouter_fp8_scale_bytes(T, d)), codes_t, int(lib.grouter_fp8_scale_bytes(d, T))]
    parts = [room(n, torch.uint8) for n in sizes]
    assert lib.grouter_quantize_fp8(x.data_ptr(), d, B.BF16, T, d, 0, *(v[1] for v in parts), st) == 0
    assert all(kept(v[0], n) for v, n in zip(parts, sizes))
    hh, yy, rs = room(T * d, BF), room(T * d, BF), room(T, torch.float32)
    w = _bf(5, d)
    assert lib.grouter_rmsnorm_fwd(x.data_ptr(), d, dy.data_ptr(), d, w.data_ptr(), T, d, B.BF16, B.BF16, 1e-6, hh[1], yy[1], None, rs[1], st) == 0
    assert kept(hh[0], T * d) and kept(yy[0], T * d) and kept(rs[0], T)
    size = lib.grouter_rmsnorm_bwd_workspace_bytes(T, d)
    dxx, dw, ws = room(T * d, BF), room(d, torch.float32), room(size, torch.uint8)
    assert lib.grouter_rmsnorm_bwd(dy.data_ptr(), x.data_ptr(), d, None, w.data_ptr(), rs[1], T, d, B.BF16, B.BF16, dxx[1], dw[1], ws[1], st) == 0
    assert kept(dxx[0], T * d) and kept(dw[0], d) and kept(ws[0], size)
    B.check_status(status=status)
