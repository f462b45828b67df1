"""Calls back to back on one stream, whose kernels start before the ones before them have ended: a gradient's product that read too early what the
kernels before it leave in the workspace would find NaN there, or another call's numbers.  Every result is, bit for bit, that of the same
call alone with the device waited for."""
import itertools

import pytest
import torch

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
DEV = "cuda:0"


def _rand(g, *s, std=1.0):
    return torch.empty(s, device=DEV).normal_(0, std, generator=g).to(BF)


def _workspace(size):
    return torch.empty(size, dtype=torch.uint8, device=DEV)


def _same(a, b):
    return all(p is None and q is None or torch.equal(p, q) for p, q in zip(a, b))


def _check(calls, outputs, workspace):
    """calls[i]() writes outputs[i]; all of them use `workspace`.  Alone first, then in a row, then in a row with the workspace filled with NaN
    (as bf16, f32 and e4m3 alike) and the outputs spoiled in front of every call."""
    def spoil(i):
        workspace.fill_(255)
        for o in outputs[i]:
            if o is not None:
                o.fill_(float("nan"))

    want = []
    for i, call in enumerate(calls):
        spoil(i)
        torch.cuda.synchronize()
        call()
        torch.cuda.synchronize()
        want.append([None if o is None else o.clone() for o in outputs[i]])
        assert all(o is None or torch.isfinite(o.float()).all() for o in outputs[i])
    for between in (lambda i: None, spoil):
        for _ in range(4):
            for i in range(len(calls)):
                spoil(i)
            for i, call in enumerate(calls):
                between(i)
                call()
            torch.cuda.synchronize()
            for i in range(len(calls)):
                assert _same(outputs[i], want[i]), i


# dx by the kernel for few tokens and by tiles; one round of tiles and several; weight gradients in one piece and in several
@pytest.mark.parametrize("T,d,H", [(8, 1024, 520), (60, 264, 136), (300, 520, 264), (4095, 1024, 2816), (9000, 264, 520)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_gated_backward(T, d, H, dtype):
    from paper_2603_06626_b200 import binding as B
    lib, g = B.load_library(), torch.Generator(device=DEV).manual_seed(T)
    ws, status = _workspace(lib.grouter_gated_ffn_bwd_workspace_bytes(T, d, H)), torch.zeros(1, dtype=torch.int32, device=DEV)
    calls, outputs, held = [], [], []
    for wants in itertools.product((True, False), repeat=3):
        if not any(wants):
            continue
        t = [_rand(g, T, d), _rand(g, T, d), _rand(g, 2 * H, d, std=d ** -0.5), _rand(g, d, H, std=H ** -0.5), _rand(g, T, 2 * H)]
        out = [torch.empty(s, dtype=kind, device=DEV) if w else None for s, kind, w in zip(((T, d), (2 * H, d), (d, H)), (BF, dtype, dtype), wants)]
        args = [x.data_ptr() for x in t] + [T, d, H, B.ACT_SILU] + [None if o is None else o.data_ptr() for o in out]
        args += [B.F32 if dtype == F32 else B.BF16, ws.data_ptr(), status.data_ptr()]

        def call(args=args):
            assert lib.grouter_gated_ffn_bwd(*args, torch.cuda.current_stream().cuda_stream) == 0
        calls.append(call)
        outputs.append(out)
        held.append(t)
    _check(calls, outputs, ws)
    B.check_status(status=status)


@pytest.mark.parametrize("T,K,N", [(8, 1032, 264), (64, 264, 520), (600, 520, 264), (9000, 1032, 520), (20000, 264, 264)])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_eight_bits_backward(T, K, N, dtype):
    from paper_2603_06626_b200 import binding as B
    lib, g = B.load_library(), torch.Generator(device=DEV).manual_seed(T)
    ws, status = _workspace(lib.grouter_linear_fp8_bwd_workspace_bytes(T, K, N)), torch.zeros(1, dtype=torch.int32, device=DEV)
    calls, outputs, held = [], [], []
    for wants in itertools.product((True, False), repeat=3):
        if not any(wants):
            continue
        xt = B.quantize_fp8(_rand(g, T, K), rows=False, transposed=True)[1]
        Wt = B.quantize_fp8(_rand(g, N, K, std=K ** -0.5), square=True, rows=False, transposed=True)[1]
        dy = _rand(g, T, N)
        out = [torch.empty(s, dtype=kind, device=DEV) if w else None for s, kind, w in zip(((T, K), (N, K), (N,)), (BF, dtype, F32), wants)]
        parts = [dy.data_ptr()] + [v.data_ptr() for q in (xt, Wt) for v in (q.codes, q.scales)]
        args = parts + [T, K, N, *[None if o is None else o.data_ptr() for o in out[:2]], B.F32 if dtype == F32 else B.BF16,
                        None if out[2] is None else out[2].data_ptr(), ws.data_ptr(), status.data_ptr()]

        def call(args=args):
            assert lib.grouter_linear_fp8_bwd(*args, torch.cuda.current_stream().cuda_stream) == 0
        calls.append(call)
        outputs.append(out)
        held.append((xt, Wt, dy))
    _check(calls, outputs, ws)
    B.check_status(status=status)


@pytest.mark.parametrize("T,d", [(3, 128), (700, 1024), (5000, 4096), (600, 16384)])
def test_what_the_kernel_before_wrote_is_what_is_read(T, d):
    """Weights and activations that a kernel of the framework wrote directly before, over and over into the same place."""
    from paper_2603_06626_b200 import binding as B
    lib, g = B.load_library(), torch.Generator(device=DEV).manual_seed(T)
    w8 = [B.quantize_fp8(_rand(g, 1, d))[0] for _ in range(3)]
    x8 = [B.quantize_fp8(_rand(g, T, d))[0] for _ in range(3)]
    dy = _rand(g, T, d)

    def values(q, to):
        rows, cols = q.shape
        assert lib.grouter_dequantize_fp8(q.codes.data_ptr(), q.scales.data_ptr(), rows, cols, cols, B.BF16, to.data_ptr(),
                                          torch.cuda.current_stream().cuda_stream) == 0

    want = []
    for wq, xq in zip(w8, x8):
        w, x = B.dequantize_fp8(wq)[0], B.dequantize_fp8(xq)
        torch.cuda.synchronize()
        y, _, rstd = B.rms_norm(x, w)
        torch.cuda.synchronize()
        want.append([y, rstd, *B.rms_norm_backward(dy, x, w, rstd), *(p for q in B.quantize_fp8(x, transposed=True) for p in (q.codes.view(torch.uint8),
                                                                                                                 q.scale_exponents()))])
        torch.cuda.synchronize()
    w, x = torch.empty(d, dtype=BF, device=DEV), torch.empty(T, d, dtype=BF, device=DEV)
    for n in range(12):
        i = n % 3
        values(x8[i], x)
        values(w8[i], w)
        y, _, rstd = B.rms_norm(x, w)
        got = [y, rstd]
        values(w8[i - 1], w)
        values(w8[i], w)
        got += B.rms_norm_backward(dy, x, w, rstd)
        values(x8[i - 1], x)
        values(x8[i], x)
        got += [p for q in B.quantize_fp8(x, transposed=True) for p in (q.codes.view(torch.uint8), q.scale_exponents())]
        torch.cuda.synchronize()
        assert _same(got, want[i])
