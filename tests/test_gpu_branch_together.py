"""The dense branch's operators on two streams and from two threads at once: nothing they use is shared but the inputs, so every result is the
one that a call alone gives."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def _calls():
    """One call of every operator and of each of its kernels (few tokens and tiles), on inputs of their own, as functions that return tensors."""
    from paper_2603_06626_b200 import binding as B
    g = torch.Generator(device="cuda:0").manual_seed(0)
    rand = lambda *s, std=1.0: torch.empty(s, device="cuda:0").normal_(0, std, generator=g).to(BF)  # noqa: E731
    d, H = 1024, 520
    Wgu, Wd, w = rand(2 * H, d, std=d ** -0.5), rand(d, H, std=H ** -0.5), rand(d)
    W8 = [B.quantize_fp8(W.contiguous(), square=True)[0] for W in (Wgu[:H], Wgu[H:], Wd)]
    Wt = B.quantize_fp8(Wgu[:H].contiguous(), square=True, rows=False, transposed=True)[1]
    calls = []
    for T in (1, 24, 60, 120, 700):
        x, dy, dh, p = rand(T, d), rand(T, d), rand(T, H), rand(T, 2 * H)

        def blocks(x=x):
            q, t = B.quantize_fp8(x, transposed=True)
            return [B.dequantize_fp8(q), B.dequantize_fp8(t)]

        def norm(x=x, dy=dy):
            y, h, rstd = B.rms_norm(x, w, residual=dy)
            return [y, h, B.dequantize_fp8(B.rms_norm(x, w, fp8=True)[0]), *B.rms_norm_backward(dy, h, w, rstd, dh=x)]

        def linear(x=x, dh=dh):
            q, t = B.quantize_fp8(x, transposed=True)
            return [B.linear_fp8(x, W8[0]), B.linear_fp8(q, W8[1]), *B.linear_fp8_backward(dh, t, Wt, want_bias=True)]

        def gated(x=x, dy=dy, p=p):
            return [B.gated_ffn(x, Wgu, Wd, residual=dy)[0], B.gated_ffn_fp8(x, *W8, residual=dy), *B.gated_ffn_backward(dy, x, Wgu, Wd, p)]

        calls += [blocks, norm, linear, gated]
    return calls


def _same(got, want):
    return all(torch.equal(a, b) for a, b in zip(got, want))


def test_two_streams():
    from paper_2603_06626_b200 import binding as B
    calls = _calls()
    want = [c() for c in calls]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for _ in range(3):
        for i in range(len(calls)):
            for s, order in enumerate((i, len(calls) - 1 - i)):
                with torch.cuda.stream(streams[s]):
                    got[s].append((order, calls[order]()))
    torch.cuda.synchronize()
    B.check_status()
    assert all(_same(out, want[i]) for one in got for i, out in one)


def test_two_threads():
    from paper_2603_06626_b200 import binding as B
    calls = _calls()
    want = [c() for c in calls]
    torch.cuda.synchronize()
    wrong = []

    def work(order):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(3):
                outs = [(i, calls[i]()) for i in order]
                torch.cuda.current_stream().synchronize()
                wrong.extend(i for i, out in outs if not _same(out, want[i]))

    threads = [threading.Thread(target=work, args=(order,)) for order in (range(len(calls)), reversed(range(len(calls))))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    B.check_status()
    assert not wrong


def test_a_graph_beside_eager_calls():
    """Two graphs of all calls, replayed on one stream while the calls run on another."""
    from paper_2603_06626_b200 import binding as B
    calls = _calls()
    want = [c() for c in calls]
    torch.cuda.synchronize()
    graphs, held = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for g in graphs:
        with torch.cuda.graph(g):
            held.append([c() for c in calls])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    eager = []
    for g in graphs + graphs:
        with torch.cuda.stream(side):
            g.replay()
        eager.append([c() for c in calls])
    torch.cuda.synchronize()
    B.check_status()
    assert all(_same(a, b) for outs in held + eager for a, b in zip(outs, want))
