"""The operators of a dense gated feed-forward branch, as work to be timed: the root-mean-square norm on the residual stream, the matrix
product in 8 bits with a scale for 128 elements, and the gated feed-forward block in bf16 and in 8 bits.

Every case is a dict of plain values; `prepare` makes its inputs on the GPU, `run` makes one pass, either in plain torch
operations (32 bits throughout, rounded once at the end) or, with `own` set, through the framework's entry points.
What is held in 8 bits is e4m3 with a power-of-two scale for 128 neighbours of a row (weights: for a square of 128 x 128).
"""
import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}
BLOCK = 128                                  # elements of a row that share a scale
EPS = 1e-6


# ---------------------------------------------------------------- cases
def listed():
    return [
        # the norm before a dense branch at the width and batch of the framework's `large` workload, adding the residual
        dict(name="rms forward", op="rms", dir="fwd", T=32768, d=4096, type="bf16", wtype="bf16", residual=True, fp8=False, pad=0),
        # the same in front of 8-bit products, at the `skewed` workload's sizes: the output leaves as codes and scales
        dict(name="rms to 8 bits", op="rms", dir="fwd", T=16384, d=2048, type="bf16", wtype="f32", residual=True, fp8=True, pad=0),
        # its backward pass at those sizes, with the gradient that comes along the residual stream
        dict(name="rms backward", op="rms", dir="bwd", T=16384, d=2048, type="bf16", wtype="f32", residual=True, fp8=False, pad=0),
        # a short batch of an odd width, cut out of a wider tensor: unaligned rows, 32-bit activations
        dict(name="rms backward odd", op="rms", dir="bwd", T=1001, d=1023, type="f32", wtype="f32", residual=False, fp8=False, pad=2),
        # one token through a square projection onto the residual stream: reading the weight is all of it
        dict(name="fp8 token", op="fp8", dir="fwd", T=1, K=4096, N=4096, bias=False, residual=True, codes=True),
        # a projection of a training step at `large` (d = 4096, 1536 outputs) from bf16 activations, which the call puts into 8 bits
        dict(name="fp8 forward", op="fp8", dir="fwd", T=32768, K=4096, N=1536, bias=False, residual=False, codes=False),
        # backward at the `skewed` workload's sizes: both gradients as 8-bit products, from the transposed codes that forward left
        dict(name="fp8 backward", op="fp8", dir="bwd", T=16384, K=2048, N=1408, bias=True, residual=False, codes=False),
        # a few tokens being generated, through the whole branch in bf16
        dict(name="gated tokens", op="gated", dir="fwd", T=8, d=4096, H=1536, act="silu", residual=True, pre=False),
        # the dense branch in a training step of `large`, with what its backward pass needs
        dict(name="gated forward", op="gated", dir="fwd", T=32768, d=4096, H=1536, act="silu", residual=True, pre=True),
        # its backward pass at a ragged batch of `small` (d = 1024, hidden 2816): all three gradients
        dict(name="gated backward ragged", op="gated", dir="bwd", T=4095, d=1024, H=2816, act="gelu", residual=False, pre=True),
        # the branch in 8 bits as it is served: a long prompt, the hidden state goes from product to product as codes
        dict(name="gated 8 bits prompt", op="gated8", T=16384, d=4096, H=1536, act="silu", residual=True),
        # ... and one token
        dict(name="gated 8 bits token", op="gated8", T=1, d=4096, H=1536, act="silu", residual=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rms", "fp8", "gated", "gated8"])
    act = rng.choice(["silu", "silu", "gelu", "relu", "none"])
    while True:
        if op == "rms":
            c = dict(op=op, dir=rng.choice(["fwd", "bwd"]), T=_log(rng, 1, 65536), d=_log(rng, 64, 16384), type=rng.choice(["bf16", "f32"]),
                     wtype=rng.choice(["bf16", "f32"]), residual=rng.random() < 0.6, fp8=False, pad=rng.choice([0, 0, 8, 5]))
            if rng.random() < 0.6:
                c["d"] = max(64, c["d"] // 64 * 64)
                c["fp8"] = c["dir"] == "fwd" and rng.random() < 0.6
                if c["fp8"]:
                    c["pad"] = rng.choice([0, 8])
            if c["T"] * c["d"] <= 1 << 27:
                return c
        elif op == "fp8":
            d = rng.choice(["fwd", "bwd"])
            c = dict(op=op, dir=d, T=_log(rng, 1, 32768), K=8 * _log(rng, 8, 1024), N=8 * _log(rng, 2, 1024), bias=rng.random() < 0.4,
                     residual=d == "fwd" and rng.random() < 0.5, codes=d == "fwd" and rng.random() < 0.5)
            if c["T"] * c["K"] * c["N"] * (2 if d == "bwd" else 1) <= 1 << 37:
                return c
        elif op == "gated":
            d = rng.choice(["fwd", "bwd"])
            c = dict(op=op, dir=d, T=_log(rng, 1, 32768), d=8 * _log(rng, 8, 512), H=8 * _log(rng, 8, 512), act=act,
                     residual=d == "fwd" and rng.random() < 0.5, pre=d == "bwd" or rng.random() < 0.5)
            if c["T"] * c["d"] * c["H"] * (6 if d == "bwd" else 3) <= 1 << 38:
                return c
        else:
            c = dict(op=op, T=_log(rng, 1, 32768), d=8 * _log(rng, 8, 512), H=8 * _log(rng, 8, 512), act=act, residual=rng.random() < 0.5)
            if c["T"] * c["d"] * c["H"] * 3 <= 1 << 38:
                return c


# ---------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape, std=1.0, mean=0.0, dtype=torch.float32):
    return torch.empty(shape, dtype=torch.float32, device=DEVICE).normal_(mean, std, generator=g).to(dtype)


def _stream(g, T, d, dtype, pad=0):
    """Activations as they are in a model: rows of different size, a few channels far larger than the others."""
    x = _normal(g, T, d + pad) * torch.rand(T, 1, generator=g, device=DEVICE).add_(0.5)
    x[:, ::97] *= 8.0
    return x.to(dtype)[:, :d]


def _pack(scales):
    """Scales [rows, blocks of 128] in the order the 8-bit products read them: 512 bytes for 128 rows and four blocks."""
    rows, nb = scales.shape
    full = torch.full(((rows + 127) // 128 * 128, (nb + 3) // 4 * 4), 127, dtype=torch.uint8, device=scales.device)
    full[:rows, :nb] = scales
    return full.reshape(-1, 4, 32, full.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).contiguous()


def _keep(s, name, codes, scales, cols):
    """A matrix in 8 bits as a program keeps it: codes, their rows a multiple of 16 long, and the scales, plain and packed."""
    wide = torch.zeros(codes.shape[0], (cols + 15) // 16 * 16, dtype=torch.uint8, device=codes.device)
    wide[:, :cols] = codes.view(torch.uint8)
    s[name] = dict(codes=wide.view(torch.float8_e4m3fn), scales=scales, packed=_pack(scales), cols=cols)


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case)
    bf = torch.bfloat16
    if case["op"] == "rms":
        T, d, ty, wt = case["T"], case["d"], TYPES[case["type"]], TYPES[case["wtype"]]
        x = _stream(g, T, d, ty, case["pad"])
        s["w"] = _normal(g, d, std=0.2, mean=1.0, dtype=wt)
        r = _stream(g, T, d, ty) if case["residual"] else None
        if case["dir"] == "fwd":
            s["x"], s["r"] = x, r
        else:
            s["h"], s["dh"] = x, _normal(g, T, d, std=0.01, dtype=ty) if case["residual"] else None
            s["dy"] = _normal(g, T, d, std=0.01, dtype=ty)
            s["rstd"] = 1.0 / torch.sqrt(x.float().square().mean(1) + EPS)
    elif case["op"] == "fp8":
        T, K, N = case["T"], case["K"], case["N"]
        x, W = _stream(g, T, K, bf), _normal(g, N, K, std=K ** -0.5, dtype=bf)
        if case["dir"] == "fwd":
            s["x"] = x
            if case["codes"]:
                _keep(s, "x8", *_quantize(x.float()), K)
            _keep(s, "W8", *_quantize_square(W.float()), K)
            s["r"] = _normal(g, T, N, dtype=bf) if case["residual"] else None
            s["b"] = _normal(g, N, std=0.1, dtype=bf) if case["bias"] else None
        else:
            s["dy"] = _normal(g, T, N, std=0.01, dtype=bf)
            _keep(s, "xt8", *_quantize(x.float().t().contiguous()), T)
            _keep(s, "Wt8", *_quantize_square(W.float().t().contiguous()), N)
    else:
        T, d, H = case["T"], case["d"], case["H"]
        x = _normal(g, T, d, dtype=bf)
        Wg, Wu = _normal(g, H, d, std=d ** -0.5, dtype=bf), _normal(g, H, d, std=d ** -0.5, dtype=bf)
        Wd = _normal(g, d, H, std=H ** -0.5, dtype=bf)
        s["x"] = x
        s["r"] = _normal(g, T, d, dtype=bf) if case["residual"] else None
        if case["op"] == "gated8":
            _keep(s, "Wg8", *_quantize_square(Wg.float()), d)
            _keep(s, "Wu8", *_quantize_square(Wu.float()), d)
            _keep(s, "Wd8", *_quantize_square(Wd.float()), H)
        else:
            s["Wgu"], s["Wd"] = torch.cat([Wg, Wu]), Wd
            if case["dir"] == "bwd":
                s["dy"] = _normal(g, T, d, std=0.01, dtype=bf)
                s["p"] = _normal(g, T, 2 * H, dtype=bf)
    return s


# ---------------------------------------------------------------- plain forms
def _power_of_two(exp):
    return ((exp.to(torch.int32) + 127) << 23).view(torch.float32)


def _exponent(top):
    """The smallest e with top <= 448 * 2^e, 448 the largest e4m3 number."""
    frac, exp = torch.frexp(top)                                         # top = frac * 2^exp, frac in [0.5, 1)
    exp = torch.where(frac > 0.875, exp - 8, exp - 9)
    return torch.where(frac == 0, torch.full_like(exp, -126), exp).clamp(-126, 126)


def _blocks(x):
    """[rows, cols] as [rows, blocks, 128], zeros behind the last column."""
    rows, cols = x.shape
    if cols % BLOCK:
        x = torch.cat([x, x.new_zeros(rows, BLOCK - cols % BLOCK)], 1)
    return x.reshape(rows, -1, BLOCK)


def _quantize(x):
    """Codes (e4m3) of a matrix, one power-of-two scale for 128 elements of a row, and the exponents + 127."""
    b = _blocks(x)
    exp = _exponent(b.abs().max(2).values)
    codes = (b * _power_of_two(-exp)[:, :, None]).to(torch.float8_e4m3fn)
    return codes.reshape(x.shape[0], -1)[:, :x.shape[1]], (exp + 127).to(torch.uint8)


def _quantize_square(x):
    """The same with one scale for 128 x 128 elements, given for each of its rows."""
    rows = x.shape[0]
    b = _blocks(x)
    top = b.abs().max(2).values
    if rows % BLOCK:
        top = torch.cat([top, top.new_zeros(BLOCK - rows % BLOCK, top.shape[1])])
    exp = _exponent(top.reshape(-1, BLOCK, top.shape[1]).max(1).values).repeat_interleave(BLOCK, 0)[:rows]
    codes = (b * _power_of_two(-exp)[:, :, None]).to(torch.float8_e4m3fn)
    return codes.reshape(rows, -1)[:, :x.shape[1]], (exp + 127).to(torch.uint8)


def _values(codes, scales, cols):
    """What codes and scales stand for, in 32 bits."""
    f = _power_of_two(scales.to(torch.int32) - 127).repeat_interleave(BLOCK, 1)
    return codes[:, :cols].float() * f[:, :cols]


def _held(q):
    return _values(q["codes"], q["scales"], q["cols"])


def _rounded(x):
    """x as 8 bits hold it."""
    return _values(*_quantize(x), x.shape[1])


def _rms_forward(x, r, w, fp8):
    h = x if r is None else (x.float() + r.float()).to(x.dtype)
    hf = h.float()
    rstd = 1.0 / torch.sqrt(hf.square().mean(1) + EPS)
    y = hf * rstd[:, None] * w.float()
    y = _rounded(y).to(torch.bfloat16) if fp8 else y.to(x.dtype)         # e4m3 times a power of two is a bf16 number
    return (y, rstd) if r is None else (y, h, rstd)


def _rms_backward(dy, h, w, rstd, dh):
    u = h.float() * rstd[:, None]
    g = dy.float() * w.float()
    dx = rstd[:, None] * (g - u * (g * u).mean(1, keepdim=True))
    if dh is not None:
        dx = dx + dh.float()
    return dx.to(h.dtype), (dy.float() * u).sum(0)


def _fp8_forward(x, W, b, r):
    y = x @ W.t()
    if b is not None:
        y = y + b.float()
    if r is not None:
        y = y + r.float()
    return y.to(torch.bfloat16)


def _fp8_backward(dy, xt, Wt, bias):
    g = dy.float()
    dx = (_rounded(g) @ Wt.t()).to(torch.bfloat16)
    dW = (_rounded(g.t().contiguous()) @ xt.t()).to(torch.bfloat16)
    return (dx, dW, g.sum(0)) if bias else (dx, dW)


_C0, _C1 = math.sqrt(2.0 / math.pi), 0.044715


def _act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.tanh(_C0 * (z + _C1 * z * z * z)))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    if act == "gelu":
        t = torch.tanh(_C0 * (z + _C1 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * _C0 * (1 + 3 * _C1 * z * z)
    return torch.ones_like(z)


def _gated_forward(x, Wgu, Wd, r, act, pre):
    H = Wd.shape[1]
    p = x.float() @ Wgu.float().t()
    y = (_act(p[:, :H], act) * p[:, H:]) @ Wd.float().t()
    if r is not None:
        y = y + r.float()
    y = y.to(torch.bfloat16)
    return (y, p.to(torch.bfloat16)) if pre else y


def _gated_backward(dy, x, Wgu, Wd, p, act):
    H = Wd.shape[1]
    gate, up = p[:, :H].float(), p[:, H:].float()
    a = _act(gate, act)
    g = dy.float()
    dh = g @ Wd.float()
    dp = torch.cat([dh * up * _act_slope(gate, act), dh * a], 1)
    bf = torch.bfloat16
    return (dp @ Wgu.float()).to(bf), (dp.t() @ x.float()).to(bf), (g.t() @ (a * up)).to(bf)


def _gated8(x, Wg, Wu, Wd, r, act):
    v = _rounded(x.float())
    h = _rounded(_act(v @ Wg.t(), act) * (v @ Wu.t()))
    y = h @ Wd.t()
    if r is not None:
        y = y + r.float()
    return y.to(torch.bfloat16)


def _run_plain(s):
    if s["op"] == "rms":
        return _rms_forward(s["x"], s["r"], s["w"], s["fp8"]) if s["dir"] == "fwd" else _rms_backward(s["dy"], s["h"], s["w"], s["rstd"], s["dh"])
    if s["op"] == "fp8":
        if s["dir"] == "fwd":
            return _fp8_forward(_held(s["x8"]) if s["codes"] else _rounded(s["x"].float()), _held(s["W8"]), s["b"], s["r"])
        return _fp8_backward(s["dy"], _held(s["xt8"]), _held(s["Wt8"]), s["bias"])
    if s["op"] == "gated":
        if s["dir"] == "fwd":
            return _gated_forward(s["x"], s["Wgu"], s["Wd"], s["r"], s["act"], s["pre"])
        return _gated_backward(s["dy"], s["x"], s["Wgu"], s["Wd"], s["p"], s["act"])
    return _gated8(s["x"], _held(s["Wg8"]), _held(s["Wu8"]), _held(s["Wd8"]), s["r"], s["act"])


def _run_own(s):
    from paper_2603_06626_b200 import binding as B

    def kept(q):
        return B.Fp8Blocks(q["codes"], q["packed"], q["cols"])

    if s["op"] == "rms":
        if s["dir"] == "bwd":
            return B.rms_norm_backward(s["dy"], s["h"], s["w"], s["rstd"], dh=s["dh"])
        y, h, rstd = B.rms_norm(s["x"], s["w"], residual=s["r"], eps=EPS, fp8=s["fp8"])
        if s["fp8"]:
            y = B.dequantize_fp8(y)
        return (y, rstd) if s["r"] is None else (y, h, rstd)
    if s["op"] == "fp8":
        if s["dir"] == "fwd":
            return B.linear_fp8(kept(s["x8"]) if s["codes"] else s["x"], kept(s["W8"]), bias=s["b"], residual=s["r"])
        dx, dW, db = B.linear_fp8_backward(s["dy"], kept(s["xt8"]), kept(s["Wt8"]), want_bias=s["bias"])
        return (dx, dW, db) if s["bias"] else (dx, dW)
    act = dict(none=B.ACT_NONE, relu=B.ACT_RELU, silu=B.ACT_SILU, gelu=B.ACT_GELU)[s["act"]]
    if s["op"] == "gated":
        if s["dir"] == "fwd":
            y, p = B.gated_ffn(s["x"], s["Wgu"], s["Wd"], act=act, residual=s["r"], save_pre=s["pre"])
            return (y, p) if s["pre"] else y
        return B.gated_ffn_backward(s["dy"], s["x"], s["Wgu"], s["Wd"], s["p"], act=act)
    return B.gated_ffn_fp8(s["x"], kept(s["Wg8"]), kept(s["Wu8"]), kept(s["Wd8"]), act=act, residual=s["r"])


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["op"] == "rms":
        T, d = case["T"], case["d"]
        n, w = T * d * BYTES[case["type"]], d * BYTES[case["wtype"]]
        if case["dir"] == "fwd":
            y = 2 * T * d if case["fp8"] else n                          # the codes' values, which this case returns
            return dict(bytes=n + y + 2 * n * case["residual"] + w + 4 * T, flops=5 * T * d)
        return dict(bytes=3 * n + n * case["residual"] + w + 4 * d + 4 * T, flops=9 * T * d)
    if case["op"] == "fp8":
        T, K, N = case["T"], case["K"], case["N"]
        one = 2 * T * K * N
        if case["dir"] == "fwd":
            return dict(bytes=T * K * (1 if case["codes"] else 2) + N * K + 2 * T * N * (1 + case["residual"]) + 2 * N * case["bias"], flops=one)
        return dict(bytes=2 * T * N + T * K + N * K + 2 * T * K + 2 * N * K + 4 * N * case["bias"], flops=2 * one)
    T, d, H = case["T"], case["d"], case["H"]
    one = 2 * T * d * H
    if case["op"] == "gated":
        if case["dir"] == "fwd":
            return dict(bytes=2 * (T * d * (2 + case["residual"]) + 3 * d * H + 2 * T * H * case["pre"]), flops=3 * one)
        return dict(bytes=2 * (3 * T * d + 2 * T * H + 6 * d * H), flops=6 * one)
    return dict(bytes=2 * T * d * (2 + case["residual"]) + 3 * d * H, flops=3 * one)


# ---------------------------------------------------------------- the definitions in 64 bits
def _eight(x):
    """x, in 64 bits, as e4m3 codes of 128 neighbours with a power-of-two scale hold it: a step of 2^-3 of each number's own power of
    two, no finer than 2^-9, the largest 448."""
    rows, cols = x.shape
    b = torch.nn.functional.pad(x, (0, -cols % BLOCK)).unflatten(1, (-1, BLOCK))
    top = b.abs().amax(2, keepdim=True)
    e = torch.ceil(torch.log2(top / 448.0))
    e = torch.where(torch.exp2(e - 1) * 448.0 >= top, e - 1, e)          # the logarithm next to a whole number
    e = torch.where(torch.exp2(e) * 448.0 < top, e + 1, e)
    scale = torch.exp2(torch.where(top > 0, e, torch.full_like(e, -126.0)).clamp(min=-126.0))
    v = b / scale
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(v / step) * step * scale).flatten(1)[:, :cols]


def exact(case, seed):
    s = prepare(case, seed)
    D = lambda t: None if t is None else t.double()  # noqa: E731

    def stands_for(q):
        e = q["scales"].double().repeat_interleave(BLOCK, 1)[:, :q["cols"]] - 127
        return q["codes"][:, :q["cols"]].double() * torch.exp2(e)

    if case["op"] == "rms":
        w, d = D(s["w"]), case["d"]
        if case["dir"] == "fwd":
            total = D(s["x"]) if s["r"] is None else D(s["x"]) + D(s["r"])
            h = total.to(TYPES[case["type"]]).double()                   # the norm is that of the stream as it is stored
            rstd = ((h * h).sum(1) / d + EPS) ** -0.5
            y = torch.einsum("td,t,d->td", h, rstd, w)
            y = _eight(y) if case["fp8"] else y
            return (y, rstd) if s["r"] is None else (y, total, rstd)
        dy, h, rstd = D(s["dy"]), D(s["h"]), D(s["rstd"])
        dot = torch.einsum("td,td,d->t", dy, h, w) / d
        dx = torch.einsum("td,d,t->td", dy, w, rstd) - torch.einsum("td,t->td", h, rstd ** 3 * dot)
        if s["dh"] is not None:
            dx = dx + D(s["dh"])
        return dx, torch.einsum("td,td,t->d", dy, h, rstd)
    if case["op"] == "fp8":
        if case["dir"] == "fwd":
            x = stands_for(s["x8"]) if case["codes"] else _eight(D(s["x"]))
            y = torch.einsum("tk,nk->tn", x, stands_for(s["W8"]))
            y = y if s["b"] is None else y + D(s["b"])
            return y if s["r"] is None else y + D(s["r"])
        dy = D(s["dy"])
        dx = torch.einsum("tn,kn->tk", _eight(dy), stands_for(s["Wt8"]))
        dW = torch.einsum("nt,kt->nk", _eight(dy.t()), stands_for(s["xt8"]))
        return (dx, dW, dy.sum(0)) if case["bias"] else (dx, dW)
    act = case["act"]

    def sig(z):
        return torch.special.expit(z)

    def inner(z):
        return 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)

    value = dict(none=lambda z: z, relu=lambda z: torch.where(z > 0, z, 0 * z), silu=lambda z: z * sig(z), gelu=lambda z: z * sig(inner(z)))[act]
    x, r = D(s["x"]), D(s["r"])
    if case["op"] == "gated8":
        v = _eight(x)
        gate, up = (torch.einsum("td,hd->th", v, stands_for(s[n])) for n in ("Wg8", "Wu8"))
        y = torch.einsum("th,dh->td", _eight(value(gate) * up), stands_for(s["Wd8"]))
        return y if r is None else y + r
    H = case["H"]
    Wg, Wu, Wd = D(s["Wgu"][:H]), D(s["Wgu"][H:]), D(s["Wd"])
    if case["dir"] == "fwd":
        gate, up = torch.einsum("td,hd->th", x, Wg), torch.einsum("td,hd->th", x, Wu)
        y = torch.einsum("th,dh->td", value(gate) * up, Wd)
        y = y if r is None else y + r
        return (y, torch.cat([gate, up], 1)) if case["pre"] else y
    slope = dict(none=lambda z: torch.ones_like(z), relu=lambda z: (z > 0).double(), silu=lambda z: sig(z) + z * sig(z) * sig(-z),
                 gelu=lambda z: sig(inner(z)) + z * sig(inner(z)) * sig(-inner(z)) * 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z ** 2))[act]
    gate, up, dy = D(s["p"][:, :H]), D(s["p"][:, H:]), D(s["dy"])
    dh = torch.einsum("td,dh->th", dy, Wd)
    dg, du = dh * up * slope(gate), dh * value(gate)
    dx = torch.einsum("th,hd->td", dg, Wg) + torch.einsum("th,hd->td", du, Wu)
    dWgu = torch.cat([torch.einsum("th,td->hd", dg, x), torch.einsum("th,td->hd", du, x)])
    return dx, dWgu, torch.einsum("td,th->dh", dy, value(gate) * up)
