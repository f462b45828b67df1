"""The operators around the routed expert layer in one training step, as work to be timed: layer norm, the linear layer
with its epilogue, the router's balance loss with the gradient of its scores, and the AdamW step.

Every case is a dict of plain values; `prepare` makes its inputs on the GPU, `run` makes one pass, either in plain torch
operations (32 bits throughout, rounded once at the end) or, with `own` set, through the framework's entry points.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}
BLOCK = 32                                   # elements that share a scale in the 8-bit optimizer state
HYPER = dict(lr=3e-4, beta1=0.9, beta2=0.95, eps=1e-8)
STEPS_BEFORE = 10                            # optimizer steps the state has behind it


# ---------------------------------------------------------------- cases
def listed():
    return [
        # the norm before the expert layer, at the width and batch of the framework's `large` workload
        dict(name="norm forward", op="norm", dir="fwd", T=32768, d=4096, type="bf16", wtype="bf16", pad=0),
        # its backward pass at the `skewed` workload's sizes, with the reduction of both weight gradients
        dict(name="norm backward", op="norm", dir="bwd", T=16384, d=2048, type="bf16", wtype="f32", pad=0),
        # a short batch of an odd width, cut out of a wider tensor: unaligned rows, 32-bit activations
        dict(name="norm backward odd", op="norm", dir="bwd", T=1001, d=1023, type="f32", wtype="f32", pad=2),
        # one token through a square projection onto the residual stream: reading the weight is all of it
        dict(name="linear token", op="linear", dir="fwd", T=1, K=4096, N=4096, act="none", bias=False, residual=True, pre=False),
        # the dense branch beside the routed experts (`large`: d = 4096, hidden 1536), forward of a training step
        dict(name="linear up", op="linear", dir="fwd", T=32768, K=4096, N=1536, act="silu", bias=True, residual=False, pre=True),
        # its way back down at a ragged batch (`small`: hidden 2816, d = 1024), added to the residual stream
        dict(name="linear down ragged", op="linear", dir="fwd", T=4095, K=2816, N=1024, act="none", bias=True, residual=True, pre=False),
        # backward of an activated projection at the `skewed` workload's sizes: three gradients
        dict(name="linear backward", op="linear", dir="bwd", T=16384, K=2048, N=1408, act="gelu", bias=True, residual=False, pre=True),
        # router training at `large`: 128 experts, 8 kept, losses and the gates' gradient joined
        dict(name="balance", op="balance", T=32768, E=128, k=8, type="f32", idx="u8", norm="softmax", gates=True, mask=False),
        # a small batch with padding tokens and sigmoid gates: latency
        dict(name="balance small masked", op="balance", T=511, E=8, k=2, type="bf16", idx="i32", norm="sigmoid", gates=True, mask=True),
        # a whole accumulation of a million tokens with 256 experts, balance and z losses only
        dict(name="balance wide", op="balance", T=1048575, E=256, k=8, type="bf16", idx="u8", norm="softmax", gates=False, mask=True),
        # one block of the `small` workload: 16 experts' weights with 32-bit gradients as the layer's backward pass leaves them
        dict(name="adamw experts", op="adamw", blocks=1, d=1024, ffn=2816, E=16, bits=32, grad="f32", param="bf16"),
        # many small tensors of odd sizes (norms, biases, score layers), states in 8 bits
        dict(name="adamw odd 8 bits", op="adamw", blocks=24, d=257, ffn=65, E=5, bits=8, grad="bf16", param="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "linear", "balance", "adamw"])
    while True:
        if op == "norm":
            c = dict(op=op, dir=rng.choice(["fwd", "bwd"]), T=_log(rng, 1, 65536), d=_log(rng, 64, 16384), type=rng.choice(["bf16", "f32"]),
                     wtype=rng.choice(["bf16", "f32"]), pad=rng.choice([0, 0, 8, 5]))
            if rng.random() < 0.5:
                c["d"] = max(64, c["d"] // 64 * 64)
            if c["T"] * c["d"] <= 1 << 27:
                return c
        elif op == "linear":
            d = rng.choice(["fwd", "bwd"])
            act = rng.choice(["none", "relu", "silu", "gelu"])
            c = dict(op=op, dir=d, T=_log(rng, 1, 32768), K=8 * _log(rng, 8, 1024), N=8 * _log(rng, 2, 1024), act=act,
                     bias=rng.random() < 0.5, residual=d == "fwd" and rng.random() < 0.5, pre=act != "none" and (d == "bwd" or rng.random() < 0.5))
            if c["T"] * c["K"] * c["N"] * (2 if d == "bwd" else 1) <= 1 << 37:
                return c
        elif op == "balance":
            E = rng.choice([8, 16, 60, 64, 128, 160, 256, _log(rng, 8, 1024)])
            c = dict(op=op, T=_log(rng, 1, 1 << 20), E=E, k=rng.randint(1, min(8, E)), type=rng.choice(["bf16", "f32"]),
                     idx="i32" if E > 256 else rng.choice(["u8", "i32"]), norm=rng.choice(["softmax", "sigmoid"]), gates=rng.random() < 0.5,
                     mask=rng.random() < 0.5)
            if c["T"] * c["E"] <= 1 << 27:
                return c
        else:
            c = dict(op=op, blocks=rng.randint(1, 16), d=_log(rng, 64, 2048), ffn=_log(rng, 64, 2048), E=_log(rng, 1, 16), bits=rng.choice([8, 32]),
                     grad=rng.choice(["f32", "bf16"]), param=rng.choice(["f32", "bf16"]))
            if sum(_sizes(c)) <= 1 << 27:
                return c


def _sizes(c):
    """Elements of every tensor of the blocks: the experts' two matrices, the score layer, the norm's weight and bias."""
    d, f, E = c["d"], c["ffn"], c["E"]
    return [E * 2 * f * d, E * d * f, E * d, d, d] * c["blocks"]


# ---------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape, std=1.0, mean=0.0, dtype=torch.float32):
    return torch.empty(shape, dtype=torch.float32, device=DEVICE).normal_(mean, std, generator=g).to(dtype)


def _spread(sizes):
    """Where each tensor starts in a flat buffer whose tensors begin on a block of their own, and its length."""
    at, total = [], 0
    for n in sizes:
        at.append(total)
        total += (n + BLOCK - 1) // BLOCK * BLOCK
    return at, total


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case)
    if case["op"] == "norm":
        T, d, ty, wt = case["T"], case["d"], TYPES[case["type"]], TYPES[case["wtype"]]
        s["x"] = (_normal(g, T, d + case["pad"]) * torch.rand(T, 1, generator=g, device=DEVICE).add_(0.5) + 0.1).to(ty)[:, :d]
        s["w"], s["b"] = _normal(g, d, std=0.2, mean=1.0, dtype=wt), _normal(g, d, std=0.2, dtype=wt)
        if case["dir"] == "bwd":
            s["dy"] = _normal(g, T, d, std=0.01, dtype=ty)
            xf = s["x"].float()
            s["mean"] = xf.mean(1)
            s["rstd"] = 1.0 / torch.sqrt((xf - s["mean"][:, None]).square().mean(1) + 1e-5)
    elif case["op"] == "linear":
        T, K, N = case["T"], case["K"], case["N"]
        bf = torch.bfloat16
        s["x"], s["W"] = _normal(g, T, K, dtype=bf), _normal(g, N, K, std=K ** -0.5, dtype=bf)
        s["b"] = _normal(g, N, std=0.1, dtype=bf) if case["bias"] else None
        if case["dir"] == "fwd":
            s["r"] = _normal(g, T, N, dtype=bf) if case["residual"] else None
        else:
            s["dy"] = _normal(g, T, N, std=0.01, dtype=bf)
            s["z"] = _normal(g, T, N, dtype=bf) if case["pre"] else None
    elif case["op"] == "balance":
        T, E, k = case["T"], case["E"], case["k"]
        logits = _normal(g, T, E, std=1.5) + _normal(g, E, std=0.7)      # some experts are liked more than others
        s["logits"] = logits.to(TYPES[case["type"]])
        s["i"] = torch.cat([c.topk(k, dim=1).indices for c in s["logits"].split(65536)]).to(torch.uint8 if case["idx"] == "u8" else torch.int32)
        s["m"] = (torch.rand(T, generator=g, device=DEVICE) < 0.9).to(torch.uint8) if case["mask"] else None
        s["dg"] = _normal(g, T, k, std=1e-3) if case["gates"] else None
    else:
        sizes = _sizes(case)
        at, total = _spread(sizes)
        views = lambda flat: [flat[a:a + n] for a, n in zip(at, sizes)]  # noqa: E731
        inside = torch.zeros(total, dtype=torch.bool, device=DEVICE)
        torch._foreach_zero_([v.view(torch.uint8) for v in views(inside)])
        torch._foreach_add_([v.view(torch.uint8) for v in views(inside)], 1)
        s["grads"] = views(_normal(g, total, std=1e-3, dtype=TYPES[case["grad"]]))
        p = _normal(g, total, std=0.02) * inside
        s["master_flat"] = p
        s["param_flat"] = p.to(torch.bfloat16) if case["param"] == "bf16" else p
        s["master"], s["param"] = views(s["master_flat"]), views(s["param_flat"])
        s["decay"] = [0.1, 0.1, 0.1, 0.0, 0.0] * case["blocks"]          # norms' weights and biases do not decay
        s["scale"] = torch.full((1,), 0.5, device=DEVICE)                # a clipping coefficient that stays on the GPU
        s["t"] = STEPS_BEFORE
        m, v = _normal(g, total, std=3e-4) * inside, _normal(g, total, std=1e-3).square() * inside
        if case["bits"] == 32:
            s["m_flat"], s["v_flat"] = m, v
            s["m"], s["v"] = views(m), views(v)
        else:
            s["m_code"], s["m_exp"] = _to_codes(m, False)
            s["r_code"], s["r_exp"] = _to_codes(torch.sqrt(v), True)
            s["at"], s["sizes"] = at, sizes
        if own:                                                          # the optimizer that a training program keeps
            from paper_2603_06626_b200 import binding
            state = dict(m=s["m_flat"], v=s["v_flat"]) if case["bits"] == 32 else \
                dict(m=s["m_code"], m_exp=s["m_exp"], v=s["r_code"], v_exp=s["r_exp"])
            if case["param"] == "bf16":
                state["master"] = s["master_flat"]
            s["optimizer"] = binding.AdamW(s["param"], s["grads"], lr=HYPER["lr"], betas=(HYPER["beta1"], HYPER["beta2"]), eps=HYPER["eps"],
                                           weight_decay=s["decay"], state_bits=case["bits"], state=state, steps_done=STEPS_BEFORE)
    return s


# ---------------------------------------------------------------- plain forms
def _norm_forward(x, w, b):
    xf = x.float()
    mean = xf.mean(1)
    c = xf - mean[:, None]
    rstd = 1.0 / torch.sqrt(c.square().mean(1) + 1e-5)
    return (c * rstd[:, None] * w.float() + b.float()).to(x.dtype), mean, rstd


def _norm_backward(dy, x, w, mean, rstd):
    h = (x.float() - mean[:, None]) * rstd[:, None]
    g = dy.float()
    gw = g * w.float()
    dx = rstd[:, None] * (gw - gw.mean(1, keepdim=True) - h * (gw * h).mean(1, keepdim=True))
    return dx.to(x.dtype), (g * h).sum(0), g.sum(0)


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


def _linear_forward(x, W, b, r, act, pre):
    z = x.float() @ W.float().t()
    if b is not None:
        z = z + b.float()
    y = _act(z, act)
    if r is not None:
        y = y + r.float()
    y = y.to(torch.bfloat16)
    return (y, z.to(torch.bfloat16)) if pre else y


def _linear_backward(dy, x, W, z, act, bias):
    dz = dy.float() if z is None else dy.float() * _act_slope(z.float(), act)
    dx, dW = (dz @ W.float()).to(torch.bfloat16), (dz.t() @ x.float()).to(torch.bfloat16)
    return (dx, dW, dz.sum(0)) if bias else (dx, dW)


BALANCE_COEF, Z_COEF = 1e-2, 1e-3


def _balance(logits, idx, mask, dg, norm):
    T, E = logits.shape
    k = idx.shape[1]
    keep = torch.ones(T, dtype=torch.bool, device=logits.device) if mask is None else mask != 0
    i = idx.long()
    counts = torch.zeros(E, dtype=torch.int32, device=logits.device)
    counts.index_add_(0, i.reshape(-1), keep[:, None].expand(T, k).reshape(-1).to(torch.int32))
    n = keep.sum().to(torch.int32).reshape(1)
    x = logits.float()
    top = x.max(1, keepdim=True).values
    e = torch.exp(x - top)
    total = e.sum(1, keepdim=True)
    p = e / total
    lse = (top + torch.log(total)).squeeze(1)
    f = counts.float() * (float(E) / torch.clamp(counts.sum(), min=1).float())
    share = (p * f).sum(1)
    live = keep.float()
    per = 1.0 / torch.clamp(n, min=1).float()
    balance, z = (share * live).sum() * per, (lse.square() * live).sum() * per
    loss = torch.cat([BALANCE_COEF * balance + Z_COEF * z, balance, z])
    d = p * ((BALANCE_COEF * per) * (f - share[:, None]) + (2 * Z_COEF * per) * lse[:, None])
    if dg is not None:
        kept = x.gather(1, i)
        if norm == "softmax":
            q = torch.exp(kept - kept.max(1, keepdim=True).values)
            q = q / q.sum(1, keepdim=True)
            back = q * (dg - (q * dg).sum(1, keepdim=True))
        else:
            q = 1 / (1 + torch.exp(-kept))
            back = q * (1 - q) * dg
        d.scatter_add_(1, i, back)
    return dict(counts=counts, tokens=n, loss=loss, dlogits=(d * live[:, None]).to(logits.dtype))


def _power_of_two(exp):
    return ((exp.to(torch.int32) + 127) << 23).view(torch.float32)


def _to_codes(flat, root):
    """8-bit codes (e4m3, one power-of-two scale for 32 elements) of a flat buffer, as (codes, exponents + 127)."""
    blocks = flat.reshape(-1, BLOCK)
    frac, exp = torch.frexp(blocks.abs().max(1).values)                  # largest = frac * 2^exp, frac in [0.5, 1)
    exp = torch.where(frac > 0.875, exp - 8, exp - 9)                    # smallest scale under which it is at most 448
    exp = torch.where(frac == 0, torch.full_like(exp, -126), exp).clamp(-126, 126)
    code = (blocks * _power_of_two(-exp)[:, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    if root:                                                             # a root that is there stays above zero
        code = torch.where((code == 0) & (blocks > 0), torch.ones_like(code), code)
    return code.reshape(-1), (exp + 127).to(torch.uint8)


def _from_codes(code, exp):
    return (code.view(torch.float8_e4m3fn).float().reshape(-1, BLOCK) * _power_of_two(exp.to(torch.int32) - 127)[:, None]).reshape(-1)


def _adamw(s):
    s["t"] += 1
    lr, b1, b2, eps = HYPER["lr"], HYPER["beta1"], HYPER["beta2"], HYPER["eps"]
    c1, c2 = 1 - b1 ** s["t"], 1 - b2 ** s["t"]
    g = torch._foreach_mul([x.float() for x in s["grads"]], s["scale"].squeeze())
    if s["bits"] == 32:
        m, v = s["m"], s["v"]
    else:
        flat_m, flat_r = _from_codes(s["m_code"], s["m_exp"]), _from_codes(s["r_code"], s["r_exp"])
        flat_v = flat_r * flat_r
        m = [flat_m[a:a + n] for a, n in zip(s["at"], s["sizes"])]
        v = [flat_v[a:a + n] for a, n in zip(s["at"], s["sizes"])]
    torch._foreach_mul_(m, b1)
    torch._foreach_add_(m, torch._foreach_mul(g, 1 - b1))
    torch._foreach_mul_(v, b2)
    torch._foreach_mul_(g, g)
    torch._foreach_mul_(g, 1 - b2)
    torch._foreach_add_(v, g)
    root = torch._foreach_sqrt(v)
    torch._foreach_mul_(root, 1 / math.sqrt(c2))
    torch._foreach_add_(root, eps)
    step = torch._foreach_div(m, root)
    torch._foreach_mul_(step, lr / c1)
    torch._foreach_mul_(s["master"], [1 - lr * w for w in s["decay"]])
    torch._foreach_sub_(s["master"], step)
    if s["param"][0].dtype != torch.float32:
        torch._foreach_copy_(s["param"], s["master"])
    if s["bits"] == 8:
        for name, x, is_root in (("m", flat_m, False), ("r", torch.sqrt(flat_v), True)):
            code, exp = _to_codes(x, is_root)
            s[name + "_code"].copy_(code)
            s[name + "_exp"].copy_(exp)


def _adamw_state(s):
    """Everything the step wrote; moments that are held in 8 bits as the values that they stand for."""
    if s["bits"] == 32:
        m, v = s["m_flat"], s["v_flat"]
    elif own:
        m, v = s["optimizer"].moments()
    else:
        m, v = _from_codes(s["m_code"], s["m_exp"]), _from_codes(s["r_code"], s["r_exp"]).square()
    return dict(param=s["param_flat"], master=s["master_flat"], m=m, v=v)


def _run_plain(s):
    if s["op"] == "norm":
        return _norm_forward(s["x"], s["w"], s["b"]) if s["dir"] == "fwd" else _norm_backward(s["dy"], s["x"], s["w"], s["mean"], s["rstd"])
    if s["op"] == "linear":
        if s["dir"] == "fwd":
            return _linear_forward(s["x"], s["W"], s["b"], s["r"], s["act"], s["pre"])
        return _linear_backward(s["dy"], s["x"], s["W"], s["z"], s["act"], s["bias"])
    if s["op"] == "balance":
        return _balance(s["logits"], s["i"], s["m"], s["dg"], s["norm"])
    _adamw(s)
    return _adamw_state(s)


def _run_own(s):
    from paper_2603_06626_b200 import binding as B
    if s["op"] == "norm":
        if s["dir"] == "fwd":
            return B.layer_norm(s["x"], s["w"], s["b"], eps=1e-5)
        return B.layer_norm_backward(s["dy"], s["x"], s["w"], s["mean"], s["rstd"])
    if s["op"] == "linear":
        act = dict(none=B.ACT_NONE, relu=B.ACT_RELU, silu=B.ACT_SILU, gelu=B.ACT_GELU)[s["act"]]
        if s["dir"] == "fwd":
            y, z = B.linear(s["x"], s["W"], bias=s["b"], act=act, residual=s["r"], save_pre=s["pre"])
            return (y, z) if s["pre"] else y
        dx, dW, db = B.linear_backward(s["dy"], s["x"], s["W"], pre=s["z"], act=act if s["z"] is not None else B.ACT_NONE, want_bias=s["bias"])
        return (dx, dW, db) if s["bias"] else (dx, dW)
    if s["op"] == "balance":
        counts, n = B.expert_counts(s["i"], s["logits"].shape[1], mask=s["m"])
        loss, d = B.balance_loss(s["logits"], s["i"], counts, n, mask=s["m"], balance_coef=BALANCE_COEF, z_coef=Z_COEF, dgates=s["dg"],
                                 norm=B.NORM_SOFTMAX if s["norm"] == "softmax" else B.NORM_SIGMOID)
        return dict(counts=counts, tokens=n, loss=loss, dlogits=d)
    s["optimizer"].step(grad_scale=s["scale"])
    return _adamw_state(s)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["op"] == "norm":
        n, w = case["T"] * case["d"] * BYTES[case["type"]], case["d"] * BYTES[case["wtype"]]
        if case["dir"] == "fwd":
            return dict(bytes=2 * n + 2 * w + 8 * case["T"], flops=8 * case["T"] * case["d"])
        return dict(bytes=3 * n + w + 8 * case["d"] + 8 * case["T"], flops=14 * case["T"] * case["d"])
    if case["op"] == "linear":
        T, K, N = case["T"], case["K"], case["N"]
        one = 2 * T * K * N
        if case["dir"] == "fwd":
            return dict(bytes=2 * (T * K + N * K + T * N * (1 + case["residual"] + case["pre"]) + N * case["bias"]), flops=one)
        return dict(bytes=2 * (T * N * (1 + case["pre"]) + 2 * T * K + 2 * N * K) + 4 * N * case["bias"], flops=2 * one)
    if case["op"] == "balance":
        T, E, k = case["T"], case["E"], case["k"]
        row = 2 * E * BYTES[case["type"]] + k * (1 if case["idx"] == "u8" else 4) + 4 * k * case["gates"] + case["mask"]
        return dict(bytes=T * row + 8 * E, flops=12 * T * E)
    n = sum(_sizes(case))
    each = BYTES[case["grad"]] + 8 + (2 if case["param"] == "bf16" else 0) + (16 if case["bits"] == 32 else 4 + 4 / BLOCK)
    extra = 8 * n if case["bits"] == 8 else 0           # the values that the codes stand for, which this case returns
    return dict(bytes=int(n * each) + extra, flops=16 * n)


# ---------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    D = lambda t: None if t is None else t.double()  # noqa: E731
    if case["op"] == "norm":
        x, w = D(s["x"]), D(s["w"])
        d = x.shape[1]
        if case["dir"] == "fwd":
            mean = x.sum(1) / d
            rstd = ((x * x).sum(1) / d - mean * mean + 1e-5) ** -0.5
            y = torch.addcmul(D(s["b"]).expand_as(x), (x - mean.unsqueeze(1)) * rstd.unsqueeze(1), w.expand_as(x))
            return y, mean, rstd
        h, g = (x - D(s["mean"]).unsqueeze(1)) * D(s["rstd"]).unsqueeze(1), D(s["dy"])
        a = torch.einsum("td,d->t", g, w) / d
        c = torch.einsum("td,td,d->t", g, h, w) / d
        dx = D(s["rstd"]).unsqueeze(1) * (g * w - a.unsqueeze(1) - h * c.unsqueeze(1))
        return dx, torch.einsum("td,td->d", g, h), torch.einsum("td->d", g)
    if case["op"] == "linear":
        act = s["act"]

        def sig(z):
            return torch.special.expit(z)

        def inner(z):
            return 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)

        x, W = D(s["x"]), D(s["W"])
        if case["dir"] == "fwd":
            z = torch.einsum("tk,nk->tn", x, W)
            if s["b"] is not None:
                z = z + D(s["b"])
            y = dict(none=lambda: z, relu=lambda: torch.where(z > 0, z, 0 * z), silu=lambda: z * sig(z), gelu=lambda: z * sig(inner(z)))[act]()
            if s["r"] is not None:
                y = y + D(s["r"])
            return (y, z) if s["pre"] else y
        g = D(s["dy"])
        if s["z"] is not None:
            z = D(s["z"])
            slope = dict(none=lambda: 1.0, relu=lambda: (z > 0).double(), silu=lambda: sig(z) + z * sig(z) * sig(-z),
                         gelu=lambda: sig(inner(z)) + z * sig(inner(z)) * sig(-inner(z)) * 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z ** 2))
            g = g * slope[act]()
        out = (torch.einsum("tn,nk->tk", g, W), torch.einsum("tn,tk->nk", g, x))
        return out + (torch.einsum("tn->n", g),) if s["bias"] else out
    if case["op"] == "balance":
        x, i = D(s["logits"]), s["i"].long()
        T, E = x.shape
        live = torch.ones(T, dtype=torch.float64, device=x.device) if s["m"] is None else (s["m"] > 0).double()
        counts = torch.bincount(i.reshape(-1), weights=live.repeat_interleave(i.shape[1]), minlength=E)
        n, total = max(1.0, float(live.sum())), max(1.0, float(counts.sum()))
        lse = torch.logsumexp(x, 1)
        p = torch.softmax(x, 1)
        f = counts * E / total
        mean_p = torch.einsum("te,t->e", p, live) / n
        balance, z = (f * mean_p).sum(), (lse ** 2 * live).sum() / n
        # through dL/dp and dL/dlse
        up = BALANCE_COEF * f / n
        d = p * (up - (p @ up).unsqueeze(1)) + (2 * Z_COEF / n) * lse.unsqueeze(1) * p
        if s["dg"] is not None:
            q, dg = x.gather(1, i), D(s["dg"])
            if s["norm"] == "softmax":
                q = torch.softmax(q, 1)
                back = q * dg - q * torch.einsum("tk,tk->t", q, dg).unsqueeze(1)
            else:
                back = torch.special.expit(q) * torch.special.expit(-q) * dg
            d = d.scatter_add(1, i, back)
        loss = torch.stack([BALANCE_COEF * balance + Z_COEF * z, balance, z])
        return dict(counts=None, tokens=None, loss=loss, dlogits=d * live.unsqueeze(1))
    # AdamW; what is kept in 8 bits has no value of its own in 64 bits: the codes are compared with the plain form's
    lr, b1, b2, eps = HYPER["lr"], HYPER["beta1"], HYPER["beta2"], HYPER["eps"]
    t = s["t"] + 1
    at, total = _spread(_sizes(case))
    g, wd = (torch.zeros(total, dtype=torch.float64, device=DEVICE) for _ in range(2))
    for a, x, w in zip(at, s["grads"], s["decay"]):
        g[a:a + x.numel()] = x.double() * float(s["scale"])
        wd[a:a + x.numel()] = w
    if case["bits"] == 32:
        m, v = D(s["m_flat"]), D(s["v_flat"])
    else:
        m, v = D(_from_codes(s["m_code"], s["m_exp"])), D(_from_codes(s["r_code"], s["r_exp"])) ** 2
    m = m + (1 - b1) * (g - m)
    v = v + (1 - b2) * (g * g - v)
    p = D(s["master_flat"]) * (1 - lr * wd) - lr * (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)) ** 0.5 + eps)
    return dict(param=p, master=p, m=m, v=v) if case["bits"] == 32 else dict(param=p, master=p, m=None, v=None)
