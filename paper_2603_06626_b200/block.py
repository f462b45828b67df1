"""A block around the routed expert layer, trained end to end: the operators of this package as they are used together.

    h   = layer_norm(x)
    s   = h W_s^T            scores of the router; k of them kept, gates = softmax over the kept ones      (grouter_route)
    out = x + experts(h; gates) + dense(h),      dense(h) = silu(h W_1^T + b_1) W_2^T + b_2
    loss = <upstream loss of out> + balance_coef * balance loss of s + z_coef * z loss of s

The router is trained here: the gradient of its gates (the layer's dgates) and of the two losses meet in the scores' gradient,
which the linear layer's backward pass takes on to W_s and h.  One AdamW object updates every tensor in one launch.

    python -m paper_2603_06626_b200.block --steps 20 --state-bits 8
"""
from __future__ import annotations

import argparse
from typing import Optional

import torch

from . import binding as B


class RoutedBlock:
    """Weights, gradients and optimizer of one block for batches of T tokens.  T, d, ffn, E and hidden are multiples of 8: the router
    head and the products work in units of 8 of each."""

    def __init__(self, T: int, d: int, ffn: int, E: int, k: int, hidden: int, device: str = "cuda:0", seed: int = 0, lr: float = 1e-3,
                 weight_decay: float = 0.01, state_bits: int = 32, balance_coef: float = 1e-2, z_coef: float = 1e-3):
        for name, size in (("T", T), ("d", d), ("ffn", ffn), ("E", E), ("hidden", hidden)):
            if size < 1 or size % 8:
                raise ValueError(f"{name}: a multiple of 8 is expected, got {size}")
        self.T, self.d, self.E, self.k = T, d, E, k
        self.balance_coef, self.z_coef = balance_coef, z_coef
        self.layer = B.GrouterLayer(T, d, ffn, E, k, device=device)
        g = torch.Generator(device=device).manual_seed(seed)

        def normal(*shape, std):
            return torch.empty(shape, device=device).normal_(0.0, std, generator=g).bfloat16()

        bf, f32 = torch.bfloat16, torch.float32
        # name: (weight, type its gradient arrives in, whether it decays)
        made = {"norm_w": (torch.ones(d, dtype=bf, device=device), f32, False), "norm_b": (torch.zeros(d, dtype=bf, device=device), f32, False),
                "W_s": (normal(E, d, std=d ** -0.5), f32, True),
                "W_gu": (normal(E, 2 * ffn, d, std=d ** -0.5), f32, True), "W_d": (normal(E, d, ffn, std=ffn ** -0.5), f32, True),
                "W_1": (normal(hidden, d, std=d ** -0.5), bf, True), "b_1": (torch.zeros(hidden, dtype=bf, device=device), f32, False),
                "W_2": (normal(d, hidden, std=hidden ** -0.5), bf, True), "b_2": (torch.zeros(d, dtype=bf, device=device), f32, False)}
        self.w = {n: w for n, (w, _, _) in made.items()}
        self.grad = {n: torch.zeros(w.shape, dtype=gt, device=device) for n, (w, gt, _) in made.items()}
        # what the block's own calls find; the word that other calls on the device share is not touched
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.optimizer = B.AdamW(self.w.values(), self.grad.values(), lr=lr, betas=(0.9, 0.95), state_bits=state_bits,
                                 weight_decay=[weight_decay if decays else 0.0 for _, _, decays in made.values()])

    def forward(self, x: torch.Tensor, mask: Optional[torch.Tensor] = None):
        """x [T,d] bf16; mask [T] (zero: padding, left out of the losses and the router's gradient) -> (out [T,d], losses f32 [3])."""
        B._expect("x", x, (self.T, self.d), torch.bfloat16, like=self.status)
        w = self.w
        h, mean, rstd = B.layer_norm(x, w["norm_w"], w["norm_b"])
        idx, gates, scores = B.route(h, w["W_s"], None, self.E, self.k, want_scores=True)
        counts, n = B.expert_counts(idx, self.E, mask=mask, status=self.status)
        losses, _ = B.balance_loss(scores, idx, counts, n, mask=mask, balance_coef=self.balance_coef, z_coef=self.z_coef, want_grad=False,
                                   status=self.status)
        self.layer.plan(idx)
        routed = self.layer.forward(h, gates, w["W_gu"], w["W_d"])
        u, pre = B.linear(h, w["W_1"], bias=w["b_1"], act=B.ACT_SILU, save_pre=True, status=self.status)
        out, _ = B.linear(u, w["W_2"], bias=w["b_2"], residual=x, status=self.status)
        out += routed
        self._saved = (x, mask, h, mean, rstd, idx, gates, scores, counts, n, u, pre)
        return out, losses

    def backward(self, dout: torch.Tensor):
        """dout [T,d] bf16: gradient of the upstream loss -> dx [T,d] bf16; the weights' gradients go to self.grad."""
        B._expect("dout", dout, (self.T, self.d), torch.bfloat16, like=self.status)
        x, mask, h, mean, rstd, idx, gates, scores, counts, n, u, pre = self._saved
        w, g = self.w, self.grad
        dh, _, _, dgates = self.layer.backward(dout, h, gates, w["W_gu"], w["W_d"], dW_gu=g["W_gu"], dW_d=g["W_d"])
        du, _, _ = B.linear_backward(dout, u, w["W_2"], dW=g["W_2"], db=g["b_2"], status=self.status)
        dh_dense, _, _ = B.linear_backward(du, h, w["W_1"], pre=pre, act=B.ACT_SILU, dW=g["W_1"], db=g["b_1"], status=self.status)
        _, dscores = B.balance_loss(scores, idx, counts, n, mask=mask, balance_coef=self.balance_coef, z_coef=self.z_coef, dgates=dgates,
                                    want_loss=False, status=self.status)
        dh_router, _, _ = B.linear_backward(dscores.bfloat16(), h, w["W_s"], dW=g["W_s"], status=self.status)
        dh += dh_dense
        dh += dh_router
        dx, _, _ = B.layer_norm_backward(dh, x, w["norm_w"], mean, rstd, dw=g["norm_w"], db=g["norm_b"])
        dx += dout
        return dx

    def step(self, grad_scale: Optional[torch.Tensor] = None) -> None:
        self.optimizer.step(grad_scale=grad_scale)

    def check_status(self) -> None:
        """Raises on what this block's kernels found since the last check."""
        self.layer.check_status()
        B.check_status(status=self.status)


def main() -> None:
    ap = argparse.ArgumentParser(description="Trains one block to follow a fixed random map of its input.")
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--state-bits", type=int, choices=(8, 32), default=32)
    a = ap.parse_args()
    T, d = 1024, 256
    block = RoutedBlock(T, d, ffn=256, E=16, k=2, hidden=512, lr=3e-3, state_bits=a.state_bits)
    g = torch.Generator(device="cuda:0").manual_seed(1)
    target = torch.empty(d, d, device="cuda:0").normal_(0, d ** -0.5, generator=g)
    for i in range(a.steps):
        x = torch.empty(T, d, device="cuda:0").normal_(generator=g).bfloat16()
        want = x.float() + torch.tanh(x.float() @ target)
        out, losses = block.forward(x)
        diff = out.float() - want
        block.backward((2.0 / T * diff).bfloat16())
        block.step()
        if i % 5 == 0 or i == a.steps - 1:
            block.check_status()
            print(f"step {i:3d}  error {diff.square().mean().item():.4f}  balance {losses[1].item():.3f}  z {losses[2].item():.3f}")


if __name__ == "__main__":
    main()
