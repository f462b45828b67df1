"""A dense block of a routed model (its first layers, or a branch that every token takes), trained in bf16 and served in 8 bits, and a
projection trained in 8 bits: the operators of the dense gated branch as they are used together.

    h   = x + r                              the residual stream, and what the layer before adds to it
    out = h + ffn(rms_norm(h)),              ffn(y) = (silu(y W_g^T) * (y W_u^T)) W_d^T
    z   = out W^T                            the projection, both operands in 8 bits

    python -m paper_2603_06626_b200.dense --steps 20 --state-bits 8
"""
from __future__ import annotations

import argparse
from typing import Optional

import torch

from . import binding as B


def _sizes(**sizes: int) -> None:
    for name, size in sizes.items():
        if size < 1 or size % 16:
            raise ValueError(f"{name}: a multiple of 16 is expected, got {size}")


class DenseBlock:
    """Weights, gradients and optimizer of one block of width d; d and hidden are multiples of 16 (rows of codes are)."""

    def __init__(self, d: int, hidden: int, device: str = "cuda:0", seed: int = 0, lr: float = 1e-3, weight_decay: float = 0.01, state_bits: int = 32,
                 eps: float = 1e-6):
        _sizes(d=d, hidden=hidden)
        self.d, self.hidden, self.eps = d, hidden, eps
        g = torch.Generator(device=device).manual_seed(seed)

        def normal(*shape, std):
            return torch.empty(shape, device=device).normal_(0.0, std, generator=g).bfloat16()

        bf, f32 = torch.bfloat16, torch.float32
        # name: (weight, type its gradient arrives in, whether it decays)
        made = {"norm_w": (torch.ones(d, dtype=bf, device=device), f32, False), "W_gu": (normal(2 * hidden, d, std=d ** -0.5), bf, True),
                "W_d": (normal(d, hidden, std=hidden ** -0.5), bf, True)}
        self.w = {n: w for n, (w, _, _) in made.items()}
        self.grad = {n: torch.zeros(w.shape, dtype=gt, device=device) for n, (w, gt, _) in made.items()}
        self.status = torch.zeros(1, dtype=torch.int32, device=device)      # what the block's own calls find
        self.optimizer = B.AdamW(self.w.values(), self.grad.values(), lr=lr, betas=(0.9, 0.95), state_bits=state_bits,
                                 weight_decay=[weight_decay if decays else 0.0 for _, _, decays in made.values()])

    def _check(self, name: str, t: torch.Tensor) -> None:
        B._expect(name, t, (t.shape[0] if t.dim() else 0, self.d), torch.bfloat16, like=self.status)

    def forward(self, x: torch.Tensor, r: Optional[torch.Tensor] = None) -> torch.Tensor:
        """x, r [T,d] bf16 -> out [T,d]: the residual stream behind the block."""
        self._check("x", x)
        w = self.w
        y, h, rstd = B.rms_norm(x, w["norm_w"], residual=r, eps=self.eps)
        out, pre = B.gated_ffn(y, w["W_gu"], w["W_d"], residual=h, save_pre=True, status=self.status)
        self._saved = (y, h, rstd, pre)
        return out

    def backward(self, dout: torch.Tensor) -> torch.Tensor:
        """dout [T,d] bf16 -> the gradient of x, which is that of r too; the weights' gradients go to self.grad."""
        self._check("dout", dout)
        y, h, rstd, pre = self._saved
        w, g = self.w, self.grad
        dy, _, _ = B.gated_ffn_backward(dout, y, w["W_gu"], w["W_d"], pre, dW_gu=g["W_gu"], dW_d=g["W_d"], status=self.status)
        dx, _ = B.rms_norm_backward(dy, h, w["norm_w"], rstd, dh=dout, dw=g["norm_w"])
        return dx

    def step(self, grad_scale: Optional[torch.Tensor] = None) -> None:
        self.optimizer.step(grad_scale=grad_scale)

    def served(self) -> "ServedBlock":
        """The block as it is now, its weights in 8 bits."""
        return ServedBlock(self)

    def check_status(self) -> None:
        """Raises on what this block's kernels found since the last check."""
        B.check_status(status=self.status)


class ServedBlock:
    """A DenseBlock's forward pass in 8 bits: the norm's output, the weights and the hidden state are codes with scales."""

    def __init__(self, block: DenseBlock):
        H = block.hidden
        self.d, self.eps, self.status = block.d, block.eps, torch.zeros_like(block.status)
        self.norm_w = block.w["norm_w"].clone()
        self.W_g, self.W_u, self.W_d = (B.quantize_fp8(W, square=True)[0] for W in (block.w["W_gu"][:H], block.w["W_gu"][H:], block.w["W_d"]))

    def forward(self, x: torch.Tensor, r: Optional[torch.Tensor] = None) -> torch.Tensor:
        y, h, _ = B.rms_norm(x, self.norm_w, residual=r, eps=self.eps, fp8=True)
        return B.gated_ffn_fp8(y, self.W_g, self.W_u, self.W_d, residual=h if h.is_contiguous() else h.contiguous(), status=self.status)

    def check_status(self) -> None:
        B.check_status(status=self.status)


class Projection8:
    """z = x W^T with both operands in 8 bits, in the backward pass too.  The weight itself stays bf16 with an f32 master copy and is put into
    8 bits in every step; d and n are multiples of 16."""

    def __init__(self, d: int, n: int, device: str = "cuda:0", seed: int = 0, lr: float = 1e-3, weight_decay: float = 0.01, state_bits: int = 32):
        _sizes(d=d, n=n)
        g = torch.Generator(device=device).manual_seed(seed)
        self.W = torch.empty(n, d, device=device).normal_(0.0, d ** -0.5, generator=g).bfloat16()
        self.grad = torch.zeros_like(self.W)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.optimizer = B.AdamW([self.W], [self.grad], lr=lr, betas=(0.9, 0.95), state_bits=state_bits, weight_decay=weight_decay)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        """x [T,d] bf16 -> z [T,n]."""
        B._expect("x", x, (x.shape[0] if x.dim() else 0, self.W.shape[1]), torch.bfloat16, like=self.W)
        W8, Wt = B.quantize_fp8(self.W, square=True, transposed=True)
        x8, xt = B.quantize_fp8(x, transposed=True)
        self._saved = (xt, Wt)
        return B.linear_fp8(x8, W8, status=self.status)

    def backward(self, dz: torch.Tensor) -> torch.Tensor:
        """dz [T,n] bf16 -> dx [T,d]; the weight's gradient goes to self.grad."""
        xt, Wt = self._saved
        return B.linear_fp8_backward(dz, xt, Wt, dW=self.grad, status=self.status)[0]

    def step(self, grad_scale: Optional[torch.Tensor] = None) -> None:
        self.optimizer.step(grad_scale=grad_scale)

    def check_status(self) -> None:
        B.check_status(status=self.status)


def main() -> None:
    ap = argparse.ArgumentParser(description="Trains a dense block and a projection in 8 bits to follow a fixed random map, then serves the block in 8 bits.")
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--state-bits", type=int, choices=(8, 32), default=32)
    a = ap.parse_args()
    T, d, n = 1024, 256, 128
    block = DenseBlock(d, hidden=512, lr=3e-3, state_bits=a.state_bits)
    head = Projection8(d, n, lr=3e-3, state_bits=a.state_bits)
    g = torch.Generator(device="cuda:0").manual_seed(1)
    target = torch.empty(d, n, device="cuda:0").normal_(0, d ** -0.5, generator=g)
    x = torch.empty(T, d, device="cuda:0").normal_(generator=g).bfloat16()
    for i in range(a.steps):
        diff = head.forward(block.forward(x)).float() - torch.tanh(x.float() @ target)
        block.backward(head.backward((2.0 / T * diff).bfloat16()))
        block.step()
        head.step()
        if i % 5 == 0 or i == a.steps - 1:
            block.check_status()
            head.check_status()
            print(f"step {i:3d}  error {diff.square().mean().item():.4f}")
    served = block.served()
    want, got = block.forward(x).float(), served.forward(x).float()
    served.check_status()
    print(f"served in 8 bits: off by {((got - want).norm() / (want - x.float()).norm()).item():.4f} of what the block adds")


if __name__ == "__main__":
    main()
