"""A residual block trained in low precision, with the library's operators from end to end.

    s = x + r                  y = rmsnorm(s) g           (8-bit rows with a scale per 32 columns)
    z = relu(y W1^T)           out = s + z W2^T           (weights in 4 bits, activations in 8)
    loss = mean over rows of |out - t|^2 / 2

Backward the same products run on transposed quantisations, the norm has its own kernel, and AdamW updates the fp32 weights of
all tensors at once, clipped by the global norm, with moments in 8 or 32 bits.  The data are a teacher block's outputs.

    python -m paper_2003_10579_amd.lowbit_block [--steps N] [--rows T] [--width D] [--hidden H] [--state-bits 8|32]
"""
from __future__ import annotations

import argparse
import math
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


class Block:
    def __init__(self, width, hidden, state_bits=8, seed=0, device="cuda"):
        import torch
        from paper_2003_10579_amd import ssgd
        g = torch.Generator(device=device).manual_seed(seed)
        self.gain = torch.ones(width, device=device)
        self.w1 = torch.randn(hidden, width, generator=g, device=device) / math.sqrt(width)
        self.w2 = torch.randn(width, hidden, generator=g, device=device) / math.sqrt(hidden)
        self.optimizer = ssgd.AdamW([self.gain, self.w1, self.w2], weight_decay=[0.0, 0.01, 0.01], max_norm=1.0, state_bits=state_bits, seed=seed)

    def quantize_weights(self):
        """What the products take: each weight along its rows (forward) and its columns (backward)."""
        from paper_2003_10579_amd import ssgd
        self.q1, self.q1t = ssgd.mx_quantize_both(self.w1, "fp4", "fp4")
        self.q2, self.q2t = ssgd.mx_quantize_both(self.w2, "fp4", "fp4")

    def forward(self, x, r):
        from paper_2003_10579_amd import ssgd
        y, s, rstd = ssgd.rmsnorm(x, self.gain, residual=r, output="fp8")
        z = ssgd.mx_matmul(y, self.q1).relu_()
        return s + ssgd.mx_linear(z, self.q2, "fp8"), (y, s, rstd, z)

    def step(self, x, r, target, lr):
        """One update; the loss before it."""
        import torch
        from paper_2003_10579_amd import ssgd
        self.quantize_weights()
        out, (y, s, rstd, z) = self.forward(x, r)
        rows = x.shape[0]
        off = out.float() - target
        loss = off.square().sum() / (2 * rows)
        dout = (off / rows).to(torch.bfloat16)
        dq, dt = ssgd.mx_quantize_both(dout, "fp8", "fp8")
        dw2 = ssgd.mx_matmul(dt, ssgd.mx_quantize_transposed(z, "fp4"), torch.float32)
        dz = ssgd.mx_matmul(dq, self.q2t) * (z > 0)
        dq, dt = ssgd.mx_quantize_both(dz, "fp8", "fp8")
        # (the activations that the product took: what it used of them in 8 bits is what the weight's gradient is of.  As the right operand they are
        # rounded once more, to 4 bits)
        dw1 = ssgd.mx_matmul(dt, ssgd.mx_quantize_transposed(ssgd.mx_dequantize(y, torch.bfloat16), "fp4"), torch.float32)
        dx, dgain = ssgd.rmsnorm_backward(ssgd.mx_matmul(dq, self.q1t), s, self.gain, rstd, dsum=dout)
        self.optimizer.step([dgain, dw1, dw2], lr)
        return loss, dx          # dx: what a block before this one would get

    def answer(self, x, r):
        """The block's output for rows of a running program, a single one for instance."""
        return self.forward(x, r)[0]


def train(steps=60, rows=4096, width=512, hidden=1024, state_bits=8, lr=3e-3, seed=0, every=10, report=print):
    import torch
    teacher = Block(width, hidden, seed=seed + 1)
    teacher.quantize_weights()
    block = Block(width, hidden, state_bits, seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 2)
    losses = []
    for k in range(steps):
        x = torch.randn(rows, width, generator=g, device="cuda").to(torch.bfloat16)
        r = torch.randn(rows, width, generator=g, device="cuda").to(torch.bfloat16)
        loss, _ = block.step(x, r, teacher.answer(x, r).float(), lr)
        losses.append(loss)
        if report and k % every == 0:
            report(f"step {k:4d}  loss {float(loss):.4f}  gradient norm {float(block.optimizer.grad_norm):.3f}")
    return block, [float(v) for v in losses]


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--rows", type=int, default=4096)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--state-bits", type=int, choices=(8, 32), default=8)
    args = ap.parse_args()
    _, losses = train(args.steps, args.rows, args.width, args.hidden, args.state_bits)
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}")


if __name__ == "__main__":
    main()
