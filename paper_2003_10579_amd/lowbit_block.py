"""A residual block trained in low precision, with the library's operators from end to end.

    s = x + r                  y = rmsnorm(s) g           (8-bit rows with a scale per 32 columns)
    z = relu(y W1^T)           out = s + z W2^T           (weights in 4 bits, activations in 8)
    loss = mean over rows of |out - t|^2 / 2

Backward the same products run on transposed quantisations, the norm has its own kernel, and AdamW updates the fp32 weights of
all tensors at once, clipped by the global norm, with moments in 8 or 32 bits.  The data are a teacher block's outputs.

With --gated N it is N gated feed-forward blocks in a row, of

    y = norm(s) w_in     p = y W_up^T     h = silu(p_even) p_odd     o = h W_down^T + b     s <- s + gate (norm(o) w_out)

where everything between two products is one operator: the gate and the activation in the first product's epilogue, the bias in the second's, both norms with the gate
and the residual in one pass.  The backward pass has y, p and h from checkpoints in 8 bits.

    python -m paper_2003_10579_amd.lowbit_block [--steps N] [--rows T] [--width D] [--hidden H] [--state-bits 8|32] [--gated N]
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


class GatedBlocks:
    """Gated feed-forward blocks on a residual stream: the first norm and the blocks, each with the norm in front of the next one."""

    def __init__(self, width, hidden, blocks=2, state_bits=8, seed=0, device="cuda"):
        import torch
        from paper_2003_10579_amd import ssgd
        g = torch.Generator(device=device).manual_seed(seed)
        normal = lambda *shape: torch.randn(shape, generator=g, device=device)  # noqa: E731
        self.blocks = blocks
        self.w_in = [torch.ones(width, device=device) for _ in range(blocks + 1)]      # the last one in front of the output
        self.w_out = [torch.ones(width, device=device) for _ in range(blocks)]
        self.gate = [1.0 + 0.2 * normal(width) for _ in range(blocks)]
        self.up = [ssgd.gate_up(normal(hidden, width), normal(hidden, width)) / math.sqrt(width) for _ in range(blocks)]
        self.down = [normal(width, hidden) / math.sqrt(hidden) for _ in range(blocks)]
        self.bias = [0.1 * normal(width) for _ in range(blocks)]
        small, large = self.w_in + self.w_out + self.gate + self.bias, self.up + self.down
        self.optimizer = ssgd.AdamW(small + large, weight_decay=[0.0] * len(small) + [0.01] * len(large), max_norm=1.0, state_bits=state_bits, seed=seed)

    def quantize_weights(self):
        from paper_2003_10579_amd import ssgd
        self.q_up = [ssgd.mx_quantize_both(w, "fp4", "fp4") for w in self.up]
        self.q_down = [ssgd.mx_quantize_both(w, "fp4", "fp4") for w in self.down]

    def forward(self, x, keep=None):
        """The output and, with keep="fp8", what the backward pass takes of every block."""
        from paper_2003_10579_amd import ssgd
        y, s, rstd = ssgd.rmsnorm(x, self.w_in[0], output="fp8")
        first, kept = rstd, []
        for k in range(self.blocks):
            h = ssgd.mx_gated(y, self.q_up[k][0], "silu", output="fp8", keep=keep)
            h, p = h if keep else (h, None)
            o = ssgd.mx_dense(h, self.q_down[k][0], bias=self.bias[k])
            after = ssgd.block_norm(o, s, self.w_out[k], self.w_in[k + 1], gate=self.gate[k], output="fp8" if k + 1 < self.blocks else None)
            kept.append((y, p, o, after))
            y, s = after[:2]
        return y, first, kept

    def answer(self, x):
        return self.forward(x)[0]

    def backward(self, dy, x, first, kept):
        """(dx, the gradients in the optimizer's order) from the gradient of the output."""
        import torch
        from paper_2003_10579_amd import ssgd
        n = self.blocks
        w_in, w_out, gate, up, down, bias = [None] * (n + 1), [None] * n, [None] * n, [None] * n, [None] * n, [None] * n
        ds = None
        for k in reversed(range(n)):
            y, p, o, (_, s, rstd_o, rstd) = kept[k]
            do, ds, w_out[k], w_in[k + 1], gate[k] = ssgd.block_norm_backward(dy, o, s, self.w_out[k], self.w_in[k + 1], rstd_o, rstd, gate=self.gate[k], dsum=ds)
            d, dt, _, bias[k] = ssgd.mx_dense_backward(do, None)
            d, dp, ht = ssgd.mx_gated_backward(ssgd.mx_matmul(d, self.q_down[k][1]), p, "silu")
            down[k] = ssgd.mx_matmul(dt, ht, torch.float32)
            up[k] = ssgd.mx_matmul(dp, ssgd.mx_transpose(y), torch.float32)
            dy = ssgd.mx_matmul(d, self.q_up[k][1])
        dx, w_in[0] = ssgd.rmsnorm_backward(dy, x, self.w_in[0], first, dsum=ds)
        return dx, w_in + w_out + gate + bias + up + down

    def step(self, x, target, lr):
        """One update; the loss before it."""
        import torch
        self.quantize_weights()
        out, first, kept = self.forward(x, keep="fp8")
        off = out.float() - target
        loss = off.square().sum() / (2 * x.shape[0])
        dx, grads = self.backward((off / x.shape[0]).to(torch.bfloat16), x, first, kept)
        self.optimizer.step(grads, lr)
        return loss, dx


def train_gated(steps=60, rows=4096, width=512, hidden=1024, blocks=2, state_bits=8, lr=3e-3, seed=0, every=10, report=print):
    import torch
    teacher = GatedBlocks(width, hidden, blocks, seed=seed + 1)
    teacher.quantize_weights()
    model = GatedBlocks(width, hidden, blocks, state_bits, seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 2)
    losses = []
    for k in range(steps):
        x = torch.randn(rows, width, generator=g, device="cuda").to(torch.bfloat16)
        loss, _ = model.step(x, teacher.answer(x).float(), lr)
        losses.append(loss)
        if report and k % every == 0:
            report(f"step {k:4d}  loss {float(loss):.4f}  gradient norm {float(model.optimizer.grad_norm):.3f}")
    return model, [float(v) for v in losses]


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
    ap.add_argument("--gated", type=int, default=0, metavar="N", help="train N gated feed-forward blocks instead")
    args = ap.parse_args()
    if args.gated:
        _, losses = train_gated(args.steps, args.rows, args.width, args.hidden, args.gated, args.state_bits)
    else:
        _, losses = train(args.steps, args.rows, args.width, args.hidden, args.state_bits)
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}")


if __name__ == "__main__":
    main()
