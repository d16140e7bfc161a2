"""A residual feed-forward block trained and served with the layer operators.

    u = rms_norm(x),  a = gelu(u w1^T + b1),  y = a w2^T + b2 + x

What the forward pass keeps for the backward pass is x, which the residual stream holds anyway, and two
8-bit checkpoints: of u (the input of w1) and of the pre-activation z of the hidden layer, from which both
the input of w2 and gelu' are taken -- 2 1/16 bytes for every hidden unit and column together, where bf16
copies of u, z and a would be 6.

    python -m paper_1801_04928_b200.feed_forward [--tokens 4096 --width 1024 --hidden 4096 --steps 30]

trains one block to reproduce another on synthetic tokens and then runs single tokens through it.
"""
from __future__ import annotations

import argparse
import time

import torch

import paper_1801_04928_b200 as lf


class FeedForwardBlock:
    """Weights, gradients and the buffers of one block for at most `tokens` tokens."""

    def __init__(self, ops, tokens: int, width: int, hidden: int, dtype=torch.bfloat16, device="cuda", seed: int = 0):
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def new(*shape, dt=dtype):
            return torch.empty(shape, dtype=dt, device=device)

        self.ops, self.dtype = ops, dtype
        # fp32 master weights; the 16-bit copies that the products read follow them
        self.master = {"w1": new(hidden, width, dt=torch.float32).normal_(0, width ** -0.5, generator=g),
                       "w2": new(width, hidden, dt=torch.float32).normal_(0, hidden ** -0.5, generator=g),
                       "b1": torch.zeros(hidden, device=device), "b2": torch.zeros(width, device=device),
                       "gain": torch.ones(width, device=device)}
        self.w1, self.w2 = new(hidden, width), new(width, hidden)
        self.grad = {k: torch.empty_like(v) for k, v in self.master.items()}
        self._refresh()
        groups = lambda n: (n + 31) // 32   # noqa: E731
        byte = torch.uint8
        self.u, self.a = new(tokens, width), new(tokens, hidden)
        self.u8 = new(tokens, width, dt=byte), new(tokens, groups(width), dt=byte)
        self.z8 = new(tokens, hidden, dt=byte), new(tokens, groups(hidden), dt=byte)
        self.dz, self.du = new(tokens, hidden), new(tokens, width)

    def _refresh(self):
        self.w1.copy_(self.master["w1"])
        self.w2.copy_(self.master["w2"])

    def forward(self, x, y, keep: bool = True):
        """y = block(x); with `keep` also the two checkpoints that backward() reads."""
        m, p = x.shape[0], self.master
        u8 = [t[:m] for t in self.u8] if keep else (None, None)
        z8 = [t[:m] for t in self.z8] if keep else (None, None)
        self.ops.rms_norm(x, p["gain"], self.u[:m], q=u8[0], s=u8[1])
        self.ops.linear(self.u[:m], self.w1, self.a[:m], bias=p["b1"], act=lf.LF_ACT_GELU, q=z8[0], s=z8[1])
        self.ops.linear(self.a[:m], self.w2, y, bias=p["b2"], residual=x)

    def backward(self, x, dy, dx):
        """Gradients of all parameters (self.grad) and dx, from dy and the checkpoints of the last forward pass."""
        m, g, gelu = x.shape[0], self.grad, lf.LF_ACT_GELU
        (uq, us), (zq, zs) = [[t[:m] for t in c] for c in (self.u8, self.z8)]
        self.ops.linear_grad_w(dy, g["w2"], gb=g["b2"], q=zq, s=zs, act=gelu)
        self.ops.linear_grad_x(dy, self.w2, self.dz[:m], q=zq, s=zs, act=gelu)
        self.ops.linear_grad_w(self.dz[:m], g["w1"], gb=g["b1"], q=uq, s=us)
        self.ops.linear_grad_x(self.dz[:m], self.w1, self.du[:m])
        self.ops.rms_norm_backward(self.du[:m], x, self.master["gain"], dx, g["gain"], dres=dy)

    def step(self, rate: float):
        for k, v in self.master.items():
            v.add_(self.grad[k], alpha=-rate)
        self._refresh()


def train(tokens: int, width: int, hidden: int, steps: int, rate: float | None = None, seed: int = 0):
    """Losses of `steps` steps that fit one block to another's outputs.  The loss's curvature along w2 grows
    with the number of hidden units: by default the rate is 10 over it."""
    rate = 10.0 / hidden if rate is None else rate
    stream = torch.cuda.current_stream().cuda_stream
    ops = lf.Operators(lf.lf_ops_workspace(tokens, max(width, hidden)), stream=stream)
    teacher, block = (FeedForwardBlock(ops, tokens, width, hidden, seed=seed + i) for i in (1, 2))
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.empty(tokens, width, device="cuda").normal_(0, 1, generator=g).to(torch.bfloat16)
    target, y, dy, dx = (torch.empty_like(x) for _ in range(4))
    teacher.forward(x, target, keep=False)
    losses = []
    for _ in range(steps):
        block.forward(x, y)
        d = y.float() - target.float()
        losses.append(0.5 * d.square().sum(1).mean())
        dy.copy_(d / tokens)
        block.backward(x, dy, dx)
        block.step(rate)
    ops.sync()
    return [v.item() for v in losses], block, ops, x


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--steps", type=int, default=30)
    a = ap.parse_args()
    torch.cuda.synchronize()
    t = time.perf_counter()
    losses, block, ops, x = train(a.tokens, a.width, a.hidden, a.steps)
    t = time.perf_counter() - t
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f} in {a.steps} steps, {1e3 * t / a.steps:.2f} ms a step with set-up")
    kept = sum(c.numel() for c in (*block.u8, *block.z8))
    print(f"kept for the backward pass: {kept / 2 ** 20:.1f} MiB in 8 bits, {2 * (block.u.numel() + 2 * block.a.numel()) / 2 ** 20:.1f} MiB in 16")
    one, out = x[:1], torch.empty_like(x[:1])
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    for _ in range(3):
        block.forward(one, out, keep=False)
    start.record()
    for _ in range(100):
        block.forward(one, out, keep=False)
    end.record()
    ops.sync()
    print(f"one token: {10 * start.elapsed_time(end):.1f} us")


if __name__ == "__main__":
    main()
