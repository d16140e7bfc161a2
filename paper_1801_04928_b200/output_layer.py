"""An output layer in 8 bits that learns from a teacher's top logits.

    u = layer_norm(x + r),  z = u w^T,  loss = sum_t weight_t T^2 KL(softmax(teacher's entries / T) || softmax(z / T))

Every product is one of 8-bit operands with a scale for each block of 128: the norm hands over its result in that form, the
weights are laid out when they change, as they lie and transposed, and the gradient of the logits is packed both ways.  The
loss and its gradient are one call, in place: dz takes the place of z.

    python -m paper_1801_04928_b200.output_layer [--tokens 2048 --width 1024 --vocab 32000 --top 32 --steps 30]

trains one layer on another's largest logits for synthetic tokens and then runs single tokens through it.
"""
from __future__ import annotations

import argparse
import time

import torch

import paper_1801_04928_b200 as lf


def blocks(n: int) -> int:
    return (n + 127) // 128


class OutputLayer:
    """Weights, gradients and the buffers of one layer for at most `tokens` tokens.  `width` and `vocab`: multiples of 8."""

    def __init__(self, ops, tokens: int, width: int, vocab: int, dtype=torch.bfloat16, device="cuda", seed: int = 0):
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def new(*shape, dt=dtype):
            return torch.empty(shape, dtype=dt, device=device)

        def packed(rows, n):                                 # e4m3 rows begin on 16-byte boundaries
            return new(rows, (n + 15) // 16 * 16, dt=torch.uint8)[:, :n]

        f32 = torch.float32
        self.ops, self.dtype, self.width, self.vocab = ops, dtype, width, vocab
        self.master = {"w": new(vocab, width, dt=f32).normal_(0, width ** -0.5, generator=g),
                       "gain": torch.ones(width, device=device), "shift": torch.zeros(width, device=device)}
        self.grad = {k: torch.empty_like(v) for k, v in self.master.items()}
        self.w = dict(q=packed(vocab, width), s=new(blocks(vocab), blocks(width), dt=f32),
                      qt=packed(width, vocab), st=new(blocks(width), blocks(vocab), dt=f32))
        self.refresh()
        # what the forward pass keeps: h, its statistics and u
        self.h, self.u, self.du = new(tokens, width), new(tokens, width), new(tokens, width)
        self.mean, self.rstd = new(tokens, dt=f32), new(tokens, dt=f32)
        self._packed, self._scales = packed, lambda *shape: new(*shape, dt=f32)
        self._forms = {}

    def refresh(self):
        self.ops.pack_tiles(self.master["w"], **self.w)

    def forms(self, m: int):
        """8-bit buffers for m tokens (scales are [blocks, m], so they go by the number)."""
        if m not in self._forms:
            p, s, n, v = self._packed, self._scales, self.width, self.vocab
            self._forms[m] = dict(u=dict(q=p(m, n), s=s(blocks(n), m), qt=p(n, m), st=s(blocks(m), n)),
                                  dz=dict(q=p(m, v), s=s(blocks(v), m), qt=p(v, m), st=s(blocks(m), v)))
        return self._forms[m]

    def forward(self, x, r, z, keep: bool = True):
        """z = layer(x + r); with `keep` also what backward() reads."""
        m, p = x.shape[0], self.master
        u8 = self.forms(m)["u"]
        if keep:
            self.ops.layer_norm(x, p["gain"], p["shift"], self.u[:m], residual=r, h=self.h[:m], q=u8["q"], s=u8["s"], mean=self.mean[:m], rstd=self.rstd[:m])
        else:
            self.ops.layer_norm(x, p["gain"], p["shift"], residual=r, q=u8["q"], s=u8["s"])
        self.ops.product_blocks(u8["q"], u8["s"], self.w["q"], self.w["s"], z)

    def backward(self, z, index, value, loss, dh, weight=None, temperature: float = 1.0):
        """loss [tokens], the gradients of all parameters (self.grad) and dh, from the logits of the last forward pass,
        which the gradient of the losses' sum with respect to them replaces."""
        m, g = z.shape[0], self.grad
        f = self.forms(m)
        self.ops.distill(z, index, value, loss, weight=weight, dz=z, temperature=temperature)
        self.ops.pack_blocks(z, **f["dz"])
        self.ops.pack_blocks(self.u[:m], qt=f["u"]["qt"], st=f["u"]["st"])
        self.ops.product_blocks(f["dz"]["qt"], f["dz"]["st"], f["u"]["qt"], f["u"]["st"], g["w"])
        self.ops.product_blocks(f["dz"]["q"], f["dz"]["s"], self.w["qt"], self.w["st"], self.du[:m])
        self.ops.layer_norm_backward(self.du[:m], self.h[:m], self.master["gain"], self.mean[:m], self.rstd[:m], dh, g["gain"], g["shift"])

    def step(self, rate: float):
        for k, v in self.master.items():
            v.add_(self.grad[k], alpha=-rate)
        self.refresh()


def train(tokens: int, width: int, vocab: int, top: int, steps: int, rate: float = 1.0, temperature: float = 2.0, seed: int = 0):
    """Mean losses of `steps` steps that fit one layer to the `top` largest logits of another."""
    stream = torch.cuda.current_stream().cuda_stream
    ops = lf.Operators(stream=stream)
    teacher, layer = (OutputLayer(ops, tokens, width, vocab, seed=seed + i) for i in (1, 2))
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x, r = (torch.empty(tokens, width, device="cuda").normal_(0, 1, generator=g).to(torch.bfloat16) for _ in range(2))
    z, dh, loss = torch.empty(tokens, vocab, dtype=torch.bfloat16, device="cuda"), torch.empty_like(x), torch.empty(tokens, device="cuda")
    teacher.forward(x, r, z, keep=False)
    value, index = z.float().topk(top, 1)
    index = index.int()
    weight = torch.full((tokens,), 1.0 / tokens, device="cuda")
    losses = []
    for _ in range(steps):
        layer.forward(x, r, z)
        layer.backward(z, index, value, loss, dh, weight=weight, temperature=temperature)
        losses.append(loss.sum())
        layer.step(rate)
    ops.sync()
    return [v.item() for v in losses], layer, ops, x, r


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--vocab", type=int, default=32000)
    ap.add_argument("--top", type=int, default=32)
    ap.add_argument("--steps", type=int, default=30)
    a = ap.parse_args()
    torch.cuda.synchronize()
    t = time.perf_counter()
    losses, layer, ops, x, r = train(a.tokens, a.width, a.vocab, a.top, a.steps)
    t = time.perf_counter() - t
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f} in {a.steps} steps, {1e3 * t / a.steps:.2f} ms a step with set-up")
    one, res, out = x[:1], r[:1], torch.empty(1, a.vocab, dtype=x.dtype, device=x.device)
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    for _ in range(3):
        layer.forward(one, res, out, keep=False)
    start.record()
    for _ in range(100):
        layer.forward(one, res, out, keep=False)
    end.record()
    ops.sync()
    print(f"logits of one token: {10 * start.elapsed_time(end):.1f} us")


if __name__ == "__main__":
    main()
