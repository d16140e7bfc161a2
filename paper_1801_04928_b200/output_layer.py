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


def pitch(n: int) -> int:
    return (n + 15) // 16 * 16


class OutputLayer:
    """Weights, gradients and the buffers of one layer for at most `tokens` tokens.  `width` and `vocab`: multiples of 8."""

    def __init__(self, ops, tokens: int, width: int, vocab: int, dtype=torch.bfloat16, device="cuda", seed: int = 0):
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def new(*shape, dt=dtype):
            return torch.empty(shape, dtype=dt, device=device)

        def packed(rows, n):                                 # e4m3 rows begin on 16-byte boundaries
            return new(rows * pitch(n), dt=torch.uint8).view(rows, pitch(n))[:, :n]

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
        # the 8-bit forms of u and of the logits' gradient: storage for all `tokens`, which smaller batches have a part of
        self.tokens, self._new, self._storage, self._views = tokens, new, {}, {}

    def refresh(self):
        self.ops.pack_tiles(self.master["w"], **self.w)

    def _cut(self, name: str, m: int, n: int):
        """An [m, n] matrix in 8 bits, as it lies (q, s) or, where the name ends in t, transposed (qt, st), in the storage of that name."""
        turned, most = name.endswith("t"), self.tokens
        if name not in self._storage:
            self._storage[name] = (self._new(n * pitch(most) if turned else most * pitch(n), dt=torch.uint8),
                                   self._new(blocks(most) * n if turned else blocks(n) * most, dt=torch.float32))
        q, s = self._storage[name]
        rows, cols = (n, m) if turned else (m, n)
        return q[:rows * pitch(cols)].view(rows, pitch(cols))[:, :cols], s[:blocks(cols) * rows].view(blocks(cols), rows)

    def form(self, name: str, m: int):
        """8-bit matrix and scales for m tokens: "u" and "ut", "dz" and "dzt" (scales are [blocks, m], so they go by the number)."""
        if not 0 <= m <= self.tokens:
            raise ValueError(f"{m} tokens in a layer that was made for {self.tokens}")
        if (name, m) not in self._views:
            self._views[name, m] = self._cut(name, m, self.width if name.startswith("u") else self.vocab)
        return self._views[name, m]

    def forward(self, x, r, z, keep: bool = True):
        """z = layer(x + r); with `keep` also what backward() reads."""
        m, p = x.shape[0], self.master
        uq, us = self.form("u", m)
        if keep:
            self.ops.layer_norm(x, p["gain"], p["shift"], self.u[:m], residual=r, h=self.h[:m], q=uq, s=us, mean=self.mean[:m], rstd=self.rstd[:m])
        else:
            self.ops.layer_norm(x, p["gain"], p["shift"], residual=r, q=uq, s=us)
        self.ops.product_blocks(uq, us, self.w["q"], self.w["s"], z)

    def backward(self, z, index, value, loss, dh, weight=None, temperature: float = 1.0):
        """loss [tokens], the gradients of all parameters (self.grad) and dh, from the logits of the last forward pass,
        which the gradient of the losses' sum with respect to them replaces."""
        m, g = z.shape[0], self.grad
        dzq, dzs = self.form("dz", m)
        dzqt, dzst = self.form("dzt", m)
        uqt, ust = self.form("ut", m)
        self.ops.distill(z, index, value, loss, weight=weight, dz=z, temperature=temperature)
        self.ops.pack_blocks(z, q=dzq, s=dzs, qt=dzqt, st=dzst)
        self.ops.pack_blocks(self.u[:m], qt=uqt, st=ust)
        self.ops.product_blocks(dzqt, dzst, uqt, ust, g["w"])
        self.ops.product_blocks(dzq, dzs, self.w["qt"], self.w["st"], self.du[:m])
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
