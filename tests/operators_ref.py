"""Plain 64-bit forms of the layer operators and the bounds their results are held to.  No code of the
library is used here."""
from __future__ import annotations

import math

import torch

D = torch.float64
# half a unit in the last place, relative, and the smallest step of the subnormals
HALF_ULP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24, torch.float32: 2.0 ** -149}
NONE, SILU, GELU, SIGMOID, TANH, RELU = 3, 4, 5, 0, 1, 2
# largest |sigma'| and |sigma''| over all arguments (rounded up): how far an error of z reaches
LIP1 = {NONE: 1.0, SILU: 1.1, GELU: 1.13, SIGMOID: 0.25, TANH: 1.0, RELU: 1.0}
LIP2 = {NONE: 0.0, SILU: 0.5, GELU: 1.2, SIGMOID: 0.1, TANH: 0.77, RELU: 0.0}


def act(z, kind):
    if kind == SIGMOID:
        return torch.sigmoid(z)
    if kind == TANH:
        return torch.tanh(z)
    if kind == RELU:
        return torch.where(z > 0, z, z * 0)
    if kind == SILU:
        return z * torch.sigmoid(z)
    if kind == GELU:
        # (1 + tanh u) / 2 = sigmoid(2 u), which keeps its relative accuracy in the left tail
        return z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
    return z


def exponent_err(z, kind):
    """Relative error of sigma(z) from rounding the argument of e^t: GELU's is a cubic, evaluated in fp32 with at most
    four roundings, so e^t is off by 4 * 2^-24 of its magnitude (the other activations' argument is z itself)."""
    return 2.0 ** -22 * (2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)).abs() if kind == GELU else torch.zeros_like(z)


def act_prime(z, kind):
    z = z.clone().requires_grad_(True)
    with torch.enable_grad():
        g, = torch.autograd.grad(act(z, kind).sum() + 0 * z.sum(), z)
    return g.detach()


def scale_bytes(v):
    """e + 127 per group of 32 columns, straight from the definition: the smallest e >= -127 with amax <= 448 * 2^e."""
    rows, n = v.shape
    groups = (n + 31) // 32
    pad = torch.zeros(rows, groups * 32, dtype=D, device=v.device)
    pad[:, :n] = v.to(D)
    amax = pad.view(rows, groups, 32).abs().amax(-1)
    e = torch.full_like(amax, -127.0)
    for k in range(-126, 121):
        e = torch.where(amax > 448.0 * 2.0 ** (k - 1), torch.full_like(e, float(k)), e)
    e = e + 127
    bad = ~torch.isfinite(pad.view(rows, groups, 32)).all(-1)
    return torch.where(bad, torch.full_like(e, 255.0), e).to(torch.uint8)


def columns(per_group, n):
    return per_group.repeat_interleave(32, dim=1)[:, :n]


def pack8(v):
    """(q, s) of the definition, for finite values."""
    s = scale_bytes(v)
    e = columns(s, v.shape[1]).to(D) - 127
    return (v.to(D) * torch.exp2(-e)).float().to(torch.float8_e4m3fn).view(torch.uint8), s


def unpack8(q, s):
    e = columns(s, q.shape[1])
    v = q.view(torch.float8_e4m3fn).to(D) * torch.exp2(e.to(D) - 127)
    return torch.where(e == 255, torch.full_like(v, float("nan")), v)


def rounded(ref, dtype, err=0.0):
    """Largest distance of a correctly rounded result from `ref` when what is rounded is within `err` of it."""
    return HALF_ULP[dtype] * (ref.abs() + err) + TINY[dtype] + err


def product_err(a, b, extra=0.0):
    """Bound on the fp32 error of a @ b (64-bit copies of 16-bit operands, exact products): the tensor core
    adds 16 terms at a time into its accumulator by truncation, 2^-23 of the largest partial sum per step;
    partial sums of splits and chunks add less than as many roundings."""
    steps = a.shape[1] / 16 + 16
    return steps * 2.0 ** -23 * (a.abs() @ b.abs() + extra)


def check(name, got, ref, bound):
    got = got.to(D)
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    assert torch.isfinite(got).all(), f"{name}: non-finite values"
    over = (got - ref).abs() - bound
    worst = over.max().item() if over.numel() else -1.0
    assert worst <= 0, f"{name}: {int((over > 0).sum())} of {over.numel()} elements beyond the bound, worst by {worst:.3e}"
