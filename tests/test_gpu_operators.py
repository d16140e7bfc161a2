"""The layer operators on the GPU against their definitions in 64 bits: values, 8-bit forms, gradients (the
formula's and central differences'), ragged sizes, strides, aliases, streams, empty inputs, values that are not
finite, refusals and waits that run out."""
import os
import subprocess
import sys
import textwrap

import pytest
import torch

import operators_ref as R
import paper_1801_04928_b200 as lf

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
GUARD = 512
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _rand(g, *shape, std=1.0, dtype=F32):
    return torch.empty(shape, device="cuda").normal_(0.0, std, generator=g).to(dtype)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


class Out:
    """An output matrix, NaN-filled (0xA5 bytes for integers), with guard bands around it."""

    def __init__(self, rows, cols, dtype, ld=None):
        ld = ld or cols
        self.raw = torch.empty(rows * ld + 2 * GUARD, dtype=dtype, device="cuda")
        self.fill = 0xA5 if dtype == torch.uint8 else float("nan")
        self.raw.fill_(self.fill)
        self.t = self.raw[GUARD:GUARD + rows * ld].view(rows, ld)[:, :cols]
        self.ld, self.rows, self.cols = ld, rows, cols

    def check(self):
        def clean(v):
            return bool(((v == 0xA5) if v.dtype == torch.uint8 else v.isnan()).all())
        assert clean(self.raw[:GUARD]) and clean(self.raw[GUARD + self.rows * self.ld:]), "written outside the matrix"
        if self.ld > self.cols:
            assert clean(self.raw[GUARD:GUARD + self.rows * self.ld].view(self.rows, self.ld)[:, self.cols:]), "written between rows"


@pytest.fixture(scope="module")
def ops():
    with lf.Operators(lf.lf_ops_workspace(8192, 4096)) as o:
        yield o


def _groups(n):
    return (n + 31) // 32


def _check_packed(name, q, s, ref, err):
    """q, s stand for values within `err` of ref: the scale is right for them up to that error, and a value is half a
    step of the format away at most (2^-4 relative; 2^-10 of the scale where e4m3 is subnormal)."""
    e = s.to(R.D) - 127
    amax_hi, amax_lo = _amax(ref.abs() + err), _amax((ref.abs() - err).clamp(min=0))
    assert bool((amax_lo <= 448 * torch.exp2(e)).all()), f"{name}: a scale is too small"
    assert bool(((amax_hi > 224 * torch.exp2(e)) | (s == 0)).all()), f"{name}: a scale is too large"
    v = R.unpack8(q, s)
    step = torch.exp2(R.columns(e, ref.shape[1]))
    R.check(name, v, ref, err + 2.0 ** -4 * (ref.abs() + err) + 2.0 ** -10 * step)


def _amax(v):
    rows, n = v.shape
    pad = torch.zeros(rows, _groups(n) * 32, dtype=v.dtype, device=v.device)
    pad[:, :n] = v
    return pad.view(rows, -1, 32).amax(-1)


# ---- dense layer, forward ----------------------------------------------------------------------------

def _linear(ops, M, K, N, dtype, act, bias=True, residual=True, ckpt=True, ld_extra=0, form=None, seed=0):
    g = _gen(1000 * M + 10 * K + N + seed)
    x = Out(M, K, dtype, K + ld_extra)
    x.t.copy_(_rand(g, M, K, dtype=dtype))
    w = _rand(g, N, K, std=K ** -0.5, dtype=dtype)
    b = _rand(g, N, std=0.3) if bias else None
    r = Out(M, N, dtype, N + 2 * ld_extra)
    r.t.copy_(_rand(g, M, N, dtype=dtype))
    y = Out(M, N, dtype, N + ld_extra)
    q, s = Out(M, N, torch.uint8), Out(M, _groups(N), torch.uint8)
    ops.linear(x.t, w, y.t, bias=b, residual=r.t if residual else None, act=act, q=q.t if ckpt else None, s=s.t if ckpt else None)
    ops.sync()
    if form:
        assert ops.stats()["form"] == form, ops.stats()
    for o in (x, r, y, q, s):
        o.check()
    z = x.t.to(R.D) @ w.to(R.D).t()
    err = R.product_err(x.t.to(R.D), w.to(R.D).t(), 1.0)
    if bias:
        z = z + b.to(R.D)
        err = err + 2.0 ** -23 * (z.abs() + b.abs().to(R.D))
    a = R.act(z, act)
    # the error of z through sigma, and 4e-6 for e^t and the quotient
    yerr = R.LIP1[act] * err + 4e-6 * (a.abs() + (1 if act == R.TANH else 0))
    ref = a
    if residual:
        ref = a + r.t.to(R.D)
        yerr = yerr + 2.0 ** -24 * ref.abs()
    R.check(f"y {M}x{K}x{N}", y.t, ref, R.rounded(ref, dtype, yerr))
    if ckpt:
        _check_packed(f"z8 {M}x{K}x{N}", q.t, s.t, z, err)


@pytest.mark.parametrize("M", [1, 2, 7, 8, 9, 16])
@pytest.mark.parametrize("K,N,dtype,act", [(8, 8, BF16, R.NONE), (4096, 40, BF16, R.GELU), (520, 1032, F16, R.SILU),
                                           (1024, 72, F16, R.RELU), (2056, 4096, BF16, R.TANH), (264, 264, F16, R.SIGMOID)])
def test_linear_few_tokens(ops, M, K, N, dtype, act):
    _linear(ops, M, K, N, dtype, act, form=lf.LF_FORM_STREAM)


@pytest.mark.parametrize("M,K,N,dtype,act", [(17, 8, 8, BF16, R.NONE), (17, 64, 136, F16, R.GELU), (127, 72, 128, BF16, R.SILU),
                                             (128, 1024, 1024, BF16, R.GELU), (129, 520, 264, F16, R.RELU), (70, 4096, 40, BF16, R.TANH),
                                             (256, 4104, 256, F16, R.SIGMOID), (509, 2048, 1024, BF16, R.NONE), (200, 16384, 64, BF16, R.GELU)])
def test_linear_split_tiles(ops, M, K, N, dtype, act):
    _linear(ops, M, K, N, dtype, act, form=lf.LF_FORM_SPLIT)


@pytest.mark.parametrize("M,K,N,dtype,act", [(2049, 72, 1288, BF16, R.GELU), (1537, 1024, 1800, F16, R.SILU), (4097, 8, 776, BF16, R.RELU),
                                             (2048, 2048, 2048, BF16, R.NONE), (5000, 520, 1032, F16, R.TANH)])
def test_linear_pairs(ops, M, K, N, dtype, act):
    _linear(ops, M, K, N, dtype, act, form=lf.LF_FORM_PAIRS)


# tiles of 160, 192 and 224 columns, 256 and 512 rows
@pytest.mark.parametrize("M,K,N,dtype,act,ckpt", [
    (409, 72, 4760, BF16, R.GELU, False), (1036, 200, 2096, F16, R.SILU, True), (312, 64, 6384, BF16, R.NONE, False), (273, 248, 6368, BF16, R.NONE, True),
    (268, 72, 7424, F16, R.TANH, False), (262, 200, 7432, BF16, R.GELU, True), (2026, 64, 2432, BF16, R.SIGMOID, False), (814, 64, 5440, F16, R.NONE, True),
    (1682, 64, 2912, BF16, R.RELU, False), (641, 64, 6776, BF16, R.GELU, True), (1062, 64, 4808, F16, R.GELU, False), (591, 64, 7592, BF16, R.NONE, True),
    (408, 1160, 12728, BF16, R.SILU, True), (1453, 12328, 1960, BF16, R.GELU, False)])
@pytest.mark.parametrize("residual", [False, True])
def test_linear_narrow_pair_tiles(ops, M, K, N, dtype, act, ckpt, residual):
    _linear(ops, M, K, N, dtype, act, residual=residual, ckpt=ckpt, ld_extra=8 if residual else 0, form=lf.LF_FORM_PAIRS)


@pytest.mark.parametrize("M,K,N,dtype,act", [(512, 4096, 3976, BF16, R.GELU), (400, 4104, 4096, F16, R.NONE), (1900, 4096, 1000, BF16, R.SIGMOID),
                                             (2048, 8200, 1024, F16, R.RELU)])
def test_linear_split_pairs(ops, M, K, N, dtype, act):
    _linear(ops, M, K, N, dtype, act, form=lf.LF_FORM_SPLIT_PAIRS)


@pytest.mark.parametrize("M,K,N", [(3, 264, 72), (130, 264, 200), (2050, 136, 1400)])
@pytest.mark.parametrize("bias,residual,ckpt,ld", [(False, False, False, 0), (True, False, True, 8), (False, True, False, 24), (True, True, True, 40)])
def test_linear_options_and_strides(ops, M, K, N, bias, residual, ckpt, ld):
    _linear(ops, M, K, N, BF16, R.GELU, bias, residual, ckpt, ld)


@pytest.mark.parametrize("M,K,N", [(5, 512, 96), (300, 512, 96), (2100, 128, 1304)])
def test_linear_adds_into_its_residual_and_repeats_bitwise(ops, M, K, N):
    g = _gen(5)
    x, w, r = _rand(g, M, K, dtype=BF16), _rand(g, N, K, std=0.05, dtype=BF16), _rand(g, M, N, dtype=BF16)
    y = torch.empty_like(r)
    ops.linear(x, w, y, residual=r, act=R.SILU)
    for _ in range(3):
        r2 = r.clone()
        ops.linear(x, w, r2, residual=r2, act=R.SILU)
        assert torch.equal(r2, y)


def test_linear_row_does_not_depend_on_its_neighbours_being_finite(ops):
    # a token with infinities or NaN spoils its own row only; in 8 bits, its own groups only
    for M, K, N in ((4, 256, 96), (40, 256, 96), (2100, 256, 1304)):
        g = _gen(6)
        x, w = _rand(g, M, K, dtype=BF16), _rand(g, N, K, std=0.05, dtype=BF16)
        y, y2 = (torch.empty(M, N, dtype=BF16, device="cuda") for _ in range(2))
        q, s, q2, s2 = (torch.empty(M, c, dtype=torch.uint8, device="cuda") for c in (N, _groups(N), N, _groups(N)))
        ops.linear(x, w, y, q=q, s=s)
        x2 = x.clone()
        x2[1, 3] = float("nan")
        x2[2, 5] = float("inf")
        ops.linear(x2, w, y2, q=q2, s=s2)
        others = [i for i in range(M) if i not in (1, 2)]
        assert torch.equal(y[others], y2[others]) and torch.equal(q[others], q2[others]) and torch.equal(s[others], s2[others])
        assert y2[1].isnan().all() and not y2[2].isfinite().any()
        assert bool((s2[1:3] == 255).all())
        v = torch.empty_like(y)
        ops.unpack8(q2, s2, v)
        assert v[1:3].isnan().all() and v[others].isfinite().all()


# ---- dense layer, backward ----------------------------------------------------------------------------

def _backward(ops, M, K, N, dtype, act, gw_dtype, eight=True, add=False, ld_extra=0, forms=(None, None)):
    g = _gen(77 + 1000 * M + 10 * K + N)
    dz = Out(M, N, dtype, N + ld_extra)
    dz.t.copy_(_rand(g, M, N, std=0.1, dtype=dtype))
    w = _rand(g, N, K, std=N ** -0.5, dtype=dtype)
    z32 = _rand(g, M, K, std=1.5)
    x = Out(M, K, dtype, K + ld_extra)
    x.t.copy_(z32.to(dtype))
    q, s = R.pack8(z32)
    zv = R.unpack8(q, s) if eight else None
    addm = Out(M, K, dtype, K + 3 * ld_extra)
    addm.t.copy_(_rand(g, M, K, std=0.1, dtype=dtype))
    dx, gw, gb = Out(M, K, dtype, K + 2 * ld_extra), Out(N, K, gw_dtype), Out(1, N, F32)
    ops.linear_grad_x(dz.t, w, dx.t, q=q if eight else None, s=s if eight else None, act=act if eight else R.NONE, add=addm.t if add else None)
    if forms[0]:
        assert ops.stats()["form"] == forms[0], ops.stats()
    if eight:
        ops.linear_grad_w(dz.t, gw.t, gb=gb.t.view(-1), q=q, s=s, act=act)
    else:
        ops.linear_grad_w(dz.t, gw.t, gb=gb.t.view(-1), x=x.t)
    if forms[1]:
        assert ops.stats()["form"] == forms[1], ops.stats()
    ops.sync()
    for o in (dz, x, addm, dx, gw, gb):
        o.check()
    d64, w64 = dz.t.to(R.D), w.to(R.D)
    t = d64 @ w64
    err = R.product_err(d64, w64)
    if eight:
        sp = R.act_prime(zv, act)
        err = err * sp.abs() + 8e-6 * t.abs()
        t = t * sp
    if add:
        t = t + addm.t.to(R.D)
        err = err + 2.0 ** -24 * t.abs()
    R.check("dx", dx.t, t, R.rounded(t, dtype, err))
    # the layer's input as it enters the products: sigma(z) rounded to 16 bits
    if eight:
        a = R.act(zv, act)
        aerr = torch.zeros_like(a) if act in (R.NONE, R.RELU) else R.rounded(a, dtype, 4e-6 * (a.abs() + 1))
        if dtype == F16:
            aerr = aerr + R.TINY[F16]
    else:
        a, aerr = x.t.to(R.D), None
    ref = d64.t() @ a
    gerr = R.product_err(d64.t(), a) + (d64.abs().t() @ aerr if aerr is not None else 0)
    R.check("gw", gw.t, ref, R.rounded(ref, gw_dtype, gerr))
    col = d64.sum(0)
    R.check("gb", gb.t.view(-1), col, (M / 16 + 16) * 2.0 ** -23 * d64.abs().sum(0) + 1e-30)


@pytest.mark.parametrize("M,K,N,dtype,act,gw", [
    (1, 8, 8, BF16, R.GELU, F32), (3, 72, 40, F16, R.NONE, F32), (64, 64, 64, BF16, R.SILU, BF16), (65, 520, 136, F16, R.SIGMOID, F16),
    (70, 1032, 520, BF16, R.RELU, F32), (129, 256, 1024, F16, R.TANH, F32), (1000, 136, 264, BF16, R.GELU, BF16), (4100, 72, 136, BF16, R.NONE, F32),
    (2047, 520, 1032, F16, R.SILU, F16)])
def test_backward_from_eight_bits(ops, M, K, N, dtype, act, gw):
    _backward(ops, M, K, N, dtype, act, gw)


@pytest.mark.parametrize("M,K,N,dtype,act,gw", [
    (2049, 1288, 1800, BF16, R.GELU, BF16), (1800, 1544, 2056, F16, R.NONE, F32), (2300, 2048, 1536, BF16, R.RELU, F32)])
def test_backward_pairs(ops, M, K, N, dtype, act, gw):
    _backward(ops, M, K, N, dtype, act, gw, forms=(lf.LF_FORM_PAIRS, lf.LF_FORM_PAIRS))


@pytest.mark.parametrize("M,K,N,dtype,gw", [(33, 136, 72, BF16, F32), (300, 1032, 264, F16, F16), (2100, 1400, 1512, BF16, F32)])
@pytest.mark.parametrize("ld", [0, 24])
def test_backward_from_sixteen_bits(ops, M, K, N, dtype, gw, ld):
    _backward(ops, M, K, N, dtype, R.NONE, gw, eight=False, add=True, ld_extra=ld)


@pytest.mark.parametrize("M,K,N,dtype,act,gw,forms", [
    (500, 4000, 4096, BF16, R.GELU, BF16, (lf.LF_FORM_SPLIT_PAIRS, None)), (4096, 2048, 1024, F16, R.SILU, F16, (None, lf.LF_FORM_SPLIT_PAIRS))])
def test_backward_split_pairs(ops, M, K, N, dtype, act, gw, forms):
    _backward(ops, M, K, N, dtype, act, gw, forms=forms)


def test_weight_gradient_over_many_tokens_keeps_fp32(ops):
    # 8192 tokens, all terms positive: truncation in the accumulator would show as a bias of 2^-23 per
    # instruction; chunks of 512 tokens added in registers stay below 32 * 2^-23 plus 16 roundings
    g = _gen(9)
    for n_out, n_in in ((64, 72), (2304, 2304)):
        M = 8192
        dz = (0.5 + torch.rand(M, n_out, device="cuda", generator=g)).to(BF16)
        x = (0.5 + torch.rand(M, n_in, device="cuda", generator=g)).to(BF16)
        gw = torch.empty(n_out, n_in, device="cuda")
        ops.linear_grad_w(dz, gw, x=x)
        ref = dz.to(R.D).t() @ x.to(R.D)
        R.check("gw", gw, ref, (32 + 16) * 2.0 ** -23 * ref)


def _one_sign(g, rows, cols, dtype, scale=1.0, dim=0):
    """Positive numbers, every row (or column) with a magnitude of its own, so that the sums spread over the roundings."""
    v = 0.75 + 0.5 * torch.rand(rows, cols, device="cuda", generator=g)
    v *= torch.exp2(torch.rand((rows, 1) if dim == 0 else (1, cols), device="cuda", generator=g)) * scale
    return v.to(dtype)


def _check_long(name, got, ref, terms):
    """Sums of terms of one sign: an accumulator takes 2048 instructions for f16, 4096 for bf16, each truncated by a unit of 2^-23 at most;
    fills, parts and warps are added with round-to-nearest.  The bound does not grow with the contraction as truncation over all
    of it would, which the mean of the errors shows: the type's own rounding averages out (4 standard deviations of its mean)."""
    dtype = got.dtype
    rel = (2048 if dtype == F16 else 4096) * 2.0 ** -23 + (terms / 16384 + 16) * 2.0 ** -24
    R.check(name, got, ref, R.rounded(ref, dtype, rel * ref))
    mean = ((got.to(R.D) - ref) / ref).mean().item()
    assert abs(mean) <= rel + 4 * R.HALF_ULP[dtype] / (3 * ref.numel()) ** 0.5, mean


@pytest.mark.parametrize("M,K,N,dtype,form", [(4, 1 << 20, 512, F16, lf.LF_FORM_STREAM), (12, 1 << 20, 256, F16, lf.LF_FORM_STREAM),
                                              (5, (1 << 18) + 8 * 77, 264, BF16, lf.LF_FORM_STREAM),
                                              (32, 1 << 20, 128, F16, lf.LF_FORM_SPLIT), (40, (1 << 20) + 72, 136, BF16, lf.LF_FORM_SPLIT),
                                              (2048, 1 << 16, 2048, F16, lf.LF_FORM_PAIRS), (2050, 66568, 2048, BF16, lf.LF_FORM_PAIRS)])
def test_long_contractions_in_sixteen_bits(ops, M, K, N, dtype, form):
    g = _gen(21)
    x, w = _one_sign(g, M, K, dtype), _one_sign(g, N, K, dtype, 64 / K)
    y = torch.empty(M, N, dtype=dtype, device="cuda")
    ops.linear(x, w, y)
    ops.sync()
    assert ops.stats()["form"] == form
    m = min(M, 64)
    _check_long("y", y[-m:], x[-m:].to(R.D) @ w.to(R.D).t(), K)


@pytest.mark.parametrize("M,K,N,form", [(64, 128, 1 << 20, lf.LF_FORM_SPLIT), (2048, 2048, 1 << 16, lf.LF_FORM_PAIRS)])
def test_long_contractions_in_sixteen_bits_grad_x(ops, M, K, N, form):
    g = _gen(22)
    dz, w = _one_sign(g, M, N, F16), _one_sign(g, N, K, F16, 64 / N, dim=1)
    dx = torch.empty(M, K, dtype=F16, device="cuda")
    ops.linear_grad_x(dz, w, dx)
    ops.sync()
    assert ops.stats()["form"] == form
    _check_long("dx", dx[:64], dz[:64].to(R.D) @ w.to(R.D), N)


@pytest.mark.parametrize("M,K,N,form", [(1 << 20, 512, 512, lf.LF_FORM_SPLIT), (1 << 17, 2048, 2048, lf.LF_FORM_PAIRS)])
def test_long_contractions_in_sixteen_bits_grad_w(ops, M, K, N, form):
    g = _gen(23)
    dz, x = _one_sign(g, M, N, F16, 64 / M, dim=1), _one_sign(g, M, K, F16, dim=1)
    gw = torch.empty(N, K, dtype=F16, device="cuda")
    ops.linear_grad_w(dz, gw, x=x)
    ops.sync()
    assert ops.stats()["form"] == form
    _check_long("gw", gw[:64], dz[:, :64].to(R.D).t() @ x.to(R.D), M)


# one fill of the accumulator and a little, with everything that the epilogues do (32768 terms of f16 and 65536 of bf16 a part, 16384 a warp)
@pytest.mark.parametrize("M,K,N,dtype,act,form", [
    (5, 262160, 72, BF16, R.GELU, lf.LF_FORM_STREAM), (13, 196680, 40, F16, R.SILU, lf.LF_FORM_STREAM), (40, 262152, 136, F16, R.TANH, lf.LF_FORM_SPLIT),
    (1030, 32776, 2056, F16, R.GELU, lf.LF_FORM_PAIRS), (1030, 32776, 3080, F16, R.NONE, lf.LF_FORM_PAIRS), (1030, 65600, 2056, BF16, R.SILU, lf.LF_FORM_PAIRS)])
@pytest.mark.parametrize("options", [False, True])
def test_long_contractions_and_their_epilogues(ops, M, K, N, dtype, act, form, options):
    _linear(ops, M, K, N, dtype, act, residual=options, ckpt=options, ld_extra=8 if options else 0, form=form)


@pytest.mark.parametrize("M,K,N,dtype,act,gw,forms", [
    (1030, 2056, 32776, F16, R.GELU, F16, (lf.LF_FORM_PAIRS, None)), (1030, 2056, 65544, BF16, R.RELU, BF16, (lf.LF_FORM_PAIRS, None)),
    (40, 136, 262152, F16, R.SIGMOID, F32, (lf.LF_FORM_SPLIT, None)), (262152, 72, 64, F16, R.NONE, F16, (None, lf.LF_FORM_SPLIT)),
    (32784, 1544, 2056, F16, R.TANH, F16, (None, lf.LF_FORM_PAIRS))])
def test_long_contractions_backward(ops, M, K, N, dtype, act, gw, forms):
    with lf.Operators(lf.lf_ops_workspace(M, K)) as o:
        _backward(o, M, K, N, dtype, act, gw, add=act != R.GELU, forms=forms)


@pytest.mark.parametrize("M,K,N", [(5, 16, 24), (40, 16, 24)])
@pytest.mark.parametrize("act", [R.GELU, R.SILU, R.SIGMOID, R.TANH, R.NONE])
def test_gradients_against_central_differences(ops, M, K, N, act):
    # C = sum(dy * (sigma(x w^T + b))) in 64 bits; the pre-activation goes through 8 bits, so the network
    # differentiated is the one whose z is the stored value: z = z8 + (x - x0) w^T + ...
    g = _gen(10 + act)
    x, w, b = _rand(g, M, K, dtype=BF16), _rand(g, N, K, std=0.4, dtype=BF16), _rand(g, N, std=0.2)
    dy = _rand(g, M, N, dtype=BF16)
    y = torch.empty(M, N, dtype=BF16, device="cuda")
    q, s = torch.empty(M, N, dtype=torch.uint8, device="cuda"), torch.empty(M, _groups(N), dtype=torch.uint8, device="cuda")
    ops.linear(x, w, y, bias=b, act=act, q=q, s=s)
    dz, dx = torch.empty_like(y), torch.empty_like(x)
    gw, gb = torch.empty(N, K, device="cuda"), torch.empty(N, device="cuda")
    ops.act_backward(dy, q, s, dz, act=act)
    ops.linear_grad_x(dz, w, dx)
    ops.linear_grad_w(dz, gw, gb=gb, x=x)
    ops.sync()
    z8, x0, w0, d64 = R.unpack8(q, s), x.to(R.D), w.to(R.D), dy.to(R.D)

    def cost(dxv, dwv, dbv):
        return (d64 * R.act(z8 + dxv @ w0.t() + x0 @ dwv.t() + dbv, act)).sum().item()

    h = 1e-4
    zx, zw, zb = torch.zeros_like(x0), torch.zeros_like(w0), torch.zeros(N, dtype=R.D, device="cuda")
    # dz is rounded to bf16, dx once more: 2^-8 of the sums of magnitudes; differences are exact to h^2
    mag = d64.abs() * R.LIP1[act]
    for got, zero, bound, slot in ((dx, zx, mag @ w0.abs(), 0), (gw, zw, mag.t() @ x0.abs(), 1), (gb, zb, mag.sum(0), 2)):
        for i in range(0, zero.numel(), max(1, zero.numel() // 24)):
            step = [zx, zw, zb]
            step[slot] = zero.clone()
            step[slot].view(-1)[i] = h
            up = cost(*step)
            step[slot].view(-1)[i] = -h
            fd = (up - cost(*step)) / (2 * h)
            assert abs(got.reshape(-1)[i].item() - fd) <= 2.0 ** -8 * bound.reshape(-1)[i].item() + 1e-6, (slot, i)


# ---- norm ---------------------------------------------------------------------------------------------

NORM_SHAPES = [(1, 8), (1, 4096), (3, 40), (300, 256), (301, 264), (17, 520), (310, 1032), (5, 2056), (300, 4096), (300, 4104), (9, 8192),
               (297, 8200), (2, 16384), (299, 16384)]


def _norm(ops, M, n, dtype, residual, ckpt, with_y=True, ld=0, eps=1e-5):
    g = _gen(3 * M + n)
    x, r = Out(M, n, dtype, n + ld), Out(M, n, dtype, n + 2 * ld)
    x.t.copy_(_rand(g, M, n, std=2.0, dtype=dtype))
    r.t.copy_(_rand(g, M, n, dtype=dtype))
    gain = 1 + _rand(g, n, std=0.2)
    h, y = Out(M, n, dtype, n + ld), Out(M, n, dtype, n + 3 * ld)
    q, s = Out(M, n, torch.uint8), Out(M, _groups(n), torch.uint8)
    ops.rms_norm(x.t, gain, y.t if with_y else None, residual=r.t if residual else None, h=h.t if residual else None,
                 q=q.t if ckpt else None, s=s.t if ckpt else None, eps=eps)
    ops.sync()
    for o in (x, r, h, y, q, s):
        o.check()
    h64 = x.t.to(R.D) + (r.t.to(R.D) if residual else 0)
    ref = h64 / (h64.square().mean(1, keepdim=True) + eps).sqrt() * gain.to(R.D)
    # the sum of squares has n terms in at most n / 32 + 16 additions per partial sum; half of its error reaches y
    err = (n / 64 + 16) * 2.0 ** -24 * ref.abs() + 2.0 ** -22 * ref.abs()
    if residual:
        R.check("h", h.t, h64, R.rounded(h64, dtype, 2.0 ** -24 * h64.abs()))
    if with_y:
        R.check("y", y.t, ref, R.rounded(ref, dtype, err))
    if ckpt:
        _check_packed("y8", q.t, s.t, ref, err)


@pytest.mark.parametrize("M,n", NORM_SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_norm(ops, M, n, dtype):
    _norm(ops, M, n, dtype, True, True)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("residual,ckpt,with_y,ld", [(False, False, True, 0), (False, True, False, 8), (True, False, True, 16), (True, True, False, 0)])
def test_norm_options_and_strides(ops, dtype, residual, ckpt, with_y, ld):
    for M, n in ((4, 1032), (333, 264)):
        _norm(ops, M, n, dtype, residual, ckpt, with_y, ld)


def test_norm_of_zero_rows_and_rows_that_are_not_finite(ops):
    x = torch.ones(6, 256, dtype=BF16, device="cuda")
    x[1] = 0
    x[2, 7] = float("inf")
    x[3, 9] = float("nan")
    x[4] = 3e38                       # the sum of squares overflows fp32, as the definition in fp32 does
    gain = torch.ones(256, device="cuda")
    y = torch.empty_like(x)
    q, s = torch.empty(6, 256, dtype=torch.uint8, device="cuda"), torch.empty(6, 8, dtype=torch.uint8, device="cuda")
    ops.rms_norm(x, gain, y, q=q, s=s, eps=0.0)
    ops.sync()
    assert y[0].eq(1).all() and y[5].eq(1).all()
    assert y[1].isnan().all() and y[2].isnan().any() and y[3].isnan().all() and y[4].eq(0).all()    # 0 / 0, inf, NaN, 3e38 / inf
    assert bool((s[1] == 255).all()) and bool((s[3] == 255).all()) and bool((s[4] == 0).all())
    ops.rms_norm(x, gain, y, q=q, s=s, eps=1e-6)
    ops.sync()
    assert y[1].eq(0).all() and bool((q[1] == 0).all()) and bool((s[1] == 0).all())
    # h and y may be written over x and residual
    a, b = torch.randn(5, 264, device="cuda").to(BF16), torch.randn(5, 264, device="cuda").to(BF16)
    h, y = torch.empty_like(a), torch.empty_like(a)
    g = torch.rand(264, device="cuda")
    ops.rms_norm(a, g, y, residual=b, h=h)
    a2, b2 = a.clone(), b.clone()
    ops.rms_norm(a2, g, a2, residual=b2, h=b2)
    assert torch.equal(a2, y) and torch.equal(b2, h)


def _norm_backward(ops, M, n, dtype, dres, dgain=True, ld=0, eps=1e-5):
    g = _gen(5 * M + n)
    h, dy, r = Out(M, n, dtype, n + ld), Out(M, n, dtype, n + 2 * ld), Out(M, n, dtype, n + ld)
    h.t.copy_(_rand(g, M, n, std=2.0, dtype=dtype))
    dy.t.copy_(_rand(g, M, n, std=0.3, dtype=dtype))
    r.t.copy_(_rand(g, M, n, std=0.3, dtype=dtype))
    gain = 1 + _rand(g, n, std=0.2)
    dh, dg = Out(M, n, dtype, n + 3 * ld), Out(1, n, F32)
    ops.rms_norm_backward(dy.t, h.t, gain, dh.t, dg.t.view(-1) if dgain else None, dres=r.t if dres else None, eps=eps)
    ops.sync()
    for o in (h, dy, r, dh, dg):
        o.check()
    h64, y64, g64 = h.t.to(R.D), dy.t.to(R.D), gain.to(R.D)
    rstd = (h64.square().mean(1, keepdim=True) + eps).rsqrt()
    hn, u = h64 * rstd, y64 * g64
    ref = rstd * (u - hn * (u * hn).mean(1, keepdim=True))
    # both row sums have errors of (n / 32 + 16) additions, relative to their sums of magnitudes
    k = (n / 32 + 16) * 2.0 ** -24
    err = k * (ref.abs() + rstd * hn.abs() * (u * hn).abs().mean(1, keepdim=True) * 2) + 2.0 ** -21 * rstd * (u.abs() + hn.abs() * (u * hn).abs().mean(1, keepdim=True))
    if dres:
        ref = ref + r.t.to(R.D)
        err = err + 2.0 ** -24 * ref.abs()
    R.check("dh", dh.t, ref, R.rounded(ref, dtype, err))
    if dgain:
        terms = (y64 * hn).abs().sum(0)
        R.check("dgain", dg.t.view(-1), (y64 * hn).sum(0), (M / 8 + 340 + n / 64) * 2.0 ** -24 * terms + 1e-30)
    else:
        assert dg.t.isnan().all()


@pytest.mark.parametrize("M,n", NORM_SHAPES + [(2000, 1024), (5000, 72)])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_norm_backward(ops, M, n, dtype):
    _norm_backward(ops, M, n, dtype, True)


@pytest.mark.parametrize("dres,dgain,ld", [(False, True, 8), (True, False, 0), (False, False, 16)])
def test_norm_backward_options_and_strides(ops, dres, dgain, ld):
    for M, n, dtype in ((4, 1032, BF16), (333, 264, F32)):
        _norm_backward(ops, M, n, dtype, dres, dgain, ld)


# one cluster of up to eight blocks, with one to eight rows each
@pytest.mark.parametrize("M,n", [(1, 4096), (2, 8), (3, 264), (5, 4088), (8, 2048), (8, 4096), (11, 520), (16, 1024), (64, 248)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dres", [False, True])
def test_norm_backward_of_few_rows_is_one_launch(ops, M, n, dtype, dres):
    _norm_backward(ops, M, n, dtype, dres)
    assert ops.stats()["launches"] == 1


@pytest.mark.parametrize("M,n,dtype", [(1, 4096, BF16), (5, 264, F16), (300, 4096, BF16), (2000, 1032, F32), (299, 16384, F32)])
@pytest.mark.parametrize("ld", [0, 16])
def test_norm_backward_over_one_of_its_inputs(ops, M, n, dtype, ld):
    g = _gen(M)
    t = [Out(M, n, dtype, n + ld) for _ in range(3)]
    for o in t:
        o.t.copy_(_rand(g, M, n, dtype=dtype))
    gain = 1 + _rand(g, n, std=0.2)
    want, dg, dg2 = torch.empty(M, n, dtype=dtype, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    ops.rms_norm_backward(t[0].t, t[1].t, gain, want, dg, dres=t[2].t)
    for over in range(3):
        kept = [o.t.clone() for o in t]
        ops.rms_norm_backward(t[0].t, t[1].t, gain, t[over].t, dg2, dres=t[2].t)
        ops.sync()
        assert torch.equal(t[over].t, want) and torch.equal(dg, dg2)
        for o, k in zip(t, kept):
            o.check()
            o.t.copy_(k)


def test_norm_backward_from_several_threads():
    # handles of their own, calls with and without dres (which need different shared memory) at the same time
    import threading
    refusals = []

    def work(dres):
        with lf.Operators() as o:
            h, gain = torch.ones(4, 16384, dtype=BF16, device="cuda"), torch.ones(16384, device="cuda")
            dh = torch.empty_like(h)
            a = lf.lf_rms_norm_backward_args(dtype=lf.LF_BF16, tokens=4, n=16384, eps=1e-5, dy=h.data_ptr(), h=h.data_ptr(), gain=gain.data_ptr(),
                                             dres=h.data_ptr() if dres else None, dh=dh.data_ptr())
            torch.cuda.synchronize()
            refusals.extend(rc for rc in (lf.lf_rms_norm_backward(o._h, a) for _ in range(3000)) if rc != lf.LF_OK)     # (ctypes lets threads run)
            o.sync()

    threads = [threading.Thread(target=work, args=(i % 2 == 0,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not refusals, (len(refusals), refusals[0])


def test_norm_backward_against_central_differences(ops):
    g = _gen(11)
    h, dy, gain = _rand(g, 3, 40), _rand(g, 3, 40), 1 + _rand(g, 40, std=0.2)
    dh, dg = torch.empty_like(h), torch.empty(40, device="cuda")
    ops.rms_norm_backward(dy, h, gain, dh, dg, eps=1e-3)
    ops.sync()
    h64, y64, g64 = h.to(R.D), dy.to(R.D), gain.to(R.D)

    def cost(hv, gv):
        return (y64 * hv / (hv.square().mean(1, keepdim=True) + 1e-3).sqrt() * gv).sum().item()

    for i in range(0, 120, 7):
        e = torch.zeros(120, dtype=R.D, device="cuda")
        e[i] = 1e-5
        e = e.view(3, 40)
        fd = (cost(h64 + e, g64) - cost(h64 - e, g64)) / 2e-5
        assert abs(dh.view(-1)[i].item() - fd) <= 1e-5 * (1 + abs(fd))
    for i in range(0, 40, 5):
        e = torch.zeros(40, dtype=R.D, device="cuda")
        e[i] = 1e-5
        fd = (cost(h64, g64 + e) - cost(h64, g64 - e)) / 2e-5
        assert abs(dg[i].item() - fd) <= 1e-5 * (1 + abs(fd))


# ---- 8 bits -------------------------------------------------------------------------------------------

def _awkward(g, M, n, dtype):
    """Magnitudes over the whole range of the type, zeros, group maxima on and next to 448 * 2^e."""
    big = {BF16: 120, F16: 14, F32: 120}[dtype]
    low = {BF16: -126, F16: -20, F32: -140}[dtype]
    v = _rand(g, M, n) * torch.exp2(torch.empty(M, 1, device="cuda").uniform_(low, big, generator=g))
    v = v * torch.exp2(torch.empty(M, n, device="cuda").uniform_(-12, 0, generator=g))
    v[:, ::5] = 0
    if M > 2:
        v[1] = 0
        v[2] = torch.tensor([448.0, 449.0, 447.0, 1.0], device="cuda").repeat((n + 3) // 4)[:n]
    return v.to(dtype)


@pytest.mark.parametrize("M,n", [(1, 8), (3, 32), (4, 40), (33, 264), (300, 1032), (5, 4096), (1000, 2056)])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_pack_and_unpack_are_the_definition(ops, M, n, dtype):
    g = _gen(M + n)
    for ld in (0, 8):
        x = Out(M, n, dtype, n + ld)
        x.t.copy_(_awkward(g, M, n, dtype))
        q, s, v = Out(M, n, torch.uint8), Out(M, _groups(n), torch.uint8), Out(M, n, dtype, n + 2 * ld)
        ops.pack8(x.t, q.t, s.t)
        ops.unpack8(q.t, s.t, v.t)
        ops.sync()
        for o in (x, q, s, v):
            o.check()
        rq, rs = R.pack8(x.t)
        assert torch.equal(s.t, rs)
        same = (q.t == rq) | ((q.t & 0x7F == 0) & (rq & 0x7F == 0))      # either zero
        assert bool(same.all())
        big = float(torch.finfo(dtype).max)
        assert torch.equal(v.t, R.unpack8(q.t, s.t).clamp(-big, big).to(dtype))


def test_groups_that_are_not_finite_read_back_as_nan(ops):
    for dtype in (BF16, F16, F32):
        x = torch.ones(2, 72, dtype=dtype, device="cuda")
        x[0, 33] = float("inf")
        x[1, 70] = float("nan")
        q, s, v = torch.empty(2, 72, dtype=torch.uint8, device="cuda"), torch.empty(2, 3, dtype=torch.uint8, device="cuda"), torch.empty_like(x)
        ops.pack8(x, q, s)
        ops.unpack8(q, s, v)
        ops.sync()
        assert s.tolist() == [[119, 255, 119], [119, 119, 255]]
        assert v[0, 32:64].isnan().all() and v[1, 64:].isnan().all()
        assert v[0, :32].eq(1).all() and v[0, 64:].eq(1).all() and v[1, :64].eq(1).all()


@pytest.mark.parametrize("act", [R.SILU, R.GELU, R.SIGMOID, R.TANH, R.RELU])
def test_gradients_through_groups_that_are_not_finite_are_nan(ops, act):
    # what z was is not known there: a gradient that looks like a number would hide it
    for dtype in (BF16, F16, F32):
        z, dy = torch.ones(3, 72, dtype=dtype, device="cuda"), torch.ones(3, 72, dtype=dtype, device="cuda")
        z[0, 33], z[1, 70] = float("inf"), float("nan")
        q, s, dz = torch.empty(3, 72, dtype=torch.uint8, device="cuda"), torch.empty(3, 3, dtype=torch.uint8, device="cuda"), torch.empty_like(z)
        ops.pack8(z, q, s)
        ops.act_backward(dy, q, s, dz, act=act)
        ops.sync()
        bad = torch.zeros(3, 72, dtype=torch.bool, device="cuda")
        bad[0, 32:64] = bad[1, 64:] = True
        assert torch.equal(dz.isnan(), bad)
    for M, K, N, form in ((40, 136, 72, lf.LF_FORM_SPLIT), (2049, 1288, 1800, lf.LF_FORM_PAIRS), (500, 4000, 4096, lf.LF_FORM_SPLIT_PAIRS)):
        g = _gen(M)
        z, dz, w = _rand(g, M, K, dtype=BF16), _rand(g, M, N, dtype=BF16), _rand(g, N, K, std=N ** -0.5, dtype=BF16)
        z[3, 40], z[M - 1, K - 1] = float("inf"), float("nan")
        q, s, dx = torch.empty(M, K, dtype=torch.uint8, device="cuda"), torch.empty(M, _groups(K), dtype=torch.uint8, device="cuda"), torch.empty_like(z)
        ops.pack8(z, q, s)
        ops.linear_grad_x(dz, w, dx, q=q, s=s, act=act)
        ops.sync()
        assert ops.stats()["form"] == form
        bad = torch.zeros(M, K, dtype=torch.bool, device="cuda")
        bad[3, 32:64] = bad[M - 1, (K - 1) // 32 * 32:] = True
        assert torch.equal(dx.isnan(), bad)


@pytest.mark.parametrize("act", [R.NONE, R.SILU, R.GELU, R.SIGMOID, R.TANH, R.RELU])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_activation_and_derivative_from_eight_bits(ops, act, dtype):
    g = _gen(act)
    for M, n in ((3, 40), (257, 1032)):
        z = _rand(g, M, n, std=4.0)
        z[0, :8] = torch.tensor([0.0, -0.0, 30.0, -30.0, 100.0, -100.0, 8.0, -8.0])
        q, s = R.pack8(z)
        v = R.unpack8(q, s)
        a, dy, dz = Out(M, n, dtype, n + 8), _rand(g, M, n, dtype=dtype), Out(M, n, dtype, n + 16)
        ops.unpack8(q, s, a.t, act=act)
        ops.act_backward(dy, q, s, dz.t, act=act)
        ops.sync()
        a.check(); dz.check()
        f = 1e-6 if dtype == F32 else 8e-6      # correctly scaled functions; special-function unit
        ref = R.act(v, act)
        R.check("a", a.t, ref, R.rounded(ref, dtype, (f + R.exponent_err(v, act)) * ref.abs() + 1e-37))
        ref = dy.to(R.D) * R.act_prime(v, act)
        # sigma' is made of terms up to 1 + |z| that cancel in the tails
        R.check("dz", dz.t, ref, R.rounded(ref, dtype, f * dy.to(R.D).abs() * (1 + v.abs()) * (2 if act in (R.TANH, R.GELU) else 1)))


# every magnitude of which the 8-bit form is kept: sigma is 0, +-1 or its argument there and sigma' 0 or 1, all of them exactly
LARGE = (1e10, 1e11, 3e11, 1e13, 2e13, 1e14, 1e19, 2e19, 1e20, 1e30, 3.4e38)


def _large(M, n):
    v = torch.tensor(LARGE, device="cuda").repeat_interleave(2)[torch.arange(M, device="cuda") % (2 * len(LARGE))]
    sign = 1 - 2 * ((torch.arange(n, device="cuda")[None, :] + torch.arange(M, device="cuda")[:, None]) % 2)
    q, s = R.pack8(v[:, None] * sign)
    assert 247 in s                            # 3.4e38 is kept as 256 * 2^120, beyond fp32
    up = sign > 0
    return q, s, up, R.unpack8(q, s)


@pytest.mark.parametrize("act", [R.NONE, R.SILU, R.GELU, R.SIGMOID, R.TANH, R.RELU])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_activation_of_the_largest_values(ops, act, dtype):
    for M, n in ((22, 40), (44, 64)):
        q, s, up, v = _large(M, n)
        big = float(torch.finfo(dtype).max)
        v = v.clamp(-big, big).to(dtype)
        a = torch.empty_like(v)
        ops.unpack8(q, s, a, act=act)
        ops.sync()
        low = {R.NONE: v, R.TANH: -torch.ones_like(v)}.get(act, torch.zeros_like(v))
        high = torch.ones_like(v) if act in (R.TANH, R.SIGMOID) else v
        assert torch.equal(a, torch.where(up, high, low))


@pytest.mark.parametrize("act", [R.NONE, R.SILU, R.GELU, R.SIGMOID, R.TANH, R.RELU])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_derivative_at_the_largest_values(ops, act, dtype):
    for M, n in ((22, 40), (44, 64)):
        q, s, up, _ = _large(M, n)
        dy, dz = _rand(_gen(act), M, n, dtype=dtype), torch.empty(M, n, dtype=dtype, device="cuda")
        ops.act_backward(dy, q, s, dz, act=act)
        ops.sync()
        slope = torch.ones_like(dy) if act == R.NONE else torch.zeros_like(dy) if act in (R.TANH, R.SIGMOID) else up.to(dtype)
        assert torch.equal(dz, dy * slope)


@pytest.mark.parametrize("act", [R.SILU, R.GELU, R.SIGMOID, R.TANH, R.RELU])
@pytest.mark.parametrize("M,K,N,form", [(44, 136, 72, lf.LF_FORM_SPLIT), (70, 136, 4096, lf.LF_FORM_SPLIT), (2049, 1288, 1800, lf.LF_FORM_PAIRS),
                                        (500, 4000, 4096, lf.LF_FORM_SPLIT_PAIRS)])
def test_gradient_through_the_derivative_at_the_largest_values(ops, act, M, K, N, form):
    q, s, up, _ = _large(M, K)
    g = _gen(M)
    dz, w = _rand(g, M, N, dtype=BF16), _rand(g, N, K, std=N ** -0.5, dtype=BF16)
    dx = torch.empty(M, K, dtype=BF16, device="cuda")
    ops.linear_grad_x(dz, w, dx, q=q, s=s, act=act)
    assert ops.stats()["form"] == form
    ops.sync()
    ref = dz.to(R.D) @ w.to(R.D)
    ref = torch.where(up, ref, 0 * ref) if act not in (R.TANH, R.SIGMOID) else 0 * ref
    R.check("dx", dx, ref, R.rounded(ref, BF16, torch.where(ref != 0, R.product_err(dz.to(R.D), w.to(R.D)), 0 * ref)))


# ---- empty inputs, large offsets, streams, refusals, waits ----------------------------------------------

def test_no_tokens(ops):
    e = lambda n, t=BF16: torch.empty(0, n, dtype=t, device="cuda")   # noqa: E731
    w, u8 = torch.ones(16, 24, dtype=BF16, device="cuda"), torch.uint8
    ops.linear(e(24), w, e(16), q=e(16, u8), s=e(1, u8))
    ops.linear_grad_x(e(16), w, e(24), q=e(24, u8), s=e(1, u8), act=R.GELU)
    for t in (F32, BF16):
        gw, gb = torch.full((16, 24), 7.0, dtype=t, device="cuda"), torch.full((16,), 7.0, device="cuda")
        ops.linear_grad_w(e(16), gw, gb=gb, x=e(24))
        assert gw.eq(0).all() and gb.eq(0).all()
    ops.rms_norm(e(24), torch.ones(24, device="cuda"), e(24))
    dg = torch.full((24,), 7.0, device="cuda")
    ops.rms_norm_backward(e(24), e(24), torch.ones(24, device="cuda"), e(24), dg)
    assert dg.eq(0).all()
    ops.pack8(e(24), e(24, u8), e(1, u8))
    ops.unpack8(e(24, u8), e(1, u8), e(24))
    ops.act_backward(e(24), e(24, u8), e(1, u8), e(24), act=R.RELU)
    ops.sync()


def test_offsets_beyond_32_bits(ops):
    # 140000 x 16384 elements are more than 2^31; the last rows are compared
    M, N, K = 140000, 16384, 8
    g = _gen(12)
    x, w = _rand(g, M, K, dtype=BF16), _rand(g, N, K, std=0.3, dtype=BF16)
    y = torch.empty(M, N, dtype=BF16, device="cuda")
    q, s = torch.empty(M, N, dtype=torch.uint8, device="cuda"), torch.empty(M, N // 32, dtype=torch.uint8, device="cuda")
    ops.linear(x, w, y, q=q, s=s)
    ops.sync()
    last = slice(M - 64, M)
    ref = x[last].to(R.D) @ w.to(R.D).t()
    err = R.product_err(x[last].to(R.D), w.to(R.D).t())
    R.check("y", y[last], ref, R.rounded(ref, BF16, err))
    _check_packed("z8", q[last], s[last], ref, err)
    del q, s
    gain = torch.ones(N, device="cuda")
    n = torch.empty_like(y)
    q, s = torch.empty(M, N, dtype=torch.uint8, device="cuda"), torch.empty(M, N // 32, dtype=torch.uint8, device="cuda")
    ops.rms_norm(y, gain, n, q=q, s=s)
    ops.sync()
    h = y[last].to(R.D)
    ref = h / (h.square().mean(1, keepdim=True) + 1e-5).sqrt()
    R.check("norm", n[last], ref, R.rounded(ref, BF16, 1e-4 * ref.abs()))
    ops.rms_norm_backward(n, y, gain, n)
    ops.unpack8(q, s, y)
    ops.sync()
    assert torch.equal(y[last], R.unpack8(q[last], s[last]).to(BF16))
    assert n[last].isfinite().all()


def test_gradients_and_packing_beyond_32_bits():
    # the same 140000 x 16384 in every matrix over tokens of the other operators.  What is summed over tokens comes from
    # the last 64 rows alone, so that a row fetched from elsewhere shows.
    M, N, K, L = 140000, 16384, 8, 64
    last = slice(M - L, M)
    g = _gen(16)
    empty = lambda *s, d=BF16: torch.empty(*s, dtype=d, device="cuda")   # noqa: E731
    wide, byte = empty(M, N), torch.uint8
    for i in range(0, M, 20000):
        wide[i:i + 20000].normal_(0.0, 1.0, generator=g)
    with lf.Operators(lf.lf_ops_workspace(M, N)) as o:
        q, s, out = empty(M, N, d=byte), empty(M, N // 32, d=byte), torch.full((M, N), float("nan"), dtype=BF16, device="cuda")
        o.pack8(wide, q, s)
        o.act_backward(wide, q, s, out, act=R.GELU)
        o.sync()
        rq, rs = R.pack8(wide[last])
        assert torch.equal(s[last], rs) and bool(((q[last] == rq) | ((q[last] & 0x7F == 0) & (rq & 0x7F == 0))).all())
        z = R.unpack8(q[last], s[last])
        w64 = wide[last].to(R.D)
        ref = w64 * R.act_prime(z, R.GELU)
        R.check("dz", out[last], ref, R.rounded(ref, BF16, 16e-6 * w64.abs() * (1 + z.abs())))
        # dx [M, N] = (dz w) * gelu'(z) + add
        dz, w = _rand(g, M, K, dtype=BF16), _rand(g, K, N, std=0.3, dtype=BF16)
        out.fill_(float("nan"))
        o.linear_grad_x(dz, w, out, q=q, s=s, act=R.GELU, add=wide)
        o.sync()
        d64 = dz[last].to(R.D)
        t, sp = d64 @ w.to(R.D), R.act_prime(z, R.GELU)
        ref = t * sp + w64
        R.check("dx", out[last], ref, R.rounded(ref, BF16, R.product_err(d64, w.to(R.D)) * sp.abs() + 8e-6 * t.abs() + 2.0 ** -24 * ref.abs()))
        # gw [K, N] from 8 bits, through the workspace
        dz[:M - L] = 0
        gw, gb = empty(K, N, d=F32), empty(K, d=F32)
        o.linear_grad_w(dz, gw, gb=gb, q=q, s=s)
        o.sync()
        R.check("gw", gw, d64.t() @ z, R.rounded(d64.t() @ z, F32, R.product_err(d64.t(), z)))
        R.check("gb", gb, d64.sum(0), (L + 340) * 2.0 ** -24 * d64.abs().sum(0))
        del q, s, dz
        # gw [N, K] and gb [N] with a wide dz
        x = _rand(g, M, K, dtype=BF16)
        wide[:M - L] = 0
        gw, gb = empty(N, K, d=F32), empty(N, d=F32)
        o.linear_grad_w(wide, gw, gb=gb, x=x)
        o.sync()
        x64 = x[last].to(R.D)
        R.check("gw", gw, w64.t() @ x64, R.rounded(w64.t() @ x64, F32, R.product_err(w64.t(), x64)))
        R.check("gb", gb, w64.sum(0), (L + 340) * 2.0 ** -24 * w64.abs().sum(0))
        # norm backward: dy (zero but for the last rows), h, dh
        h = empty(M, N)
        for i in range(0, M, 20000):
            h[i:i + 20000].normal_(0.0, 1.0, generator=g)
        gain, dg = 1 + _rand(g, N, std=0.2), empty(N, d=F32)
        out.fill_(float("nan"))
        o.rms_norm_backward(wide, h, gain, out, dg)
        o.sync()
    assert out[:M - L:1000].eq(0).all()
    h64, g64 = h[last].to(R.D), gain.to(R.D)
    rstd = (h64.square().mean(1, keepdim=True) + 1e-5).rsqrt()
    hn, u = h64 * rstd, w64 * g64
    ref = rstd * (u - hn * (u * hn).mean(1, keepdim=True))
    mag = rstd * (u.abs() + hn.abs() * (u * hn).abs().mean(1, keepdim=True))
    R.check("dh", out[last], ref, R.rounded(ref, BF16, ((N / 32 + 16) * 2.0 ** -23 + 2.0 ** -21) * mag))
    R.check("dgain", dg, (w64 * hn).sum(0), (L + 340 + N / 64) * 2.0 ** -24 * (w64 * hn).abs().sum(0))


def test_work_goes_to_the_stream_that_was_set():
    st = torch.cuda.Stream()
    M, K, N = 300, 512, 264
    g = _gen(13)
    x, w = _rand(g, M, K, dtype=BF16), _rand(g, N, K, std=0.05, dtype=BF16)
    y, y2 = (torch.zeros(M, N, dtype=BF16, device="cuda") for _ in range(2))
    torch.cuda.synchronize()
    with lf.Operators(stream=st.cuda_stream) as o:
        graph = torch.cuda.CUDAGraph()          # calls allocate nothing, so they can be captured
        o.linear(x, w, y)
        st.synchronize()
        with torch.cuda.graph(graph, stream=st):
            o.set_stream(torch.cuda.current_stream().cuda_stream)
            o.linear(x, w, y2)
        assert y2.eq(0).all()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, y2) and bool((y != 0).any())
        o.set_stream(None)


def test_a_new_handle_is_ready_for_any_stream():
    # what create queues (counters and the status word set to zero) is done when it returns, whatever was queued before it
    st = torch.cuda.Stream()
    g = _gen(15)
    dz, x = _rand(g, 3000, 520, dtype=BF16), _rand(g, 3000, 64, dtype=BF16)
    gw, gb = torch.empty(520, 64, device="cuda"), torch.empty(520, device="cuda")
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)             # 0.1 s of the default stream
    with lf.Operators(stream=st.cuda_stream) as o:
        assert torch.cuda.default_stream().query()
        o.linear_grad_w(dz, gw, gb=gb, x=x)
        o.sync()
    ref = dz.to(R.D).sum(0)
    R.check("gb", gb, ref, (3000 / 16 + 16) * 2.0 ** -23 * dz.to(R.D).abs().sum(0))


@pytest.mark.parametrize("M,K,N", [(200, 1024, 264), (2049, 512, 1288), (4096, 512, 4096), (512, 4096, 4096)])
def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_right(M, K, N):
    g = _gen(14)
    x, w = _rand(g, M, K, dtype=BF16), _rand(g, N, K, std=0.05, dtype=BF16)
    y, y2 = (torch.empty(M, N, dtype=BF16, device="cuda") for _ in range(2))
    with lf.Operators() as o:
        o.linear(x, w, y)
        o.sync()
        o.set_option(lf.LF_OPT_WAIT_BUDGET_US, 20000)
        o.set_option(lf.LF_OPT_WITHHOLD, 1)
        o.linear(x, w, y2)
        assert lf.lf_ops_sync(o._h) == lf.LF_ETIMEOUT
        assert o.stats()["device_status"] != 0
        o.set_option(lf.LF_OPT_WITHHOLD, 0)
        o.linear(x, w, y2)
        o.sync()
        assert o.stats()["device_status"] == 0
        assert torch.equal(y, y2)


def test_refusals(ops):
    t = lambda *s, d=BF16: torch.zeros(*s, dtype=d, device="cuda")   # noqa: E731
    u8 = torch.uint8
    x, w, y = t(4, 64), t(32, 64), t(4, 32)

    def refused(status, f, *a, **k):
        with pytest.raises(lf.LeapfrogError) as e:
            f(*a, **k)
        assert e.value.status == status, e.value

    for bad in (t(4, 64, d=F32), t(4, 64, d=R.D), t(4, 72), t(64), x.cpu(), t(64, 4).t()):
        refused(lf.LF_EINVAL, ops.linear, bad, w, y)
    refused(lf.LF_EINVAL, ops.linear, x, w, t(4, 32, d=F16))
    refused(lf.LF_EINVAL, ops.linear, x, w, t(5, 32))
    refused(lf.LF_EINVAL, ops.linear, x, w, y, bias=t(32))                       # bias is float32
    refused(lf.LF_EINVAL, ops.linear, x, w, y, act=6)
    refused(lf.LF_EINVAL, ops.linear, x, w, y, act=-1)
    refused(lf.LF_EINVAL, ops.linear, t(4, 60), t(32, 60), y)                    # width not a multiple of 8
    refused(lf.LF_EINVAL, ops.linear, t(4, 68)[:, :64], w, y)                    # rows not 16-byte aligned
    refused(lf.LF_EALIGN, ops.linear, t(4 * 64 + 8)[4:260].view(4, 64), w, y)
    refused(lf.LF_ENULL, ops.linear, x, w, y, q=t(4, 32, d=u8))
    refused(lf.LF_EINVAL, ops.linear, x, w, y, q=t(4, 32, d=u8), s=t(4, 2, d=u8))
    refused(lf.LF_EINVAL, ops.linear, x, t(32, 64)[:, :64].t().contiguous(), y)
    dz, dx, gw = t(4, 32), t(4, 64), t(32, 64, d=F32)
    q, s = t(4, 64, d=u8), t(4, 2, d=u8)
    refused(lf.LF_EINVAL, ops.linear_grad_x, dz, w, dx, act=R.GELU)              # sigma' needs z
    refused(lf.LF_EINVAL, ops.linear_grad_w, dz, gw, x=x, q=q, s=s)              # one form of the input
    refused(lf.LF_EINVAL, ops.linear_grad_w, dz, gw, x=x, act=R.GELU)
    refused(lf.LF_ENULL, ops.linear_grad_w, dz, gw)
    refused(lf.LF_EINVAL, ops.linear_grad_w, dz, t(32, 64, d=F16), x=x)
    with lf.Operators() as small:
        refused(lf.LF_ECAPACITY, small.linear_grad_w, dz, gw, q=q, s=s)
        small.linear_grad_w(dz, gw, x=x)
        small.sync()
    gain = t(64, d=F32)
    refused(lf.LF_ENULL, ops.rms_norm, x, gain)                                  # nothing to write
    refused(lf.LF_EINVAL, ops.rms_norm, x, gain, t(4, 64), eps=-1.0)
    refused(lf.LF_EINVAL, ops.rms_norm, x, gain, t(4, 64), eps=float("nan"))
    refused(lf.LF_EINVAL, ops.rms_norm, t(1, 16392), t(16392, d=F32), t(1, 16392))
    refused(lf.LF_EINVAL, ops.rms_norm_backward, x, x, t(72, d=F32), x)
    refused(lf.LF_ENULL, ops.pack8, x, q, None)
    refused(lf.LF_EINVAL, ops.unpack8, q, s, x, act=17)
    refused(lf.LF_EINVAL, ops.act_backward, x, q, s, t(4, 64, d=F16))
    refused(lf.LF_EINVAL, ops.set_option, lf.LF_OPT_WITHHOLD, 2)
    refused(lf.LF_EINVAL, ops.set_option, lf.LF_OPT_VARIANT, 1)
    refused(lf.LF_EINVAL, lf.Operators, 1024)
    ops.sync()


@pytest.mark.filterwarnings("ignore:Sparse CSR")
def test_tensors_without_memory_of_their_own_are_refused(ops):
    # inside vmap a tensor has no address; the process goes on and the message names the argument
    x, q, s = torch.zeros(3, 4, 64, dtype=BF16, device="cuda"), torch.zeros(4, 64, dtype=torch.uint8, device="cuda"), torch.zeros(4, 2, dtype=torch.uint8, device="cuda")

    def call(v):
        ops.pack8(v, q, s)
        return v

    with pytest.raises(lf.LeapfrogError, match="argument x") as e:
        torch.vmap(call)(x)
    assert e.value.status == lf.LF_EINVAL
    with pytest.raises(lf.LeapfrogError, match="argument x"):
        ops.pack8(x[0].to_sparse_csr(), q, s)
    ops.pack8(x[0], q, s)
    ops.sync()


def test_tensors_of_another_device_are_refused():
    with lf.Operators() as o:
        assert o.stats()["device"] == torch.cuda.current_device()
        x, w, y = (torch.zeros(r, c, dtype=BF16, device="cuda") for r, c in ((4, 64), (32, 64), (4, 32)))
        gain, byte = torch.ones(64, device="cuda"), torch.zeros(4, 64, dtype=torch.uint8, device="cuda")
        scales = torch.zeros(4, 2, dtype=torch.uint8, device="cuda")
        o.linear(x, w, y)
        o.sync()
        o._device += 1                         # as if the handle were another GPU's
        for f, *a in ((o.linear, x, w, y), (o.linear_grad_x, y, w, x), (o.linear_grad_w, y, w), (o.rms_norm, x, gain, x),
                      (o.rms_norm_backward, x, x, gain, x), (o.pack8, x, byte, scales), (o.unpack8, byte, scales, x), (o.act_backward, x, byte, scales, x)):
            with pytest.raises(lf.LeapfrogError, match=f"cuda:{o._device} needed") as e:
                f(*a)
            assert e.value.status == lf.LF_EINVAL


def _written(ops):
    """Every operator as (call, outputs, inputs)."""
    t = lambda r, c, d=BF16: torch.zeros(r, c, dtype=d, device="cuda")     # noqa: E731
    byte = torch.uint8
    x, w, y, dz, dx, r, h = t(4, 64), t(32, 64), t(4, 32), t(4, 32), t(4, 64), t(4, 64), t(4, 64)
    gw, gb, bias, gain, dg = t(32, 64, F32), torch.zeros(32, device="cuda"), torch.zeros(32, device="cuda"), torch.ones(64, device="cuda"), torch.zeros(64, device="cuda")
    qy, sy, qx, sx = t(4, 32, byte), t(4, 1, byte), t(4, 64, byte), t(4, 2, byte)
    return [(lambda: ops.linear(x, w, y, bias=bias, residual=dz, q=qy, s=sy), (y, qy, sy), (x, w, bias, dz)),
            (lambda: ops.linear_grad_x(dz, w, dx, q=qx, s=sx, act=R.GELU, add=r), (dx,), (dz, w, qx, sx, r)),
            (lambda: ops.linear_grad_w(dz, gw, gb=gb, q=qx, s=sx, act=R.GELU), (gw, gb), (dz, qx, sx)),
            (lambda: ops.linear_grad_w(dz, gw, gb=gb, x=x), (gw, gb), (dz, x)),
            (lambda: ops.rms_norm(x, gain, dx, residual=r, h=h, q=qx, s=sx), (dx, h, qx, sx), (x, gain, r)),
            (lambda: ops.rms_norm_backward(x, h, gain, dx, dg, dres=r), (dx, dg), (x, h, gain, r)),
            (lambda: ops.pack8(x, qx, sx), (qx, sx), (x,)),
            (lambda: ops.unpack8(qx, sx, dx), (dx,), (qx, sx)),
            (lambda: ops.act_backward(x, qx, sx, dx, act=R.RELU), (dx,), (x, qx, sx))]


def test_outputs_are_marked_as_written(ops):
    # what autograd goes by to see that a tensor it has kept was overwritten
    for call, outputs, inputs in _written(ops):
        before = [v._version for v in outputs + inputs]
        call()
        assert [v._version for v in outputs] == [b + 1 for b in before[:len(outputs)]]
        assert [v._version for v in inputs] == before[len(outputs):]
    with torch.inference_mode():
        for call, _, _ in _written(ops):
            call()
    ops.sync()
    kept, q, s = torch.zeros(4, 64, device="cuda", requires_grad=True), torch.zeros(4, 64, dtype=torch.uint8, device="cuda"), torch.full((4, 2), 127, dtype=torch.uint8, device="cuda")
    mid = kept * 1.0
    out = mid.square().sum()                   # its gradient needs mid
    ops.unpack8(q, s, mid.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.backward()


def test_a_lazy_copy_is_not_written_through(ops):
    x = torch.ones(4, 64, dtype=BF16, device="cuda")
    q, s = torch.empty(4, 64, dtype=torch.uint8, device="cuda"), torch.empty(4, 2, dtype=torch.uint8, device="cuda")
    ops.pack8(x, q, s)
    lazy, q2, s2 = torch._lazy_clone(x), torch._lazy_clone(q), torch._lazy_clone(s)
    ops.unpack8(q2, s2, lazy, act=R.TANH)      # reads two lazy copies and writes a third
    ops.pack8(lazy, q2, s2)
    ops.sync()
    assert x.eq(1).all() and lazy.eq(0.76171875).all()                     # tanh 1 in bf16
    assert torch.equal(R.unpack8(q, s), x.to(R.D)) and bool((R.unpack8(q2, s2) != 1).all())


@pytest.mark.parametrize("first", ["o.sync()", "ctx.sync()"])
def test_a_call_that_cuda_refuses_is_not_reported_by_the_next_one(first):
    # waiting for a stream that is being captured is refused (and ends the capture); what follows knows nothing of it.  In a
    # process of its own, for the capture's sake.
    code = f"""
        import torch, paper_1801_04928_b200 as lf, lf_inputs
        L, N = 3, 256
        t = {{k: v.cuda() for k, v in lf_inputs.make_inputs(L, N, 1, "uniform", 7, "cpu").items()}}
        new = lambda *s: torch.empty(s, device="cuda")
        z, a, delta, gw, gb = new(L, 1, N), new(L + 1, 1, N), new(L, 1, N), new(L, N, N), new(L, N)
        o, ctx = lf.Operators(), lf.Leapfrog(L, N, 1, 2)
        x, w, y = new(20, 64).bfloat16(), new(64, 64).bfloat16(), new(20, 64).bfloat16()
        variants = (lf.LF_VARIANT_STREAMS, lf.LF_VARIANT_FUSED)
        for v in variants:                     # (first launches set kernels up)
            ctx.set_option(lf.LF_OPT_VARIANT, v)
            ctx.forward(t["w"], t["b"], t["x"], z, a)
            ctx.backward(t["w"], z, a, t["y"], delta, gw, gb)
        for v in variants:
            st, seen = torch.cuda.Stream(), None
            try:
                with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=st):
                    o.set_stream(st.cuda_stream)
                    ctx.set_stream(st.cuda_stream)
                    try:
                        {first}
                    except lf.LeapfrogError as e:
                        seen = e.status
            except RuntimeError:
                pass
            assert seen == lf.LF_ECUDA, seen
            o.set_stream(None)
            ctx.set_stream(None)
            ctx.set_option(lf.LF_OPT_VARIANT, v)
            ctx.forward(t["w"], t["b"], t["x"], z, a)
            ctx.backward(t["w"], z, a, t["y"], delta, gw, gb)
            o.linear(x, w, y)
            ctx.sync()
            o.sync()
    """
    r = subprocess.run([sys.executable, "-c", textwrap.dedent(code)], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
