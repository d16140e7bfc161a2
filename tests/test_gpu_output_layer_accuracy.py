"""Accuracy of layer norm's gradient and of the loss against a teacher where means, offsets and low temperatures make fp32 numbers
cancel: bounds that a form which subtracts first keeps, and one that subtracts rounded products or logarithms does not."""
import pytest
import torch

import operators_ref as R
import output_layer_ref as O
import paper_1801_04928_b200 as lf
from test_gpu_operators import Out, _gen, _rand

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
DTYPES = [F32, BF16, F16]
U = O.U


@pytest.fixture(scope="module")
def ops():
    with lf.Operators() as o:
        yield o


# ---- the norm's gradient --------------------------------------------------------------------------------

def _norm_backward(ops, dy, h, gain, mean, rstd):
    """Results and bounds.  c = (h - m) r is a difference and a product: two roundings of c itself, whatever the mean.  Sums of a row are
    64 additions in a row at most, of a column a hundredth of the rows and 64."""
    M, n = h.shape
    dh, dg, db = Out(M, n, h.dtype), Out(1, n, F32), Out(1, n, F32)
    ops.layer_norm_backward(dy, h, gain, mean, rstd, dh.t, dg.t, db.t)
    ops.sync()
    for o in (dh, dg, db):
        o.check()
    (rh, rg, rb), _ = O.layer_norm_backward(dy, h, gain, mean, rstd)
    u, r = dy.to(R.D) * gain.to(R.D), rstd.to(R.D)[:, None]
    c = (h.to(R.D) - mean.to(R.D)[:, None]) * r
    mu, mc = u.mean(1, keepdim=True), (u * c).mean(1, keepdim=True)
    c_err = 2.001 * U * c.abs()
    mu_err = 66 * U * u.abs().mean(1, keepdim=True)
    mc_err = 66 * U * (u * c).abs().mean(1, keepdim=True) + (u.abs() * c_err).mean(1, keepdim=True)
    dh_err = r * (4 * U * (u.abs() + mu.abs() + (c * mc).abs()) + mu_err + c.abs() * mc_err + c_err * mc.abs())
    adds = (M / 100 + 64) * U
    dg_err = adds * (dy.to(R.D) * c).abs().sum(0) + (dy.abs() * c_err).sum(0)
    R.check("dh", dh.t, rh, R.rounded(rh, h.dtype, dh_err))
    R.check("dgain", dg.t[0], rg, R.rounded(rg, F32, dg_err))
    R.check("dbias", db.t[0], rb, R.rounded(rb, F32, adds * dy.to(R.D).abs().sum(0)))
    return dh.t, dg.t[0], db.t[0]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shift", [0.5, 300.0, -5000.0])
@pytest.mark.parametrize("M,n", [(1, 8), (5, 264), (31, 1032), (17, 8192), (301, 512), (400, 2056), (299, 16384)])
def test_norm_gradient_of_shifted_rows(ops, M, n, shift, dtype):
    g = _gen(M + n)
    h, dy = (_rand(g, M, n, std=2.0) + shift).to(dtype), _rand(g, M, n, std=0.1).to(dtype)
    hd = h.to(R.D)
    mean = hd.mean(1).float()
    rstd = (1 / torch.sqrt(hd.var(1, unbiased=False) + 1e-5)).float()
    _norm_backward(ops, dy, h, 1 + _rand(g, n, std=0.2), mean, rstd)


@pytest.mark.parametrize("M,n", [(3, 264), (40, 1032), (700, 520)])
def test_norm_gradient_of_constant_rows(ops, M, n):
    """h - m is 0, so the gain's gradient is nothing but zeros."""
    g = _gen(n)
    h = torch.linspace(-1000.3, 777.7, M, device="cuda")[:, None].expand(M, n).contiguous()
    rstd = torch.full((M,), 1e-5 ** -0.5, device="cuda")
    _, dg, _ = _norm_backward(ops, _rand(g, M, n), h, 1 + _rand(g, n, std=0.2), h[:, 0].contiguous(), rstd)
    assert bool((dg == 0).all())


# ---- the loss -------------------------------------------------------------------------------------------

def _loss(ops, z, index, value, tau, kind, weight=None):
    """(loss, dz) by one call or by two."""
    loss, lse, dz = Out(1, z.shape[0], F32), Out(1, z.shape[0], F32), Out(*z.shape, z.dtype)
    given = dict(weight=weight, temperature=tau)
    ops.distill(z, index, value, loss.t, lse.t, dz=dz.t if kind == "both" else None, **given)
    if kind == "two calls":
        ops.distill_backward(z, index, value, lse.t, dz.t, **given)
    ops.sync()
    for o in (loss, lse, dz):
        o.check()
    return loss.t[0], dz.t


@pytest.mark.parametrize("kind", ["both", "two calls"])
@pytest.mark.parametrize("V,top", [(700, 40), (40000, 40), (3001, 512)])
@pytest.mark.parametrize("tau", [1.0, 0.5, 0.7])
def test_weights_of_the_teacher(ops, tau, V, top, kind):
    """Where the student gives the entries no mass at all, dz is -T p: p is rounded once, and so is the product, whatever the entries' span."""
    g = _gen(V)
    M = 5
    z = torch.full((M, V), -300.0, device="cuda")
    z[:, 3] = 0.0
    index = torch.stack([4 + torch.randperm(V - 4, generator=g, device="cuda")[:top] for _ in range(M)]).int()
    value = -60.0 * tau * torch.rand(M, top, generator=g, device="cuda")
    _, dz = _loss(ops, z, index, value, tau, kind)
    tau32 = torch.tensor(tau, dtype=F32).item()                   # T as it is handed over
    p = torch.softmax(value.to(R.D) / tau32, 1)
    R.check("dz", dz.gather(1, index.long()), -tau32 * p, 2.001 * U * tau32 * p + 2.0 ** -149)


def _student(g, M, V, std):
    return _rand(g, M, V, std=std)


@pytest.mark.parametrize("kind", ["both", "two calls"])
@pytest.mark.parametrize("M,V", [(16, 1000), (12, 5000), (10, 20001), (9, 50001), (9, 131072), (300, 9000)])
@pytest.mark.parametrize("tau,shift", [(1.0, 0.0), (1.0, 60.0), (1.0, -250.0), (1.0, 900.0), (0.05, 30.0), (3.0, 5000.0)])
def test_gradient_of_shifted_logits(ops, M, V, tau, shift, kind):
    """An offset of a row changes nothing: q is as good as its largest logit and the sum of the differences' exponentials are, however large
    lse is, whose rounding to fp32 alone would be 2^-24 |lse|."""
    g = _gen(V)
    z = _student(g, M, V, 2.0 * tau) + shift
    index = torch.randint(0, V, (M, 3), generator=g, device="cuda").int()
    value = _rand(g, M, 3) * tau
    _, dz = _loss(ops, z, index, value, tau, kind)
    tau32 = torch.tensor(tau, dtype=F32).item()
    x = z.to(R.D) / tau32
    d = x.amax(1, keepdim=True) - x
    q = torch.softmax(x, 1)
    p = torch.softmax(value.to(R.D) / tau32, 1)
    mass = torch.zeros_like(q).scatter_add_(1, index.long(), p)
    ref = tau32 * (q - mass)
    # e^((z - m) / T): the difference, log2(e) / T (2 U) and their product, and 4 U of the function
    e_err = 4 * U * d + 4 * U
    # the sum: of a thread at most seven times 16 terms, seven additions and a change of the maximum each (4 U and once more the terms' own), then 13 over
    # lanes, warps and parts with two more changes
    s_err = (q * (2 * e_err)).sum(1, keepdim=True) + (7 * 7 + 13 + 9 * 4) * U
    err = tau32 * (q * (e_err + s_err + 4 * U) + mass * 4 * U) + 3 * U * ref.abs() + 2.0 ** -120
    R.check("dz", dz, ref, err)


def test_entries_in_another_order_are_refused(ops):
    """As many values as indices, but a row for each entry instead of each token."""
    z, index, value = _rand(_gen(1), 4, 50), torch.zeros(4, 3, dtype=torch.int32, device="cuda"), torch.zeros(4, 3, device="cuda")
    loss, lse, dz = torch.empty(4, device="cuda"), torch.empty(4, device="cuda"), torch.empty(4, 50, device="cuda")
    for bad in (value.t().contiguous(), value.view(2, 6), value.view(4, 3, 1)):
        with pytest.raises(lf.LeapfrogError) as e:
            ops.distill(z, index, bad, loss, lse)
        assert e.value.status == lf.LF_EINVAL and "argument value" in str(e.value)
        with pytest.raises(lf.LeapfrogError) as e:
            ops.distill_backward(z, index, bad, lse, dz)
        assert e.value.status == lf.LF_EINVAL
    ops.distill(z, index, value.view(-1), loss, lse)
    ops.distill_backward(z, index, value, lse, dz)
    ops.sync()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [40, 5000, 70001])
def test_gradient_far_from_zero_by_two_calls(ops, V, dtype):
    """Rows at the type's lowest number and at -60000, where no fp32 lse holds a fraction: every row, and q to its own rounding."""
    g = _gen(V)
    z = torch.full((3, V), torch.finfo(dtype).min, dtype=dtype, device="cuda")
    z[1] = -60000.0
    z[1, ::2] = -60000.0 + (32 if dtype == F16 else 256)
    z[2, 7:] = 0
    index, value = torch.randint(7, V, (3, 5), generator=g, device="cuda").int(), _rand(g, 3, 5)
    q, p = torch.softmax(z.to(R.D), 1), torch.softmax(value.to(R.D), 1)
    mass = torch.zeros_like(q).scatter_add_(1, index.long(), p)
    ref = q - mass
    # differences are 0 or far below any that counts: what is left are the sum (of a thread 7 * 17 additions and changes of the maximum at most where eight parts have
    # the row, 17 times as many where a block has it alone) and a few roundings; weights of 16-bit logits are off by their argument's 3 U and 6 more
    adds = 7 * 11 + 13 + 9 * 4
    if dtype != F32:
        adds = (V // (16 * 256) + 7) * 11 + 13 + 9 * 4
    err = q * (adds + 12) * U + mass * (9 + 3 * value.abs().max()) * U
    for in_place in (False, True):
        loss, lse = torch.empty(3, device="cuda"), torch.empty(3, device="cuda")
        to = z.clone()
        ops.distill(z, index, value, loss, lse)
        ops.distill_backward(to if in_place else z, index, value, lse, to)
        ops.sync()
        R.check("dz", to, ref, R.rounded(ref, dtype, err))


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("M,V", [(60, 20001), (300, 20001), (320, 30000)])
def test_longest_lists_of_many_rows(ops, M, V, in_place):
    """512 entries beside parts of rows that are held in registers or take most of a block's shared memory: each way the same gradient."""
    g = _gen(M)
    z = _student(g, M, V, 2.0)
    index, value = torch.rand(M, V, generator=g, device="cuda").topk(512, 1).indices.int(), _rand(g, M, 512)
    weight = torch.rand(M, generator=g, device="cuda")
    _, dz = _loss(ops, z, index, value, 1.0, "both", weight)
    loss, lse = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    to = z.clone()
    ops.distill(z, index, value, loss, lse, weight=weight)
    ops.distill_backward(to if in_place else z, index, value, lse, to, weight=weight)
    ops.sync()
    w = weight.to(R.D)[:, None]
    q, p = torch.softmax(z.to(R.D), 1), torch.softmax(value.to(R.D), 1)
    mass = torch.zeros_like(q).scatter_add_(1, index.long(), p)
    d = z.to(R.D).amax(1, keepdim=True) - z.to(R.D)
    # as for shifted logits; the weight is one more rounding
    e_err = 4 * U * d + 4 * U
    s_err = (q * (2 * e_err)).sum(1, keepdim=True) + (7 * 7 + 13 + 9 * 4) * U
    err = w * (q * (e_err + s_err + 5 * U) + mass * 5 * U) + 3 * U * (w * (q - mass)).abs() + 2.0 ** -120
    for got in (dz, to):
        R.check("dz", got, w * (q - mass), err)
