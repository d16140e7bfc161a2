"""Layer norm, products in 8 bits with a scale for each block of 128 and the loss against a teacher's top logits on the GPU, against
their definitions in 64 bits: values, 8-bit forms, gradients (the formula's and central differences'), ragged sizes, strides, aliases, masks
that leave nothing, empty inputs, values that are not finite, streams and graphs, refusals and waits that run out."""
import math

import pytest
import torch

import operators_ref as R
import output_layer_ref as O
import paper_1801_04928_b200 as lf
from test_gpu_operators import Out, _gen, _rand

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
DTYPES = [F32, BF16, F16]


@pytest.fixture(scope="module")
def ops():
    with lf.Operators() as o:
        yield o


def _blocks(n):
    return (n + 127) // 128


def _ld16(n, extra=0):
    return (n + 15) // 16 * 16 + extra


def _bytes(rows, n, extra=0):
    return Out(rows, n, torch.uint8, _ld16(n, extra))


def _scales(d0, d1):
    return Out(d0, d1, F32)


# ---- layer norm ---------------------------------------------------------------------------------------

def _norm(ops, M, n, dtype, residual=True, bias=True, packed=True, stats=True, plain=True, ld_extra=0, shift=0.7, seed=0):
    g = _gen(100 * M + n + seed)
    x, r = Out(M, n, dtype, n + ld_extra), Out(M, n, dtype, n + 2 * ld_extra)
    x.t.copy_(_rand(g, M, n, std=2.0) + shift)
    r.t.copy_(_rand(g, M, n))
    gain, b = 1 + _rand(g, n, std=0.2), _rand(g, n, std=0.3) if bias else None
    h, y = Out(M, n, dtype, n + ld_extra), Out(M, n, dtype, n)
    q, s = _bytes(M, n, 2 * ld_extra), _scales(_blocks(n), M)
    mean, rstd = Out(1, M, F32), Out(1, M, F32)
    ops.layer_norm(x.t, gain, b, y.t if plain else None, residual=r.t if residual else None, h=h.t if residual else None,
                   q=q.t if packed else None, s=s.t if packed else None, mean=mean.t if stats else None, rstd=rstd.t if stats else None)
    ops.sync()
    for o in (x, r, h, y, q, s, mean, rstd):
        o.check()
    rh, rm, rr, ry = O.layer_norm(x.t, gain, b, r.t if residual else None)
    m_err, r_err, y_err = O.layer_norm_err(rh, rm, rr, ry, gain, b)
    if residual:
        R.check("h", h.t, rh, R.rounded(rh, dtype, O.U * rh.abs()))
    if plain:
        R.check("y", y.t, ry, R.rounded(ry, dtype, y_err))
    if stats:
        R.check("mean", mean.t.t(), rm, R.rounded(rm, F32, m_err))
        R.check("rstd", rstd.t.t(), rr, R.rounded(rr, F32, r_err))
    if packed:
        v, sc = O.values(q.t, s.t), O.spread(s.t, M, n)
        assert bool((torch.frexp(s.t)[0] == 0.5).all())           # a power of two
        # a value is half a step of the format away at most (2^-4 relative, 2^-10 of the scale where e4m3 is subnormal)
        R.check("y8", v, ry, y_err + 2.0 ** -4 * (ry.abs() + y_err) + 2.0 ** -10 * sc)
        for j in range(_blocks(n)):
            amax, err = ry[:, j * 128:(j + 1) * 128].abs().amax(1), y_err[:, j * 128:(j + 1) * 128].amax(1)
            assert bool((amax - err <= 448 * s.t[j]).all()) and bool(((amax + err > 224 * s.t[j]) | (s.t[j] == 2.0 ** -126)).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,n", [(1, 8), (1, 4096), (3, 136), (5, 256), (7, 264), (2, 2056), (300, 72), (301, 512), (299, 1000), (400, 1032),
                                 (333, 4104), (310, 8192), (297, 16384), (9, 16384)])
def test_layer_norm(ops, M, n, dtype):
    _norm(ops, M, n, dtype)


@pytest.mark.parametrize("kw", [dict(residual=False), dict(bias=False), dict(packed=False, stats=False), dict(plain=False), dict(ld_extra=16),
                                dict(shift=300.0), dict(residual=False, bias=False, packed=False)])
@pytest.mark.parametrize("M,n", [(6, 1032), (700, 520)])
def test_layer_norm_forms(ops, M, n, kw):
    _norm(ops, M, n, F32, **kw)
    if kw.get("shift") is None:
        _norm(ops, M, n, BF16, **kw)


def test_layer_norm_in_place(ops):
    g = _gen(3)
    x, r = _rand(g, 50, 1032, dtype=BF16), _rand(g, 50, 1032, dtype=BF16)
    gain, b = 1 + _rand(g, 1032, std=0.2), _rand(g, 1032)
    h, y = torch.empty_like(x), torch.empty_like(x)
    ops.layer_norm(x, gain, b, y, residual=r, h=h)
    x2, r2 = x.clone(), r.clone()
    ops.layer_norm(x2, gain, b, x2, residual=r2, h=r2)
    ops.sync()
    assert torch.equal(x2, y) and torch.equal(r2, h)


def _norm_backward(ops, M, n, dtype, dres=True, dgain=True, dbias=True, ld_extra=0, seed=0):
    g = _gen(77 * M + n + seed)
    dy, h, res = (Out(M, n, dtype, n + k * ld_extra) for k in (1, 2, 3))
    dy.t.copy_(_rand(g, M, n, std=0.1))
    h.t.copy_(_rand(g, M, n, std=2.0) + 0.5)
    res.t.copy_(_rand(g, M, n, std=0.1))
    gain = 1 + _rand(g, n, std=0.2)
    hd = h.t.to(R.D)
    mean = hd.mean(1).float()
    rstd = (1 / torch.sqrt(hd.var(1, unbiased=False) + 1e-5)).float()
    dh, dg, db = Out(M, n, dtype, n + ld_extra), Out(1, n, F32), Out(1, n, F32)
    ops.layer_norm_backward(dy.t, h.t, gain, mean, rstd, dh.t, dg.t if dgain else None, db.t if dbias else None, dres=res.t if dres else None)
    ops.sync()
    for o in (dy, h, res, dh, dg, db):
        o.check()
    ref, err = O.layer_norm_backward(dy.t, h.t, gain, mean, rstd, res.t if dres else None)
    R.check("dh", dh.t, ref[0], R.rounded(ref[0], dtype, err[0]))
    for on, got, r, e in ((dgain, dg, ref[1], err[1]), (dbias, db, ref[2], err[2])):
        if on:
            R.check("column sums", got.t[0], r, R.rounded(r, F32, e))
        else:
            assert bool(got.t.isnan().all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,n", [(1, 8), (1, 4096), (2, 136), (5, 264), (31, 1032), (17, 8192), (3, 16384), (300, 72), (301, 512), (333, 1000), (400, 2056),
                                 (620, 4104), (310, 8192), (299, 16384), (5000, 64)])
def test_layer_norm_backward(ops, M, n, dtype):
    _norm_backward(ops, M, n, dtype)


@pytest.mark.parametrize("kw", [dict(dres=False), dict(dgain=False), dict(dbias=False), dict(dgain=False, dbias=False), dict(ld_extra=16)])
@pytest.mark.parametrize("M,n", [(6, 1032), (700, 520)])
def test_layer_norm_backward_forms(ops, M, n, kw):
    _norm_backward(ops, M, n, F32, **kw)
    _norm_backward(ops, M, n, F16, **kw)


def test_layer_norm_backward_in_place_and_repeatable(ops):
    g = _gen(5)
    M, n = 900, 1032
    dy, h, res = _rand(g, M, n, dtype=BF16), _rand(g, M, n, dtype=BF16), _rand(g, M, n, dtype=BF16)
    gain, mean, rstd = 1 + _rand(g, n, std=0.2), _rand(g, M, std=0.1), 1 + _rand(g, M, std=0.1).abs()
    dh, dg, db = torch.empty_like(dy), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    ops.layer_norm_backward(dy, h, gain, mean, rstd, dh, dg, db, dres=res)
    for which in range(3):
        t = [dy.clone(), h.clone(), res.clone()]
        dg2, db2 = torch.empty_like(dg), torch.empty_like(db)
        ops.layer_norm_backward(t[0], t[1], gain, mean, rstd, t[which], dg2, db2, dres=t[2])
        ops.sync()
        assert torch.equal(t[which], dh) and torch.equal(dg2, dg) and torch.equal(db2, db)


def test_layer_norm_gradient_against_differences(ops):
    g = _gen(8)
    M, n = 3, 40
    x, gain, b, c = _rand(g, M, n), 1 + _rand(g, n, std=0.2), _rand(g, n), _rand(g, M, n)
    mean, rstd, dh, dg, db = torch.empty(M, device="cuda"), torch.empty(M, device="cuda"), torch.empty_like(x), torch.empty_like(gain), torch.empty_like(b)
    ops.layer_norm(x, gain, b, torch.empty_like(x), mean=mean, rstd=rstd)
    ops.layer_norm_backward(c, x, gain, mean, rstd, dh, dg, db)
    ops.sync()

    def f(x, gain, b):
        return (O.layer_norm(x, gain, b)[3] * c.to(R.D)).sum()
    step = 1e-5
    for which, grad in ((0, dh), (1, dg), (2, db)):
        args = [x.to(R.D), gain.to(R.D), b.to(R.D)]
        for i in range(0, args[which].numel(), 7):
            lo, hi = [a.clone() for a in args], [a.clone() for a in args]
            lo[which].view(-1)[i] -= step
            hi[which].view(-1)[i] += step
            d = (f(*hi) - f(*lo)) / (2 * step)
            assert abs(d - grad.view(-1)[i]) < 1e-4 * max(1.0, abs(d)), (which, i)


# ---- blocks of 128 ------------------------------------------------------------------------------------

def _wide_range(g, M, n, dtype):
    v = _rand(g, M, n)
    v *= torch.exp2(torch.randint(-12, 6, (M, 1), generator=g, device="cuda").float())
    v[:, torch.randint(0, n, (max(1, n // 50),), generator=g, device="cuda")] *= 30
    return v.to(dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,n", [(1, 8), (1, 4096), (15, 136), (16, 128), (128, 128), (129, 264), (70, 520), (300, 1032), (1000, 72), (257, 2048)])
def test_pack(ops, M, n, dtype):
    g = _gen(M * 7 + n)
    x = Out(M, n, dtype, n + 8)
    x.t.copy_(_wide_range(g, M, n, dtype))
    for tiles in (False, True):
        for forms in ("both", "q", "qt"):
            q, qt = _bytes(M, n, 16), _bytes(n, M, 32)
            s = _scales(_blocks(M), _blocks(n)) if tiles else _scales(_blocks(n), M)
            st = _scales(_blocks(n), _blocks(M)) if tiles else _scales(_blocks(M), n)
            given = {k: o.t for k, o in dict(q=q, s=s, qt=qt, st=st).items() if forms == "both" or k.endswith("t") == (forms == "qt")}
            (ops.pack_tiles if tiles else ops.pack_blocks)(x.t, **given)
            ops.sync()
            for o in (x, q, s, qt, st):
                o.check()
            if forms != "qt":
                rq, rs = O.pack(x.t, tiles)
                assert torch.equal(s.t, rs) and torch.equal(O.values(q.t, s.t, tiles), O.values(rq, rs, tiles)), (tiles, forms)
            if forms != "q":
                rq, rs = O.pack(x.t.t(), tiles)
                assert torch.equal(st.t, rs) and torch.equal(O.values(qt.t, st.t, tiles), O.values(rq, rs, tiles)), (tiles, forms)


def test_pack_ends_of_the_range(ops):
    """Zeros, the smallest and the largest numbers, borders of a scale, infinities and NaN."""
    x = torch.zeros(8, 256, device="cuda")
    x[1, 3], x[2, 3], x[3, 3], x[4, 3] = 2.0 ** -149, 3.4e38, 448.0, 448.0001
    x[5, 3], x[6, 3], x[7, 3] = math.inf, math.nan, -448.0 * 2.0 ** -126
    q, s, qt, st = _bytes(8, 256), _scales(2, 8), _bytes(256, 8), _scales(1, 256)
    ops.pack_blocks(x, q.t, s.t, qt.t, st.t)
    ops.sync()
    assert s.t[0].tolist()[:5] == [2.0 ** -126, 2.0 ** -126, 2.0 ** 120, 1.0, 2.0] and s.t[0, 7].item() == 2.0 ** -126
    assert bool(s.t[0, 5:7].isnan().all()) and bool((s.t[1] == 2.0 ** -126).all())
    assert bool(st.t[0, 3].isnan()) and bool((st.t[0, 4:] == 2.0 ** -126).all())
    v = O.values(q.t, s.t)
    assert bool(v[5:7, :128].isnan().all()) and bool((v[:, 128:] == 0).all())
    assert v[3, 3] == 448 and v[4, 3] == 448 and v[7, 3] == -448.0 * 2.0 ** -126 and v[0].abs().max() == 0


def _operands(g, M, N, K, tiles, extra=0):
    a, sa = O.pack(_wide_range(g, M, K, F32)) if K else (torch.zeros(M, 0, dtype=torch.uint8, device="cuda"), torch.zeros(0, M, device="cuda"))
    b, sb = O.pack(_wide_range(g, N, K, F32), tiles) if K else (torch.zeros(N, 0, dtype=torch.uint8, device="cuda"), torch.zeros(0, N, device="cuda"))
    # any fp32 number is a scale
    sa, sb = sa * (1 + 0.9 * torch.rand(sa.shape, generator=g, device="cuda")), sb * (1 + 0.9 * torch.rand(sb.shape, generator=g, device="cuda"))
    qa, qb = _bytes(M, K, extra), _bytes(N, K, 2 * extra)
    for o, v in ((qa, a), (qb, b)):
        o.raw.fill_(0x7F)                # NaN behind the rows' ends and around: none of it is to be read
        o.t.copy_(v)
    return qa, sa, qb, sb


def _product(ops, M, N, K, dtype, tiles, bias=True, add=True, extra=0, form=None, seed=0):
    g = _gen(31 * M + 7 * N + K + seed)
    qa, sa, qb, sb = _operands(g, M, N, K, tiles, extra)
    mags = 10.0
    b = _rand(g, N, std=mags) if bias else None
    r = Out(M, N, dtype, N + extra)
    r.t.copy_(_rand(g, M, N, std=mags))
    add = add and dtype != F32
    d = Out(M, N, dtype, N + extra)
    ops.product_blocks(qa.t, sa, qb.t, sb, d.t, bias=b, add=r.t if add else None)
    ops.sync()
    if form:
        assert ops.stats()["form"] == form, ops.stats()
    d.check()
    ref, err = O.product(qa.t, sa, qb.t, sb, tiles) if K else (torch.zeros(M, N, dtype=R.D, device="cuda"), torch.zeros(M, N, dtype=R.D, device="cuda"))
    if bias:
        ref = ref + b.to(R.D)
        err = err + O.U * (ref.abs() + b.abs())
    if add:
        ref = ref + r.t.to(R.D)
        err = err + O.U * ref.abs()
    bound, got = R.rounded(ref, dtype, err), d.t.to(R.D)
    if dtype == F16:
        # beyond 65520 the nearest f16 number is infinity (some sums are: the operands span many magnitudes)
        over = ref.abs() - err >= 65520
        assert torch.equal(got[over], torch.copysign(torch.full_like(got[over], math.inf), ref[over]))
        got = torch.where(over | ((ref.abs() + err >= 65520) & got.isinf()), ref, got)
    R.check(f"d {M}x{K}x{N}", got, ref, bound)


@pytest.mark.parametrize("tiles", [True, False])
@pytest.mark.parametrize("M", [1, 2, 7, 8, 9, 16])
@pytest.mark.parametrize("N,K,dtype", [(8, 1, F32), (40, 64, BF16), (8, 4096, F16), (1032, 520, F16), (264, 131, F32), (4104, 1032, BF16), (5000, 256, F32)])
def test_product_few_tokens(ops, M, N, K, dtype, tiles):
    _product(ops, M, N, K, dtype, tiles, form=lf.LF_FORM_STREAM)


@pytest.mark.parametrize("tiles", [True, False])
@pytest.mark.parametrize("M,N,K,dtype", [(17, 8, 1, F32), (17, 136, 64, F16), (127, 128, 130, BF16), (128, 1024, 1024, BF16), (129, 264, 520, F16), (70, 40, 4096, F32),
                                         (256, 256, 4104, F16), (509, 1024, 2048, BF16), (200, 64, 16384, BF16), (1024, 520, 70, F32)])
def test_product_split_tiles(ops, M, N, K, dtype, tiles):
    _product(ops, M, N, K, dtype, tiles, form=lf.LF_FORM_SPLIT)


@pytest.mark.parametrize("tiles", [True, False])
@pytest.mark.parametrize("M,N,K,dtype", [(2049, 1288, 72, BF16), (1537, 1800, 1024, F16), (4097, 776, 8, F32), (2048, 2048, 2048, BF16), (5000, 1032, 520, F16),
                                         (3000, 3000, 1500, F32), (2500, 4000, 4000, F32)])
def test_product_pairs(ops, M, N, K, dtype, tiles):
    _product(ops, M, N, K, dtype, tiles, form=lf.LF_FORM_PAIRS)


@pytest.mark.parametrize("kw", [dict(bias=False), dict(add=False), dict(bias=False, add=False), dict(extra=16), dict(extra=48)])
@pytest.mark.parametrize("M,N,K", [(5, 520, 200), (100, 520, 200), (2100, 1032, 200)])
def test_product_forms(ops, M, N, K, kw):
    _product(ops, M, N, K, BF16, True, **kw)
    _product(ops, M, N, K, F16, False, **kw)


@pytest.mark.parametrize("tiles", [True, False])
@pytest.mark.parametrize("M,N,K", [(5, 520, 1200), (16, 4104, 200), (100, 520, 4104), (200, 1032, 200), (2100, 2056, 200), (0, 8, 8), (40, 16, 0)])
def test_product_adds_in_place(ops, M, N, K, tiles):
    """`add` may be the very matrix that the result goes to: the bits of a call with one of its own."""
    g = _gen(M + N + K)
    for dtype in (BF16, F16):
        qa, sa, qb, sb = _operands(g, M, N, K, tiles and K > 0)
        add, d, own = Out(M, N, dtype, N + 16), Out(M, N, dtype, N + 16), Out(M, N, dtype, N + 16)
        add.t.copy_(_rand(g, M, N, std=10.0))
        own.t.copy_(add.t)
        ops.product_blocks(qa.t, sa, qb.t, sb, d.t, add=add.t)
        ops.product_blocks(qa.t, sa, qb.t, sb, own.t, add=own.t)
        ops.sync()
        own.check()
        assert torch.equal(own.t, d.t) and bool((own.t != add.t).any()) == (M > 0 and K > 0)


@pytest.mark.parametrize("M", [3, 40])
def test_product_of_nothing(ops, M):
    for dtype in DTYPES:
        _product(ops, M, 72, 0, dtype, False)
        _product(ops, M, 72, 0, dtype, False, bias=False, add=False)


def test_product_infinities_reach_their_rows_and_columns_only(ops):
    for M in (4, 100):
        g = _gen(M)
        x, w = _rand(g, M, 300, dtype=BF16), _rand(g, 72, 300, dtype=BF16)
        x[1, 5] = math.inf
        q, s, wq, ws = _bytes(M, 300), _scales(3, M), _bytes(72, 300), _scales(1, 3)
        d = torch.empty(M, 72, device="cuda")
        with pytest.raises(lf.LeapfrogError):
            ops.pack_blocks(x, q.t, s.t)                  # (300 is no multiple of 8)
        x, w = x[:, :296], w[:, :296].contiguous()
        q, s, wq, ws = _bytes(M, 296), _scales(3, M), _bytes(72, 296), _scales(1, 3)
        ops.pack_blocks(x.contiguous(), q.t, s.t)
        ops.pack_tiles(w, wq.t, ws.t)
        ops.product_blocks(q.t, s.t, wq.t, ws.t, d)
        ops.sync()
        bad = d.isnan().all(1)
        assert bad.tolist() == [i == 1 for i in range(M)] and bool(d[~bad].isfinite().all())


def test_three_products_of_a_layer(ops):
    """Forward and both gradients of y = x w^T from the packed forms, against the same sums of the values they stand for."""
    g = _gen(12)
    T, I, N = 270, 392, 648
    x, w, dz = _rand(g, T, I, dtype=BF16), _rand(g, N, I, std=0.1, dtype=BF16), _rand(g, T, N, dtype=BF16)
    P = {}
    for name, t in (("x", x), ("dz", dz)):
        m, n = t.shape
        P[name] = dict(q=_bytes(m, n).t, s=_scales(_blocks(n), m).t, qt=_bytes(n, m).t, st=_scales(_blocks(m), n).t)
        ops.pack_blocks(t, **P[name])
    P["w"] = dict(q=_bytes(N, I).t, s=_scales(_blocks(N), _blocks(I)).t, qt=_bytes(I, N).t, st=_scales(_blocks(I), _blocks(N)).t)
    ops.pack_tiles(w, **P["w"])
    y, dx, gw = torch.empty(T, N, device="cuda"), torch.empty(T, I, device="cuda"), torch.empty(N, I, device="cuda")
    ops.product_blocks(P["x"]["q"], P["x"]["s"], P["w"]["q"], P["w"]["s"], y)
    ops.product_blocks(P["dz"]["q"], P["dz"]["s"], P["w"]["qt"], P["w"]["st"], dx)
    ops.product_blocks(P["dz"]["qt"], P["dz"]["st"], P["x"]["qt"], P["x"]["st"], gw)
    ops.sync()
    for got, (a, b, tiles) in ((y, (("x", ""), ("w", ""), True)), (dx, (("dz", ""), ("w", "t"), True)), (gw, (("dz", "t"), ("x", "t"), False))):
        ref, err = O.product(P[a[0]]["q" + a[1]], P[a[0]]["s" + a[1]], P[b[0]]["q" + b[1]], P[b[0]]["s" + b[1]], tiles)
        R.check("product", got, ref, R.rounded(ref, F32, err))
        # and the 8-bit forms are close to what was packed: half a step of e4m3 on either side
    full = dz.to(R.D).t() @ x.to(R.D)
    assert ((gw - full).norm() / full.norm()).item() < 2 * 2.0 ** -4


# ---- loss ---------------------------------------------------------------------------------------------

def _student(g, M, V, dtype, ld_extra=0, lead=0):
    z = Out(M, V, dtype, V + ld_extra)
    z.t.copy_(_rand(g, M, V, std=3.0))
    return z


def _teacher(g, M, V, top):
    index = torch.stack([torch.randperm(V, generator=g, device="cuda")[:top] for _ in range(M)]).int()
    return index, _rand(g, M, top, std=2.0) + 5


def _distill(ops, z, index, value, weight, tau, dtype, ld_extra=0, what=("both", "forward", "backward", "in place")):
    M, V = z.t.shape
    ref, err = O.distill(z.t, index, value, weight if weight is not None else torch.ones(M, device="cuda"), tau)
    saved = z.t.clone()
    for kind in what:
        loss, lse, dz = Out(1, M, F32), Out(1, M, F32), Out(M, V, dtype, V + ld_extra)
        given = dict(weight=weight, temperature=tau)
        if kind == "both":
            ops.distill(z.t, index, value, loss.t, lse.t, dz=dz.t, **given)
        elif kind == "in place":
            ops.distill(z.t, index, value, loss.t, lse.t, dz=z.t, **given)
        else:
            ops.distill(z.t, index, value, loss.t, lse.t, **given)
            if kind == "backward":
                ops.distill_backward(z.t, index, value, lse.t, dz.t, **given)
        ops.sync()
        for o in (z, loss, lse, dz):
            o.check()
        R.check("loss " + kind, loss.t[0], ref[0], R.rounded(ref[0], F32, err[0]))
        R.check("lse " + kind, lse.t[0], ref[1], R.rounded(ref[1], F32, err[1]))
        if kind in ("both", "backward"):
            R.check("dz " + kind, dz.t, ref[2], R.rounded(ref[2], dtype, err[2]))
        if kind == "in place":
            R.check("dz " + kind, z.t, ref[2], R.rounded(ref[2], dtype, err[2]))
            z.t.copy_(saved)
        else:
            assert torch.equal(z.t, saved)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,V,top,tau", [(1, 1, 1, 1.0), (3, 7, 7, 2.0), (2, 100, 3, 1.0), (5, 1001, 32, 0.5), (1, 50001, 8, 2.0), (4, 50001, 33, 1.0), (300, 257, 5, 3.5),
                                         (2, 131072, 256, 1.0), (150, 20003, 64, 1.0), (700, 4096, 512, 1.5), (1, 600001, 16, 1.0)])
def test_distill(ops, M, V, top, tau, dtype):
    g = _gen(M + V)
    z = _student(g, M, V, dtype)
    index, value = _teacher(g, M, V, top)
    weight = torch.rand(M, generator=g, device="cuda") + 0.1
    _distill(ops, z, index, value, weight, tau, dtype)
    _distill(ops, z, index, value, None, tau, dtype, what=("both",))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V,ld_extra", [(1000, 8), (1000, 1), (1003, 5), (9999, 3)])
def test_distill_strides(ops, V, ld_extra, dtype):
    g = _gen(V + ld_extra)
    z = _student(g, 9, V, dtype, ld_extra)
    index, value = _teacher(g, 9, V, 20)
    for extra in (0, 1, 8):
        _distill(ops, z, index, value, None, 1.0, dtype, ld_extra=extra, what=("both", "backward"))
    _distill(ops, z, index, value, None, 1.0, dtype, what=("in place",))


@pytest.mark.parametrize("dtype", DTYPES)
def test_distill_lists(ops, dtype):
    """Entries that do not exist, lists of nothing, the same index several times, weights of zero and below, masked logits."""
    g = _gen(4)
    M, V, top = 12, 3001, 40
    z = _student(g, M, V, dtype)
    index, value = _teacher(g, M, V, top)
    index[0, 20:] = -1
    index[1, ::2] = -7
    index[2] = -1                       # nothing
    value[3, 5:] = -math.inf
    value[4] = -math.inf                # nothing
    index[5] = index[5, 0]              # one index, forty times
    index[6, 10:20] = index[6, 0:10]
    index[7, 1:] = -1
    z.t[8, :] = -math.inf
    z.t[8, index[8].long()] = 1.0       # masked logits outside of the list
    z.t[9, 100:2900] = torch.finfo(dtype).min
    index[9] = torch.arange(top, device="cuda")
    weight = torch.rand(M, generator=g, device="cuda")
    weight[10], weight[11] = 0.0, -1.0
    _distill(ops, z, index, value, weight, 1.0, dtype)


@pytest.mark.parametrize("V", [700, 40000])
def test_distill_what_is_not_finite(ops, V):
    g = _gen(V)
    M, top = 8, 6
    z = _student(g, M, V, F32)
    index, value = _teacher(g, M, V, top)
    weight = torch.ones(M, device="cuda")
    z.t[0, 3] = math.nan
    z.t[1, :] = -math.inf
    index[2, 1] = V                     # beyond the vocabulary
    value[3, 0] = math.nan
    z.t[4, 9], weight[4] = math.nan, 0.0
    z.t[5, index[5, 0].long()] = -math.inf      # a wanted logit is impossible: the loss is infinite, the gradient the formula's
    index[6], z.t[6, 9] = -1, math.inf
    for kind in ("both", "backward"):
        loss, lse, dz = Out(1, M, F32), Out(1, M, F32), Out(M, V, F32)
        ops.distill(z.t, index, value, loss.t, lse.t, weight=weight, dz=dz.t if kind == "both" else None)
        if kind == "backward":
            ops.distill_backward(z.t, index, value, lse.t, dz.t, weight=weight)
        ops.sync()
        for r in (0, 1, 2, 3):
            assert bool(loss.t[0, r].isnan()), r
        for r in (0, 1, 2):
            assert bool(dz.t[r].isnan().all()), r
        assert bool(dz.t[3, index[3].long()].isnan().all())
        assert loss.t[0, 4] == 0 and bool((dz.t[4] == 0).all())
        assert loss.t[0, 5] == math.inf and bool(dz.t[5].isfinite().all())
        assert loss.t[0, 6] == 0 and bool((dz.t[6] == 0).all())
        ref, err = O.distill(z.t[7:], index[7:], value[7:], weight[7:], 1.0)
        R.check("dz", dz.t[7:], ref[2], R.rounded(ref[2], F32, err[2]))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", [40, 5000, 70001])
def test_distill_rows_of_the_lowest_number(ops, V, dtype):
    """Every logit masked with the type's lowest number: a uniform softmax; and rows that are shifted as far, in both calls and in place."""
    g = _gen(V)
    low = torch.finfo(dtype).min
    z = torch.full((4, V), low, dtype=dtype, device="cuda")
    z[1] = -60000.0
    z[1, ::2] = -60000.0 + (32 if dtype == F16 else 256)
    z[2, 7:] = 0
    index, value = torch.randint(7, V, (4, 5), generator=g, device="cuda").int(), _rand(g, 4, 5)
    index[:, 4] = index[:, 0]
    weight = torch.ones(4, device="cuda")
    q = torch.softmax(z.to(R.D), 1)
    p = torch.softmax(value.to(R.D), 1)
    dz_ref = q.scatter_add(1, index.long(), -p)
    loss_ref = (p * (p.log() - torch.log_softmax(z.to(R.D), 1).gather(1, index.long()))).sum(1)
    err = 1e-5 * q + 2.0 ** -20 * (p.sum(1, keepdim=True) + 0 * q) * (dz_ref < 0)
    loss, lse, dz = torch.empty(4, device="cuda"), torch.empty(4, device="cuda"), torch.empty_like(z)
    ops.distill(z, index, value, loss, lse, weight=weight, dz=dz)
    R.check("loss", loss[[0, 2, 3]], loss_ref[[0, 2, 3]], 1e-5 * loss_ref[[0, 2, 3]].abs() + 1e-5)
    R.check("dz", dz, dz_ref, R.rounded(dz_ref, dtype, err))
    for in_place in (False, True):
        to = z.clone() if in_place else torch.empty_like(z)
        ops.distill_backward(to if in_place else z, index, value, lse, to, weight=weight)
        ops.sync()
        keep = [0, 2, 3] if dtype == F16 else [0, 1, 2, 3]          # (60000 is not beyond 65536, where lse in fp32 is off by 2^-9)
        R.check("dz backward", to[keep], dz_ref[keep], R.rounded(dz_ref[keep], dtype, err[keep] + 2.0 ** -7 * q[keep]))


def test_distill_gradient_against_differences(ops):
    g = _gen(21)
    M, V, top, tau = 3, 30, 5, 1.7
    z = _student(g, M, V, F32)
    index, value = _teacher(g, M, V, top)
    weight = torch.rand(M, generator=g, device="cuda")
    loss, dz = torch.empty(M, device="cuda"), torch.empty(M, V, device="cuda")
    ops.distill(z.t, index, value, loss, weight=weight, dz=dz, temperature=tau)
    ops.sync()
    for i in range(0, M * V, 4):
        lo, hi = z.t.to(R.D).clone(), z.t.to(R.D).clone()
        lo.view(-1)[i] -= 1e-5
        hi.view(-1)[i] += 1e-5
        d = (O.distill(hi, index, value, weight, tau)[0][0].sum() - O.distill(lo, index, value, weight, tau)[0][0].sum()) / 2e-5
        assert abs(d - dz.reshape(-1)[i]) < 1e-5, i


# ---- empty inputs, streams, graphs, refusals, waits -----------------------------------------------------

def test_no_tokens(ops):
    n = 136
    gain = torch.ones(n, device="cuda")
    e, ef, eb = torch.empty(0, n, dtype=BF16, device="cuda"), torch.empty(0, device="cuda"), torch.empty(0, n, dtype=torch.uint8, device="cuda")
    dg, db = torch.full((n,), 5.0, device="cuda"), torch.full((n,), 5.0, device="cuda")
    ops.layer_norm(e, gain, None, e, mean=ef, rstd=ef, q=eb, s=torch.empty(2, 0, device="cuda"))
    ops.layer_norm_backward(e, e, gain, ef, ef, e, dg, db)
    ops.pack_blocks(e, eb, torch.empty(2, 0, device="cuda"), torch.empty(n, 0, dtype=torch.uint8, device="cuda"), torch.empty(0, n, device="cuda"))
    w, ws = _bytes(8, n), torch.ones(1, 2, device="cuda")
    ops.product_blocks(eb, torch.empty(2, 0, device="cuda"), w.t, ws, torch.empty(0, 8, device="cuda"))
    # a gradient over no tokens is zero
    gw = torch.full((n, 8), 5.0, device="cuda")
    ops.product_blocks(torch.empty(n, 0, dtype=torch.uint8, device="cuda"), torch.empty(0, n, device="cuda"),
                       torch.empty(8, 0, dtype=torch.uint8, device="cuda"), torch.empty(0, 8, device="cuda"), gw)
    ei, ev = torch.empty(0, 3, dtype=torch.int32, device="cuda"), torch.empty(0, 3, device="cuda")
    ops.distill(e, ei, ev, ef, ef, dz=e)
    ops.distill_backward(e, ei, ev, ef, e)
    ops.sync()
    assert bool((dg == 0).all()) and bool((db == 0).all()) and bool((gw == 0).all())


def _run_all(ops, T, I, V, top, buf):
    """Norm, packed result, logits, loss with gradient, both gradients of the weights' product, the norm's gradient."""
    b = buf
    ops.layer_norm(b["x"], b["gain"], b["bias"], residual=b["r"], h=b["h"], y=b["y"], q=b["q"], s=b["s"], mean=b["mean"], rstd=b["rstd"])
    ops.pack_blocks(b["y"], qt=b["yqt"], st=b["yst"])
    ops.pack_tiles(b["w"], b["wq"], b["ws"], b["wqt"], b["wst"])
    ops.product_blocks(b["q"], b["s"], b["wq"], b["ws"], b["z"], bias=b["vb"])
    ops.distill(b["z"], b["index"], b["value"], b["loss"], b["lse"], weight=b["weight"], dz=b["dz"], temperature=2.0)
    ops.pack_blocks(b["dz"], b["dq"], b["ds"], b["dqt"], b["dst"])
    ops.product_blocks(b["dq"], b["ds"], b["wqt"], b["wst"], b["dy"])
    ops.product_blocks(b["dqt"], b["dst"], b["yqt"], b["yst"], b["gw"])
    ops.layer_norm_backward(b["dy"], b["h"], b["gain"], b["mean"], b["rstd"], b["dh"], b["dg"], b["db"])


def _buffers(T, I, V, top, seed=0):
    g = _gen(seed)

    def new(*s, dt=F32):
        return torch.empty(s, dtype=dt, device="cuda")
    b = dict(x=_rand(g, T, I, dtype=BF16), r=_rand(g, T, I, dtype=BF16), gain=1 + _rand(g, I, std=0.1), bias=_rand(g, I, std=0.1),
             w=_rand(g, V, I, std=I ** -0.5, dtype=BF16), vb=_rand(g, V, std=0.1), weight=torch.rand(T, generator=g, device="cuda"))
    b["index"], b["value"] = _teacher(g, T, V, top)
    b.update(h=new(T, I, dt=BF16), y=new(T, I, dt=BF16), mean=new(T), rstd=new(T), q=_bytes(T, I).t, s=new(_blocks(I), T), yqt=_bytes(I, T).t, yst=new(_blocks(T), I),
             wq=_bytes(V, I).t, ws=new(_blocks(V), _blocks(I)), wqt=_bytes(I, V).t, wst=new(_blocks(I), _blocks(V)), z=new(T, V, dt=BF16),
             loss=new(T), lse=new(T), dz=new(T, V, dt=BF16), dq=_bytes(T, V).t, ds=new(_blocks(V), T), dqt=_bytes(V, T).t, dst=new(_blocks(T), V),
             dy=new(T, I, dt=BF16), gw=new(V, I), dh=new(T, I, dt=BF16), dg=new(I), db=new(I))
    return b


@pytest.mark.parametrize("T,I,V,top", [(1, 264, 1000, 5), (70, 520, 2008, 16), (600, 1032, 5000, 64)])
def test_an_output_layer(ops, T, I, V, top):
    """The operators in a row, each held to its definition on what the ones before it left."""
    b = _buffers(T, I, V, top)
    _run_all(ops, T, I, V, top, b)
    ops.sync()
    rh, rm, rr, ry = O.layer_norm(b["x"], b["gain"], b["bias"], b["r"])
    R.check("y", b["y"], ry, R.rounded(ry, BF16, O.layer_norm_err(rh, rm, rr, ry, b["gain"], b["bias"])[2]))
    ref, err = O.product(b["q"], b["s"], b["wq"], b["ws"], True)
    ref = ref + b["vb"].to(R.D)
    R.check("z", b["z"], ref, R.rounded(ref, BF16, err + O.U * (ref.abs() + b["vb"].abs())))
    ref, err = O.distill(b["z"], b["index"], b["value"], b["weight"], 2.0)
    R.check("loss", b["loss"], ref[0], R.rounded(ref[0], F32, err[0]))
    R.check("dz", b["dz"], ref[2], R.rounded(ref[2], BF16, err[2]))
    rq, rs = O.pack(b["dz"].t())
    assert torch.equal(O.values(b["dqt"], b["dst"]), O.values(rq, rs))
    ref, err = O.product(b["dqt"], b["dst"], b["yqt"], b["yst"], False)
    R.check("gw", b["gw"], ref, R.rounded(ref, F32, err))
    ref, err = O.product(b["dq"], b["ds"], b["wqt"], b["wst"], True)
    R.check("dy", b["dy"], ref, R.rounded(ref, BF16, err))
    ref, err = O.layer_norm_backward(b["dy"], b["h"], b["gain"], b["mean"], b["rstd"])
    R.check("dh", b["dh"], ref[0], R.rounded(ref[0], BF16, err[0]))
    R.check("dg", b["dg"], ref[1], R.rounded(ref[1], F32, err[1]))


def test_captured_and_replayed_on_another_stream():
    """A captured run gives the bits of a plain one, with new inputs in the same buffers too, beside another handle's run."""
    sizes = (70, 520, 2008, 16)
    keys = ("h", "y", "z", "loss", "lse", "dz", "dy", "gw", "dh", "dg", "db")
    with lf.Operators() as plain:
        want = []
        for seed in (1, 2):
            b = _buffers(*sizes, seed=seed)
            _run_all(plain, *sizes, b)
            plain.sync()
            want.append({k: b[k].clone() for k in keys})
    stream = torch.cuda.Stream()
    with lf.Operators(stream=stream.cuda_stream) as ops:
        b = _buffers(*sizes, seed=1)
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            _run_all(ops, *sizes, b)
        graph = torch.cuda.CUDAGraph()
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            _run_all(ops, *sizes, b)
        for seed in (1, 2, 1):
            for k, v in _buffers(*sizes, seed=seed).items():
                b[k].copy_(v) if k in ("x", "r", "gain", "bias", "w", "vb", "weight", "index", "value") else b[k].zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for k in keys:
                assert torch.equal(b[k], want[seed - 1][k]), (seed, k)
        del graph


def test_two_handles_at_once():
    """Two handles on two streams, each with a workspace of its own, their kernels side by side: the bits of one after the other."""
    cases = [(16, 1032, 4104, 40), (300, 2056, 3000, 64)]
    with lf.Operators() as plain:
        want = []
        for sizes in cases:
            b = _buffers(*sizes)
            _run_all(plain, *sizes, b)
            plain.sync()
            want.append({k: v.clone() for k, v in b.items()})
    streams = [torch.cuda.Stream() for _ in cases]
    handles = [lf.Operators(stream=s.cuda_stream) for s in streams]
    try:
        bufs = [_buffers(*sizes) for sizes in cases]
        torch.cuda.synchronize()
        for _ in range(10):
            for ops, sizes, b in zip(handles, cases, bufs):
                _run_all(ops, *sizes, b)
        for ops in handles:
            ops.sync()
        for b, w in zip(bufs, want):
            for k in ("h", "y", "z", "loss", "lse", "dz", "dy", "gw", "dh", "dg", "db"):
                assert torch.equal(b[k], w[k]), k
    finally:
        for ops in handles:
            ops.close()


def test_results_do_not_depend_on_timing(ops):
    for sizes in ((16, 1032, 4104, 40), (300, 2056, 3000, 64)):
        b = _buffers(*sizes)
        _run_all(ops, *sizes, b)
        ops.sync()
        first = {k: v.clone() for k, v in b.items()}
        for _ in range(20):
            _run_all(ops, *sizes, b)
        ops.sync()
        for k, v in b.items():
            assert torch.equal(v, first[k]) or k in ("q", "yqt", "wq", "wqt", "dq", "dqt"), k


def test_offsets_beyond_32_bits(ops):
    V, M = 131072, 17000                                            # 2.2e9 logits
    z = torch.zeros(M, V, dtype=BF16, device="cuda")
    index = torch.full((M, 1), V - 1, dtype=torch.int32, device="cuda")
    value, loss, lse = torch.zeros(M, 1, device="cuda"), torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
    z[-1, -1] = 20.0
    ops.distill(z, index, value, loss, lse, dz=z)
    ops.sync()
    l = math.log(V)
    assert bool(((loss[:-1] - l).abs() < 1e-4).all()) and abs(loss[-1].item() - (math.log(math.exp(20) + V - 1) - 20)) < 1e-5
    assert abs(z[-2, -1].float().item() + 1) < 2.0 ** -8 and abs(z[0, 0].float().item() * V - 1) < 2.0 ** -7
    del z
    n, M = 16384, 140000                                            # 2.3e9 values
    x = torch.ones(M, n, dtype=BF16, device="cuda")
    x[-1, -1] = 3.0
    x[-1, 0] = 448.0
    q, s = torch.empty(M, n, dtype=torch.uint8, device="cuda"), torch.empty(n // 128, M, device="cuda")
    ops.pack_blocks(x, q, s)
    ops.sync()
    assert s[0, -1] == 1 and s[127, -1] == 2.0 ** -7 and s[0, 0] == 2.0 ** -8
    assert q[-1, -1:].view(torch.float8_e4m3fn).float().item() == 384 and q[-2, -1:].view(torch.float8_e4m3fn).float().item() == 256


def _refused(f, *a, status=lf.LF_EINVAL, **k):
    with pytest.raises(lf.LeapfrogError) as e:
        f(*a, **k)
    assert e.value.status == status, (e.value.status, status)


def test_refusals(ops):
    n = 136
    x, gain, m = torch.zeros(4, n, device="cuda"), torch.ones(n, device="cuda"), torch.zeros(4, device="cuda")
    q, s = _bytes(4, n).t, torch.zeros(2, 4, device="cuda")
    _refused(ops.layer_norm, x, gain, None, status=lf.LF_ENULL)                              # no result
    _refused(ops.layer_norm, x, gain, None, x, mean=m, status=lf.LF_ENULL)                   # half of a pair
    _refused(ops.layer_norm, x, gain, None, q=q, status=lf.LF_ENULL)
    _refused(ops.layer_norm, x, gain[:8], None, x)
    _refused(ops.layer_norm, x, gain, None, x, eps=-1.0)
    _refused(ops.layer_norm, x, gain, None, x, eps=math.nan)
    _refused(ops.layer_norm, x, gain, None, x.to(BF16))
    _refused(ops.layer_norm, x, gain, None, q=torch.empty(4, n, dtype=torch.uint8, device="cuda"), s=s)   # rows 136 bytes apart
    _refused(ops.layer_norm, x, gain, None, q=q, s=torch.zeros(4, 2, device="cuda"))
    _refused(ops.layer_norm, torch.zeros(1, 16392, device="cuda"), torch.ones(16392, device="cuda"), None, torch.zeros(1, 16392, device="cuda"))
    _refused(ops.layer_norm_backward, x, x, gain, None, m, x, status=lf.LF_ENULL)
    _refused(ops.layer_norm_backward, x, x, gain, m, m[:3], x)
    _refused(ops.pack_blocks, x, status=lf.LF_ENULL)
    _refused(ops.pack_blocks, x, q, status=lf.LF_ENULL)
    _refused(ops.pack_blocks, x, q, torch.zeros(2, 5, device="cuda"))
    _refused(ops.pack_blocks, x.double(), q, s)
    _refused(ops.pack_tiles, x, q, s)                                                        # scales of the other form
    wq, ws, d = _bytes(72, n).t, torch.zeros(1, 2, device="cuda"), torch.zeros(4, 72, device="cuda")
    ops.product_blocks(q, s, wq, ws, d)
    _refused(ops.product_blocks, q, s, wq, torch.zeros(2, 1, device="cuda"), d)
    _refused(ops.product_blocks, q, s, wq[:, :128], ws, d)
    _refused(ops.product_blocks, q, None, wq, ws, d, status=lf.LF_ENULL)
    _refused(ops.product_blocks, q, s, wq, None, d, status=lf.LF_ENULL)
    _refused(ops.product_blocks, q, s, wq, ws, d, add=d)                                     # no residual of an fp32 result
    _refused(ops.product_blocks, q, s, wq[:4], ws, d[:, :4])
    _refused(ops.product_blocks, q, s, wq, ws, d.double())
    _refused(ops.product_blocks, q.float(), s, wq, ws, d)
    z, i, v = torch.zeros(4, 50, device="cuda"), torch.zeros(4, 3, dtype=torch.int32, device="cuda"), torch.zeros(4, 3, device="cuda")
    ops.distill(z, i, v, m)
    for bad in (0.0, -1.0, math.inf, math.nan, 1e-9):
        _refused(ops.distill, z, i, v, m, temperature=bad)
    _refused(ops.distill, z, i, v, None, status=lf.LF_ENULL)
    _refused(ops.distill, z, i.long(), v, m)
    _refused(ops.distill, z, i[:3], v[:3], m)
    _refused(ops.distill, z, i, v[:, :2], m)
    _refused(ops.distill, z, torch.zeros(4, 513, dtype=torch.int32, device="cuda"), torch.zeros(4, 513, device="cuda"), m)
    _refused(ops.distill, z, i[:, :0], v[:, :0], m, status=lf.LF_ENULL)
    _refused(ops.distill, z[:, ::2], i, v, m)
    _refused(ops.distill, z, i, v, m, dz=z.to(F16))
    _refused(ops.distill_backward, z, i, v, None, z, status=lf.LF_ENULL)
    _refused(ops.distill_backward, z, i, v, m, None, status=lf.LF_ENULL)
    ops.sync()


@pytest.mark.parametrize("M,N,K", [(100, 264, 1024), (2600, 2600, 512)])
def test_a_wait_that_runs_out(M, N, K):
    """A stage that is never loaded: the launch ends by itself, the status says so, the next call is clean."""
    with lf.Operators() as ops:
        g = _gen(2)
        qa, sa, qb, sb = _operands(g, M, N, K, True)
        d = torch.empty(M, N, device="cuda")
        ops.set_option(lf.LF_OPT_WAIT_BUDGET_US, 20000)
        ops.set_option(lf.LF_OPT_WITHHOLD, 1)
        ops.product_blocks(qa.t, sa, qb.t, sb, d)
        with pytest.raises(lf.LeapfrogError) as e:
            ops.sync()
        assert e.value.status == lf.LF_ETIMEOUT
        ops.set_option(lf.LF_OPT_WITHHOLD, 0)
        ops.set_option(lf.LF_OPT_WAIT_BUDGET_US, 2000000)
        ops.product_blocks(qa.t, sa, qb.t, sb, d)
        ops.sync()
        ref, err = O.product(qa.t, sa, qb.t, sb, True)
        R.check("after", d, ref, R.rounded(ref, F32, err))


# ---- the layer made of them ----------------------------------------------------------------------------

def _product8(a, b):
    """a b^T of 64-bit matrices and how far the product of their 8-bit forms may be from it: a value is off by 2^-4 of itself, or by
    2^-10 of its block's scale, which is less than 1 / 224 of the largest magnitude."""
    ea, eb = (2.0 ** -4 * v.abs() + 2.0 ** -10 / 224 * v.abs().max() for v in (a, b))
    return a @ b.t(), ea @ (b.abs() + eb).t() + a.abs() @ eb.t()


@pytest.mark.parametrize("tokens,width,vocab", [(3, 64, 264), (130, 264, 1000), (520, 512, 2504)])
def test_output_layer_gradients(tokens, width, vocab):
    from paper_1801_04928_b200.output_layer import OutputLayer
    g = _gen(tokens)
    with lf.Operators() as ops:
        layer = OutputLayer(ops, tokens + 5, width, vocab, seed=tokens)
        layer.master["gain"].add_(_rand(g, width, std=0.2))
        layer.master["shift"].add_(_rand(g, width, std=0.2))
        x, r = _rand(g, tokens, width, dtype=BF16), _rand(g, tokens, width, dtype=BF16)
        index, value = _teacher(g, tokens, vocab, 7)
        weight = torch.rand(tokens, generator=g, device="cuda")
        z, loss, dh = torch.empty(tokens, vocab, dtype=BF16, device="cuda"), torch.empty(tokens, device="cuda"), torch.empty_like(x)
        layer.forward(x, r, z)
        logits = z.clone()
        layer.backward(z, index, value, loss, dh, weight=weight, temperature=2.0)
        ops.sync()
    p, w = layer.master, layer.master["w"].to(R.D)
    rh, rm, rr, ry = O.layer_norm(x, p["gain"], p["shift"], r)
    ref, err = _product8(ry, w)
    R.check("logits", logits, ref, R.rounded(ref, BF16, 1.001 * err))
    ref, err = O.distill(logits, index, value, weight, 2.0)
    R.check("loss", loss, ref[0], R.rounded(ref[0], F32, err[0]))
    R.check("dz", z, ref[2], R.rounded(ref[2], BF16, err[2]))
    dz, u, du = z.to(R.D), layer.u[:tokens].to(R.D), layer.du[:tokens]
    for name, got, (a, b) in (("gw", layer.grad["w"], (dz.t(), u.t())), ("du", du, (dz, w.t()))):
        ref, err = _product8(a.contiguous(), b.contiguous())
        R.check(name, got, ref, R.rounded(ref, got.dtype, 1.001 * err))
    ref, err = O.layer_norm_backward(du, layer.h[:tokens], p["gain"], layer.mean[:tokens], layer.rstd[:tokens])
    for name, got, a, e in (("dh", dh, ref[0], err[0]), ("gain", layer.grad["gain"], ref[1], err[1]), ("shift", layer.grad["shift"], ref[2], err[2])):
        R.check(name, got, a, R.rounded(a, got.dtype, e))


def test_output_layer_runs():
    from paper_1801_04928_b200.output_layer import train
    losses, layer, ops, x, r = train(130, 128, 1000, 8, 3)
    assert all(math.isfinite(v) and v >= 0 for v in losses)
    # one token through the few-token kernels: the same sums in another order
    z, one = torch.empty(130, 1000, dtype=BF16, device="cuda"), torch.empty(1, 1000, dtype=BF16, device="cuda")
    layer.forward(x, r, z, keep=False)
    layer.forward(x[5:6], r[5:6], one, keep=False)
    ops.sync()
    d = (one[0].double() - z[5].double()).abs()
    assert bool((d <= 2 * 2.0 ** -8 * z[5].double().abs() + 1e-4).all())
    ops.close()


OUTPUTS = ("h", "y", "mean", "rstd", "q", "s", "yqt", "yst", "wq", "ws", "wqt", "wst", "z", "loss", "lse", "dz", "dq", "ds", "dqt", "dst", "dy", "gw", "dh", "dg", "db")


def test_every_run_gives_the_same_bits(ops):
    """Each of the runs, all that they write, the 8-bit matrices too: outputs are cleared before a run and compared after it."""
    for sizes in ((16, 1032, 4104, 40), (300, 2056, 3000, 64)):
        b = _buffers(*sizes)
        _run_all(ops, *sizes, b)
        first = {k: b[k].clone() for k in OUTPUTS}
        different = torch.zeros(len(OUTPUTS), dtype=torch.int64, device="cuda")
        for _ in range(20):
            for k in OUTPUTS:
                b[k].zero_()
            _run_all(ops, *sizes, b)
            different += torch.stack([(b[k] != first[k]).sum() for k in OUTPUTS])
        ops.sync()
        assert all(bool(first[k].float().isfinite().all()) for k in OUTPUTS)
        assert not bool(different.any()), dict(zip(OUTPUTS, different.tolist()))


def test_two_handles_at_once_in_every_round():
    """As the runs of two handles side by side, each round of them compared."""
    cases = [(16, 1032, 4104, 40), (300, 2056, 3000, 64)]
    with lf.Operators() as plain:
        want = []
        for sizes in cases:
            b = _buffers(*sizes)
            _run_all(plain, *sizes, b)
            plain.sync()
            want.append({k: b[k].clone() for k in OUTPUTS})
    streams = [torch.cuda.Stream() for _ in cases]
    handles = [lf.Operators(stream=s.cuda_stream) for s in streams]
    try:
        bufs = [_buffers(*sizes) for sizes in cases]
        different = [torch.zeros(len(OUTPUTS), dtype=torch.int64, device="cuda") for _ in cases]
        torch.cuda.synchronize()
        for _ in range(10):
            for ops, sizes, b in zip(handles, cases, bufs):
                _run_all(ops, *sizes, b)
            for s, b, w, d in zip(streams, bufs, want, different):
                with torch.cuda.stream(s):
                    d += torch.stack([(b[k] != w[k]).sum() for k in OUTPUTS])
                    for k in OUTPUTS:
                        b[k].zero_()
        torch.cuda.synchronize()
        for d in different:
            assert not bool(d.any()), dict(zip(OUTPUTS, d.tolist()))
    finally:
        for ops in handles:
            ops.close()


@pytest.mark.parametrize("tokens,width,vocab,temperature", [(300, 264, 1000, 2.0), (40, 512, 2504, 1.0)])
def test_output_layer_gradients_against_automatic_differentiation(tokens, width, vocab, temperature):
    """From the loss to the parameters and the layer's input, all of it differentiated in 64 bits.  An e4m3 number is off by 2^-4 of itself at most, 3.6 % in the mean
    square, a sum of products of two by 5.1 % of its terms' root sum of squares; the logits (of deviation 1.4: x + r has unit variance after the norm, w's
    rows unit length, the gain 1.2) carry 7 % into the softmax, and the gradient one or two more such products: 10 %, and a factor of two for terms that cancel."""
    from paper_1801_04928_b200.output_layer import OutputLayer
    g = _gen(vocab)
    with lf.Operators() as ops:
        layer = OutputLayer(ops, tokens, width, vocab, seed=tokens)
        layer.master["gain"].add_(_rand(g, width, std=0.2))
        layer.master["shift"].add_(_rand(g, width, std=0.2))
        x, r = _rand(g, tokens, width, dtype=BF16), _rand(g, tokens, width, dtype=BF16)
        index, value = _teacher(g, tokens, vocab, 7)
        weight = torch.rand(tokens, generator=g, device="cuda")
        z, loss, dh = torch.empty(tokens, vocab, dtype=BF16, device="cuda"), torch.empty(tokens, device="cuda"), torch.empty_like(x)
        layer.forward(x, r, z)
        layer.backward(z, index, value, loss, dh, weight=weight, temperature=temperature)
        ops.sync()
    leaves = [t.to(R.D).requires_grad_(True) for t in (layer.master["w"], layer.master["gain"], layer.master["shift"], x)]
    w, gain, shift, xd = leaves
    h = xd + r.to(R.D)
    c = h - h.mean(1, keepdim=True)
    u = c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5) * gain + shift
    logq = torch.log_softmax(u @ w.t() / temperature, 1).gather(1, index.clamp(min=0).long())
    p = torch.softmax(value.to(R.D) / temperature, 1)
    assert bool((index >= 0).all())
    each = weight.to(R.D) * temperature ** 2 * (p * (p.log() - logq)).sum(1)
    want = torch.autograd.grad(each.sum(), leaves)
    assert (loss - each).norm() <= 0.2 * each.norm()
    for name, got, ref in zip(("w", "gain", "shift", "x"), (layer.grad["w"], layer.grad["gain"], layer.grad["shift"], dh), want):
        off = ((got.to(R.D) - ref).norm() / ref.norm()).item()
        assert off <= 0.2, (name, off)
