"""Cases, plain forms and 64-bit definitions of the operators of an output layer that is trained from a teacher.

Operators: layer norm with the residual's addition (both directions), matrix products in 8 bits with a scale for
each block of 128 (a dense layer forward, its backward pass, and the layer behind a norm that hands it its 8-bit
form), and the loss against a teacher's top logits with its gradient.  Sizes: `tokens` rows, `n_in` columns of the
input (of the norm), `n_out` columns of the output; the loss has `n_out` logits and `top` of the teacher's.

The 8-bit form: 128 consecutive values of a row (of a column, where the contraction runs over the rows), or a tile of
128 x 128 weights, share a power of two 2^e, the smallest one with max|v| <= 448 * 2^e and e >= -126, and hold e4m3
numbers v * 2^-e rounded to nearest.  Scales are float32 numbers, one line for each block of the contraction.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BLOCK = 128
EPS = 1e-5
_handle = None


def _case(name, op, tokens, n_in, n_out, dtype, residual=False, top=0, temperature=1.0, mode=""):
    return {"name": name, "op": op, "tokens": tokens, "n_in": n_in, "n_out": n_out, "dtype": dtype, "residual": residual,
            "top": top, "temperature": temperature, "mode": mode}


def listed():
    return [
        # the norm in front of a layer for one new token
        _case("norm 1 x 4096", "norm", 1, 4096, 0, "bf16", residual=True),
        # the same for a full training batch, with the statistics that the backward pass reads
        _case("norm 16384 x 4096", "norm", 16384, 4096, 0, "bf16", residual=True),
        # its backward pass in fp32, ragged sizes, nothing on the residual path
        _case("norm backward 999 x 1032", "norm_backward", 999, 1032, 0, "f32"),
        # its backward pass for a full training batch
        _case("norm backward 16384 x 8192", "norm_backward", 16384, 8192, 0, "bf16", residual=True),
        # logits of one new token: norm, then the output layer, weights read once
        _case("head 1 x 4096 x 32768", "head", 1, 4096, 32768, "bf16", residual=True),
        # a small decoding batch, widths that are no multiple of any tile
        _case("linear8 16 x 1032 x 4104", "linear8", 16, 1032, 4104, "f16", residual=True),
        # a short prompt
        _case("linear8 509 x 4096 x 1024", "linear8", 509, 4096, 1024, "bf16"),
        # the widening layer of a feed-forward block on a full training batch
        _case("linear8 8192 x 4096 x 16384", "linear8", 8192, 4096, 16384, "bf16"),
        # backward pass of a small layer, ragged sizes
        _case("backward8 70 x 520 x 1024", "backward8", 70, 520, 1024, "f16"),
        # backward pass of the narrowing layer of a feed-forward block on a full training batch
        _case("backward8 8192 x 16384 x 4096", "backward8", 8192, 16384, 4096, "bf16"),
        # a small batch with an odd vocabulary in fp32, loss and gradient as two calls, as automatic differentiation makes them
        _case("distill 64 x 50001", "distill", 64, 0, 50001, "f32", top=8, temperature=2.0, mode="two calls"),
        # a full training batch with a large vocabulary, loss and gradient at once
        _case("distill 8192 x 131072", "distill", 8192, 0, 131072, "bf16", top=64, mode="at once"),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _width(rng, hi=16384):
    return min(hi, max(64, 8 * round(_log(rng, 64, hi) / 8)))


def draw(rng):
    op = rng.choice(["norm", "norm_backward", "linear8", "linear8", "backward8", "backward8", "head", "distill", "distill"])
    n_in = n_out = top = 0
    residual, temperature, mode = rng.random() < 0.6, 1.0, ""
    dtype = rng.choice(["bf16", "f16", "f32"])
    if op in ("norm", "norm_backward"):
        while True:
            tokens, n_in = int(_log(rng, 1, 16384)), _width(rng)
            if tokens * n_in <= (16384 * 8192 if dtype != "f32" else 8192 * 8192):
                break
    elif op == "distill":
        residual = False
        top, temperature, mode = int(_log(rng, 1, 256)), rng.choice([1.0, 1.0, 2.0, 3.5]), rng.choice(["two calls", "at once"])
        while True:
            tokens, n_out = int(_log(rng, 1, 8192)), int(_log(rng, 1000, 131072))
            if tokens * n_out <= (8192 * 65536 if dtype != "f32" else 4096 * 65536):
                break
    else:
        dtype = "bf16" if op == "head" else rng.choice(["bf16", "bf16", "f16"])
        residual = residual and op != "backward8"
        while True:
            tokens = int(_log(rng, *{"head": (1, 64), "linear8": (1, 8192), "backward8": (16, 8192)}[op]))
            n_in, n_out = _width(rng), _width(rng, 65536 if op == "head" else 16384)
            if tokens * n_in * n_out <= 8192 * 4096 * 16384 and tokens * max(n_in, n_out) <= 8192 * 16384:
                break
    return {"op": op, "tokens": tokens, "n_in": n_in, "n_out": n_out, "dtype": dtype, "residual": residual, "top": top,
            "temperature": temperature, "mode": mode}


# ---- inputs ---------------------------------------------------------------------------------------

def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def _exponent(amax):
    m, e = torch.frexp(amax)                      # amax = m * 2^e, m in [0.5, 1); 448 = 0.875 * 2^9
    return torch.where(m == 0, -126, torch.where(m <= 0.875, e - 9, e - 8)).clamp(min=-126)


def _pad(v, dim):
    """Zeros behind the end, up to whole blocks along `dim`."""
    more = -v.shape[dim] % BLOCK
    if not more:
        return v
    shape = list(v.shape)
    shape[dim] = more
    return torch.cat([v, v.new_zeros(shape)], dim)


def _rows8(v):
    """Values of a matrix in 8 bits, blocks of 128 along its rows, as fp32."""
    rows, n = v.shape
    g = _pad(v, 1).reshape(rows, -1, BLOCK)
    e = _exponent(g.abs().amax(-1, keepdim=True))
    return torch.ldexp(torch.ldexp(g, -e).to(torch.float8_e4m3fn).float(), e).reshape(rows, -1)[:, :n]


def _tiles8(v):
    """Weights in 8 bits, tiles of 128 x 128: (e4m3 bytes [rows, n], scales [row blocks, column blocks])."""
    rows, n = v.shape
    g = _pad(_pad(v, 0), 1).reshape(_blocks(rows), BLOCK, _blocks(n), BLOCK)
    e = _exponent(g.abs().amax((1, 3), keepdim=True))
    q = torch.ldexp(g, -e).to(torch.float8_e4m3fn).reshape(_blocks(rows) * BLOCK, -1)[:rows, :n]
    return q, torch.ldexp(torch.ones_like(e, dtype=torch.float32), e).reshape(_blocks(rows), _blocks(n))


def _tile_values(q, s, dtype=torch.float32):
    rows, n = q.shape
    return q.to(dtype) * s.to(dtype).repeat_interleave(BLOCK, 0).repeat_interleave(BLOCK, 1)[:rows, :n]


def _bytes(rows, n):
    """A matrix of bytes whose rows begin on 16-byte boundaries."""
    return torch.empty(rows, (n + 15) // 16 * 16, dtype=torch.uint8, device="cuda")[:, :n]


def prepare(case, seed):
    M, K, N, T = case["tokens"], case["n_in"], case["n_out"], DTYPES[case["dtype"]]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=g)

    def activations(rows, n):
        # unit variance around a mean, a few columns an order of magnitude larger, as residual streams have them
        v = normal(rows, n) + 0.3
        wide = torch.randint(0, n, (max(1, n // 256),), generator=g, device="cuda")
        v[:, wide] *= 12.0
        return v

    def out(*shape, dtype=T):
        return torch.empty(shape, dtype=dtype, device="cuda")

    def weights():
        # in 8 bits, as they lie and transposed: laid out once, when they change
        q, s = _tiles8(normal(N, K, std=K ** -0.5))
        return q, s

    s, op = dict(case), case["op"]
    f32 = torch.float32
    if op in ("norm", "head"):
        s["x"] = activations(M, K).to(T)
        s["r"] = normal(M, K).to(T) if case["residual"] else None
        s["g"], s["b"] = 1.0 + normal(K, std=0.1), normal(K, std=0.1)
        s["h"] = out(M, K) if case["residual"] else None
        s["y"] = out(M, K if op == "norm" else N)
        if op == "norm":
            s["mean"], s["rstd"] = out(M, dtype=f32), out(M, dtype=f32)
    elif op == "norm_backward":
        s["h"] = activations(M, K).to(T)
        s["g"] = 1.0 + normal(K, std=0.1)
        s["dy"] = normal(M, K, std=0.02).to(T)
        s["r"] = normal(M, K, std=0.02).to(T) if case["residual"] else None
        h = s["h"].double()
        s["mean"] = h.mean(1).float()
        s["rstd"] = torch.rsqrt(h.var(1, unbiased=False) + EPS).float()
        s["dh"], s["dg"], s["db"] = out(M, K), out(K, dtype=f32), out(K, dtype=f32)
    elif op == "distill":
        V, top = N, min(case["top"], N)
        s["z"] = torch.empty((M, V), dtype=T, device="cuda").normal_(0.0, 2.0, generator=g)
        # distinct indices: one in each of `top` equal parts of the vocabulary; some lists are shorter
        part = V // top
        idx = torch.randint(0, part, (M, top), generator=g, device="cuda") + part * torch.arange(top, device="cuda")
        val = 12.0 - 6.0 * torch.rand((M, top), generator=g, device="cuda").sort(1).values
        # the student has learned something already
        s["z"].scatter_(1, idx, (val + normal(M, top)).to(T))
        short = torch.rand((M, 1), generator=g, device="cuda") < 0.1
        idx = torch.where(short & (torch.arange(top, device="cuda") >= (top + 1) // 2), -1, idx)
        s["idx"], s["val"] = idx.int(), val
        # padding has no weight; what has, counts as a mean over the batch (f16 gradients are kept in range by a loss scale)
        s["weight"] = (torch.rand((M,), generator=g, device="cuda") < 0.95).float() * ((1024.0 if T == torch.float16 else 1.0) / M)
        s["loss"], s["lse"], s["dz"] = out(M, dtype=f32), out(M, dtype=f32), out(M, V)
    else:
        s["x"] = activations(M, K).to(T)
        if op == "linear8":
            s["b"] = normal(N, std=0.1)
            s["r"] = normal(M, N).to(T) if case["residual"] else None
            s["y"] = out(M, N)
        else:
            s["dz"] = normal(M, N, std=0.02).to(T)
            s["dx"], s["gw"] = out(M, K), out(N, K, dtype=f32)
            s["dzq"], s["dzs"] = _bytes(M, N), out(_blocks(N), M, dtype=f32)
            s["dzqt"], s["dzst"] = _bytes(N, M), out(_blocks(M), N, dtype=f32)
            s["xqt"], s["xst"] = _bytes(K, M), out(_blocks(M), K, dtype=f32)
    if op in ("head", "linear8", "backward8"):
        q, scales = weights()
        s["w"], s["ws"] = q, scales
        if op == "backward8":                   # the transposed form is what its products read
            s["wq"], s["wqs"] = _bytes(K, N), scales.t().contiguous()
            s["wq"].copy_(q.view(torch.uint8).t())
        else:
            s["wq"], s["wqs"] = _bytes(N, K), scales
            s["wq"].copy_(q.view(torch.uint8))
            s["xq"], s["xs"] = _bytes(M, K), out(_blocks(K), M, dtype=f32)
    return s


# ---- plain form -----------------------------------------------------------------------------------

def _plain_norm(s):
    h = s["x"].float() + s["r"].float() if s["residual"] else s["x"].float()
    mean = h.mean(1, keepdim=True)
    d = h - mean
    rstd = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
    return h, mean, rstd, d * rstd * s["g"] + s["b"]


def _plain(s):
    T, op = DTYPES[s["dtype"]], s["op"]
    if op == "norm":
        h, mean, rstd, y = _plain_norm(s)
        res = {"y": y.to(T), "mean": mean.squeeze(1), "rstd": rstd.squeeze(1)}
        if s["residual"]:
            res["h"] = h.to(T)
        return res
    if op == "norm_backward":
        dy, rstd = s["dy"].float(), s["rstd"].unsqueeze(1)
        hn, u = (s["h"].float() - s["mean"].unsqueeze(1)) * rstd, dy * s["g"]
        dh = rstd * (u - u.mean(1, keepdim=True) - hn * (u * hn).mean(1, keepdim=True))
        return {"dh": (dh + s["r"].float() if s["residual"] else dh).to(T), "dg": (dy * hn).sum(0), "db": dy.sum(0)}
    if op == "head":
        h, _, _, y = _plain_norm(s)
        res = {"y": (_rows8(y) @ _tile_values(s["w"], s["ws"]).t()).to(T)}
        if s["residual"]:
            res["h"] = h.to(T)
        return res
    if op == "linear8":
        y = _rows8(s["x"].float()) @ _tile_values(s["w"], s["ws"]).t() + s["b"]
        return {"y": (y + s["r"].float() if s["residual"] else y).to(T)}
    if op == "backward8":
        dz, x = s["dz"].float(), s["x"].float()
        return {"dx": (_rows8(dz) @ _tile_values(s["w"], s["ws"])).to(T), "gw": _rows8(dz.t()) @ _rows8(x.t()).t()}
    # the loss: a difference of numbers larger than itself, so what there is one of for each entry is in 64 bits
    tau, w = s["temperature"], s["weight"]
    have, at = s["idx"] >= 0, s["idx"].clamp(min=0).long()
    t = torch.where(have, s["val"].double() / tau, -math.inf)
    t = t - t.amax(1, keepdim=True)
    p = torch.exp(t) / torch.exp(t).sum(1, keepdim=True)
    x = s["z"].float() / tau
    picked = s["z"].gather(1, at).double() / tau
    m = x.amax(1, keepdim=True)
    e = torch.exp(x.sub_(m))
    total = e.sum(1, keepdim=True)
    lse = m.double() + torch.log(total.double())
    logp = t - torch.log(torch.exp(t).sum(1, keepdim=True))
    kl = torch.where(have, p * (logp - picked + lse), 0.0).sum(1)
    dz = e.div_(total).scatter_add_(1, at, -torch.where(have, p, 0.0).float()).mul_((w * tau).unsqueeze(1))
    return {"loss": (kl * tau * tau * w).float(), "lse": lse.squeeze(1).float(), "dz": dz.to(T)}


# ---- the framework's operators --------------------------------------------------------------------

def _own(s):
    global _handle
    import paper_1801_04928_b200 as lf
    if _handle is None:
        _handle = lf.Operators()
    ops, op = _handle, s["op"]
    if op == "norm":
        ops.layer_norm(s["x"], s["g"], s["b"], s["y"], residual=s["r"], h=s["h"], mean=s["mean"], rstd=s["rstd"], eps=EPS)
        res = {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    elif op == "norm_backward":
        ops.layer_norm_backward(s["dy"], s["h"], s["g"], s["mean"], s["rstd"], s["dh"], s["dg"], s["db"], dres=s["r"])
        return {"dh": s["dh"], "dg": s["dg"], "db": s["db"]}
    elif op == "head":
        ops.layer_norm(s["x"], s["g"], s["b"], residual=s["r"], h=s["h"], q=s["xq"], s=s["xs"], eps=EPS)
        ops.product_blocks(s["xq"], s["xs"], s["wq"], s["wqs"], s["y"])
        res = {"y": s["y"]}
    elif op == "linear8":
        ops.pack_blocks(s["x"], q=s["xq"], s=s["xs"])
        ops.product_blocks(s["xq"], s["xs"], s["wq"], s["wqs"], s["y"], bias=s["b"], add=s["r"])
        return {"y": s["y"]}
    elif op == "backward8":
        ops.pack_blocks(s["dz"], q=s["dzq"], s=s["dzs"], qt=s["dzqt"], st=s["dzst"])
        ops.pack_blocks(s["x"], qt=s["xqt"], st=s["xst"])
        ops.product_blocks(s["dzq"], s["dzs"], s["wq"], s["wqs"], s["dx"])
        ops.product_blocks(s["dzqt"], s["dzst"], s["xqt"], s["xst"], s["gw"])
        return {"dx": s["dx"], "gw": s["gw"]}
    else:
        given = dict(lse=s["lse"], weight=s["weight"], temperature=s["temperature"])
        if s["mode"] == "at once":
            ops.distill(s["z"], s["idx"], s["val"], s["loss"], dz=s["dz"], **given)
        else:
            ops.distill(s["z"], s["idx"], s["val"], s["loss"], **given)
            ops.distill_backward(s["z"], s["idx"], s["val"], dz=s["dz"], **given)
        return {"loss": s["loss"], "lse": s["lse"], "dz": s["dz"]}
    if s["residual"]:
        res["h"] = s["h"]
    return res


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    M, K, N = case["tokens"], case["n_in"], case["n_out"]
    t = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "norm":
        return {"bytes": t * M * K * (4 if case["residual"] else 2) + 8 * K + 8 * M, "flops": 8 * M * K}
    if case["op"] == "norm_backward":
        return {"bytes": t * M * K * (4 if case["residual"] else 3) + 12 * K + 8 * M, "flops": 14 * M * K}
    if case["op"] == "head":            # the 8-bit form between the two is no output
        return {"bytes": t * M * K * (3 if case["residual"] else 1) + N * K + t * M * N, "flops": 2 * M * N * K}
    if case["op"] == "linear8":
        return {"bytes": t * (M * K + M * N * (2 if case["residual"] else 1)) + N * K + 4 * N, "flops": 2 * M * N * K}
    if case["op"] == "backward8":
        return {"bytes": t * (M * N + 2 * M * K) + N * K + 4 * N * K, "flops": 4 * M * N * K}
    return {"bytes": 2 * t * M * N + 8 * M * case["top"] + 12 * M, "flops": 6 * M * N}


# ---- the definitions in 64 bits -------------------------------------------------------------------

def _exact8(v, tile=False):
    """What the 8-bit form of a 64-bit matrix stands for: blocks of 128 along rows, or tiles; written from the definition."""
    res = torch.empty_like(v)
    for i in range(0, v.shape[1], BLOCK):
        for j in range(0, v.shape[0], BLOCK) if tile else (0,):
            b = v[j:j + BLOCK, i:i + BLOCK] if tile else v[:, i:i + BLOCK]
            amax = b.abs().amax() if tile else b.abs().amax(1, keepdim=True)
            e = torch.ceil(torch.log2(amax / 448.0)).clamp(min=-126.0)
            e = torch.where(amax > 448.0 * torch.exp2(e), e + 1, torch.where((amax <= 224.0 * torch.exp2(e)) & (e > -126), e - 1, e))
            a = b * torch.exp2(-e)
            # three bits behind the leading one; steps of 2^-9 below 2^-6
            step = torch.exp2(torch.floor(torch.log2(a.abs().clamp(min=2.0 ** -6))) - 3)
            (res[j:j + BLOCK, i:i + BLOCK] if tile else res[:, i:i + BLOCK]).copy_(torch.round(a / step) * step * torch.exp2(e))
    return res


def exact(case, seed):
    s = prepare(case, seed)
    D, op = torch.float64, case["op"]

    def weights():
        return s["w"].to(D) * s["ws"].to(D).repeat_interleave(BLOCK, 0)[:s["w"].shape[0]].repeat_interleave(BLOCK, 1)[:, :s["w"].shape[1]]

    if op in ("norm", "head"):
        h = s["x"].to(D)
        if case["residual"]:
            h = h + s["r"].to(D)
        mean, var = h.mean(1), h.var(1, unbiased=False)
        y = (h - mean[:, None]) / torch.sqrt(var + EPS)[:, None] * s["g"].to(D) + s["b"].to(D)
        res = {"y": y, "mean": mean, "rstd": 1 / torch.sqrt(var + EPS)} if op == "norm" else {"y": _exact8(y) @ weights().t()}
        if case["residual"]:
            res["h"] = h
        return res
    if op == "norm_backward":
        # y_j = g_j (h_j - m) r:  dh_j = r g_j dy_j - r / n sum_i g_i dy_i - (h_j - m) r^3 / n sum_i g_i dy_i (h_i - m)
        c, r, n = s["h"].to(D) - s["mean"].to(D)[:, None], s["rstd"].to(D)[:, None], case["n_in"]
        u = s["dy"].to(D) * s["g"].to(D)
        dh = r * u - r / n * u.sum(1, keepdim=True) - c * r ** 3 / n * (u * c).sum(1, keepdim=True)
        return {"dh": dh + s["r"].to(D) if case["residual"] else dh, "dg": (s["dy"].to(D) * c * r).sum(0), "db": s["dy"].to(D).sum(0)}
    if op == "linear8":
        y = torch.mm(_exact8(s["x"].to(D)), weights().t()).add_(s["b"].to(D))
        return {"y": y + s["r"].to(D) if case["residual"] else y}
    if op == "backward8":
        dz, x = s["dz"].to(D), s["x"].to(D)
        return {"dx": torch.mm(_exact8(dz), weights()), "gw": torch.mm(_exact8(dz.t().contiguous()), _exact8(x.t().contiguous()).t())}
    # loss = w T^2 sum_k p_k (ln p_k - ln q_k), p and q softmaxes at temperature T; dz = w T (q - p)
    tau, w = case["temperature"], s["weight"].to(D)
    logq = torch.log_softmax(s["z"].to(D).div_(tau), 1)
    lse = s["z"][:, 0].to(D) / tau - logq[:, 0]
    have, at = s["idx"] >= 0, s["idx"].clamp(min=0).long()
    logp = torch.log_softmax(torch.where(have, s["val"].to(D) / tau, -math.inf), 1)
    terms = torch.where(have, logp.exp() * (logp - logq.gather(1, at)), 0.0)
    dz = logq.exp_().scatter_add_(1, at, -torch.where(have, logp.exp(), 0.0)).mul_((w * tau)[:, None])
    return {"loss": w * tau * tau * terms.sum(1), "lse": lse, "dz": dz}
