"""The layer operators' cases: what is run, on which inputs, and their plain form in elementary torch operations.

Operators: a dense layer with bias, activation and residual (forward), its backward pass from an 8-bit
checkpoint, the root-mean-square norm with the residual's addition (both directions), and the 8-bit
checkpoints of activations themselves.  Sizes: `tokens` rows, `n_in` columns of the input, `n_out`
columns of the output (norms and checkpoints have one width, `n_in`).

The 8-bit form of a matrix: in every row, groups of 32 columns share one power of two 2^e, the smallest
one with max|v| <= 448 * 2^e, and hold e4m3 numbers v * 2^-e rounded to nearest.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
GROUP = 32
EPS = 1e-5
_handle = None


def _case(name, op, tokens, n_in, n_out, dtype, act="none", residual=False, ckpt=False):
    return {"name": name, "op": op, "tokens": tokens, "n_in": n_in, "n_out": n_out, "dtype": dtype, "act": act,
            "residual": residual, "ckpt": ckpt}


def listed():
    return [
        # one new token through a square projection that adds to the residual stream: weights are read once
        _case("linear 1 x 4096 x 4096", "linear", 1, 4096, 4096, "bf16", residual=True),
        # a small decoding batch, widths that are no multiple of any tile
        _case("linear 16 x 1032 x 4104", "linear", 16, 1032, 4104, "f16", act="silu"),
        # a short prompt or a small training batch that keeps its pre-activations in 8 bits
        _case("linear 509 x 4096 x 1024", "linear", 509, 4096, 1024, "bf16", act="relu", residual=True, ckpt=True),
        # the widening layer of a feed-forward block on a full training batch
        _case("linear 8192 x 4096 x 16384", "linear", 8192, 4096, 16384, "bf16", act="gelu"),
        # backward pass of a small network's layer, ragged sizes
        _case("backward 70 x 520 x 1024", "linear_backward", 70, 520, 1024, "f16", act="sigmoid"),
        # backward pass of the narrowing layer of a feed-forward block on a full training batch
        _case("backward 8192 x 16384 x 4096", "linear_backward", 8192, 16384, 4096, "bf16", act="gelu"),
        # the norm in front of a layer for one new token
        _case("norm 1 x 4096", "norm", 1, 4096, 0, "bf16", residual=True, ckpt=True),
        # the same for a full training batch, with the 8-bit copy that the backward pass reads
        _case("norm 16384 x 4096", "norm", 16384, 4096, 0, "bf16", residual=True, ckpt=True),
        # its backward pass in fp32, ragged sizes, nothing on the residual path
        _case("norm backward 999 x 1032", "norm_backward", 999, 1032, 0, "f32"),
        # its backward pass for a full training batch
        _case("norm backward 16384 x 8192", "norm_backward", 16384, 8192, 0, "bf16", residual=True),
        # checkpoint of an fp32 network's activations: packed, read back as activations, applied to a gradient
        _case("checkpoint 256 x 4096", "checkpoint", 256, 4096, 0, "f32", act="sigmoid"),
        # the same for the widest activations of a feed-forward block
        _case("checkpoint 8192 x 16384", "checkpoint", 8192, 16384, 0, "bf16", act="gelu"),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _width(rng, hi=16384):
    return min(hi, max(64, 8 * round(_log(rng, 64, hi) / 8)))


def draw(rng):
    op = rng.choice(["linear", "linear", "linear", "linear_backward", "linear_backward", "norm", "norm_backward", "checkpoint"])
    n_out, act, residual, ckpt = 0, "none", False, False
    if op in ("linear", "linear_backward"):
        dtype = rng.choice(["bf16", "bf16", "f16"])
        act = rng.choice(["none", "gelu", "silu", "relu", "sigmoid", "tanh"])
        most = 8192 * 4096 * 16384
        while True:
            tokens = int(_log(rng, 1, 8192)) if op == "linear" else int(_log(rng, 16, 8192))
            n_in, n_out = _width(rng), _width(rng)
            if tokens * n_in * n_out <= most and tokens * max(n_in, n_out) <= 8192 * 16384:
                break
        if op == "linear":
            residual, ckpt = rng.random() < 0.5, rng.random() < 0.3
    else:
        dtype = rng.choice(["bf16", "f16", "f32"])
        while True:
            tokens, n_in = int(_log(rng, 1, 16384)), _width(rng)
            if tokens * n_in <= (16384 * 8192 if dtype != "f32" else 8192 * 8192):
                break
        if op == "checkpoint":
            act = rng.choice(["none", "gelu", "silu", "relu", "sigmoid", "tanh"])
        else:
            residual = rng.random() < 0.7
            ckpt = op == "norm" and rng.random() < 0.5
    return {"op": op, "tokens": tokens, "n_in": n_in, "n_out": n_out, "dtype": dtype, "act": act, "residual": residual, "ckpt": ckpt}


# ---- inputs ---------------------------------------------------------------------------------------

def _groups(n):
    return (n + GROUP - 1) // GROUP


def _pad(v):
    """[rows, n] -> [rows, groups, 32], zeros behind the end of a row."""
    rows, n = v.shape
    v = torch.cat([v, v.new_zeros((rows, _groups(n) * GROUP - n))], 1) if n % GROUP else v
    return v.reshape(rows, -1, GROUP)


def _to_8_bits(v):
    """The 8-bit form of an fp32 matrix: (e4m3 bytes [rows, n], exponent bytes [rows, groups])."""
    rows, n = v.shape
    g = _pad(v)
    m, e = torch.frexp(g.abs().amax(-1))          # amax = m * 2^e, m in [0.5, 1); 448 = 0.875 * 2^9
    e = torch.where(m == 0, -127, torch.where(m <= 0.875, e - 9, e - 8)).clamp(min=-127)
    q = torch.ldexp(g, -e.unsqueeze(-1)).to(torch.float8_e4m3fn)
    return q.reshape(rows, -1)[:, :n].contiguous().view(torch.uint8), (e + 127).to(torch.uint8)


def _from_8_bits(q, s, dtype=torch.float32):
    rows, n = q.shape
    e = s.to(torch.int32) - 127
    g = _pad(q.view(torch.float8_e4m3fn).to(dtype))
    return torch.ldexp(g, e.unsqueeze(-1).to(dtype) if dtype == torch.float64 else e.unsqueeze(-1)).reshape(rows, -1)[:, :n]


def prepare(case, seed):
    M, K, N, T = case["tokens"], case["n_in"], case["n_out"], DTYPES[case["dtype"]]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=g)

    def activations(rows, n):
        # unit variance, a few columns an order of magnitude larger, as residual streams have them
        v = normal(rows, n)
        wide = torch.randint(0, n, (max(1, n // 256),), generator=g, device="cuda")
        v[:, wide] *= 12.0
        return v

    def out(*shape, dtype=T):
        return torch.empty(shape, dtype=dtype, device="cuda")

    s = dict(case)
    if case["op"] == "linear":
        s["x"] = activations(M, K).to(T)
        s["w"] = normal(N, K, std=K ** -0.5).to(T)
        s["b"] = normal(N, std=0.1)
        s["r"] = normal(M, N).to(T) if case["residual"] else None
        s["y"] = out(M, N)
    elif case["op"] == "linear_backward":
        s["dz"] = normal(M, N, std=0.02).to(T)
        s["w"] = normal(N, K, std=K ** -0.5).to(T)
        s["q"], s["s"] = _to_8_bits(activations(M, K))
        s["dx"] = out(M, K)
        # act(value) is rounded to 16 bits on its way into the products unless it already has so few: then
        # the weight gradient is kept in fp32
        s["gw"] = out(N, K, dtype=torch.float32 if case["act"] in ("none", "relu") else T)
        s["gb"] = out(N, dtype=torch.float32)
    elif case["op"] == "norm":
        s["x"] = activations(M, K).to(T)
        s["r"] = normal(M, K).to(T) if case["residual"] else None
        s["g"] = 1.0 + normal(K, std=0.1)
        s["h"] = out(M, K) if case["residual"] else None
        s["y"] = out(M, K)
    elif case["op"] == "norm_backward":
        s["h"] = activations(M, K).to(T)
        s["g"] = 1.0 + normal(K, std=0.1)
        s["dy"] = normal(M, K, std=0.02).to(T)
        s["r"] = normal(M, K, std=0.02).to(T) if case["residual"] else None
        s["dh"] = out(M, K)
        s["dg"] = out(K, dtype=torch.float32)
    else:
        s["z"] = activations(M, K).to(T)
        s["dy"] = normal(M, K, std=0.02).to(T)
        s["a"] = out(M, K)
        s["dz"] = out(M, K)
    if case["ckpt"] or case["op"] == "checkpoint":
        n = N if case["op"] == "linear" else K
        s["q"] = out(M, n, dtype=torch.uint8)
        s["s"] = out(M, _groups(n), dtype=torch.uint8)
        s["v"] = out(M, n)
    return s


# ---- plain form -----------------------------------------------------------------------------------

def _sigmoid(t):
    return 1.0 / (1.0 + torch.exp(-t))


def _act(z, kind):
    if kind == "sigmoid":
        return _sigmoid(z)
    if kind == "tanh":
        return torch.tanh(z)
    if kind == "relu":
        return torch.clamp(z, min=0.0)
    if kind == "silu":
        return z * _sigmoid(z)
    if kind == "gelu":      # 0.5 z (1 + tanh(u)) = z sigmoid(2 u)
        return z * _sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z))
    return z


def _act_prime(z, kind):
    if kind == "sigmoid":
        a = _sigmoid(z)
        return a * (1.0 - a)
    if kind == "tanh":
        return 1.0 - torch.tanh(z) ** 2
    if kind == "relu":
        return (z > 0).to(z.dtype)
    if kind == "silu":
        a = _sigmoid(z)
        return a + z * a * (1.0 - a)
    if kind == "gelu":
        c = 2.0 * math.sqrt(2.0 / math.pi)
        a = _sigmoid(c * (z + 0.044715 * z * z * z))
        return a + z * a * (1.0 - a) * c * (1.0 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def _plain(s):
    T, act = DTYPES[s["dtype"]], s["act"]
    if s["op"] == "linear":
        z = s["x"].float() @ s["w"].float().t() + s["b"]
        y = _act(z, act)
        res = {"y": (y + s["r"].float() if s["residual"] else y).to(T)}
        if s["ckpt"]:
            res["z8"] = _from_8_bits(*_to_8_bits(z)).to(T)
        return res
    if s["op"] == "linear_backward":
        dz, z = s["dz"].float(), _from_8_bits(s["q"], s["s"])
        dx = (dz @ s["w"].float()) * _act_prime(z, act)
        return {"dx": dx.to(T), "gw": (dz.t() @ _act(z, act)).to(s["gw"].dtype), "gb": dz.sum(0)}
    if s["op"] == "norm":
        h = s["x"].float() + s["r"].float() if s["residual"] else s["x"].float()
        y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s["g"]
        res = {"y": y.to(T)}
        if s["residual"]:
            res["h"] = h.to(T)
        if s["ckpt"]:
            res["y8"] = _from_8_bits(*_to_8_bits(y)).to(T)
        return res
    if s["op"] == "norm_backward":
        h, dy = s["h"].float(), s["dy"].float()
        rstd = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
        hn, u = h * rstd, dy * s["g"]
        dh = rstd * (u - hn * (u * hn).mean(1, keepdim=True))
        return {"dh": (dh + s["r"].float() if s["residual"] else dh).to(T), "dg": (dy * hn).sum(0)}
    z = _from_8_bits(*_to_8_bits(s["z"].float()))
    return {"v": z.to(T), "a": _act(z, act).to(T), "dz": (s["dy"].float() * _act_prime(z, act)).to(T)}


# ---- the framework's operators --------------------------------------------------------------------

def _own(s):
    global _handle
    import paper_1801_04928_b200 as lf
    if _handle is None:
        # one handle for the whole program: a workspace for the largest layer input that is unpacked
        _handle = lf.Operators(workspace_bytes=lf.lf_ops_workspace(8192, 16384))
    ops, act = _handle, getattr(lf, "LF_ACT_" + s["act"].upper())
    if s["op"] == "linear":
        if not s["ckpt"]:
            ops.linear(s["x"], s["w"], s["y"], bias=s["b"], residual=s["r"], act=act)
            return {"y": s["y"]}
        ops.linear(s["x"], s["w"], s["y"], bias=s["b"], residual=s["r"], act=act, q=s["q"], s=s["s"])
        ops.unpack8(s["q"], s["s"], s["v"])
        return {"y": s["y"], "z8": s["v"]}
    if s["op"] == "linear_backward":
        ops.linear_grad_x(s["dz"], s["w"], s["dx"], q=s["q"], s=s["s"], act=act)
        ops.linear_grad_w(s["dz"], s["gw"], gb=s["gb"], q=s["q"], s=s["s"], act=act)
        return {"dx": s["dx"], "gw": s["gw"], "gb": s["gb"]}
    if s["op"] == "norm":
        res = {"y": s["y"]}
        ops.rms_norm(s["x"], s["g"], s["y"], residual=s["r"], h=s["h"], q=s.get("q"), s=s.get("s"), eps=EPS)
        if s["residual"]:
            res["h"] = s["h"]
        if s["ckpt"]:
            ops.unpack8(s["q"], s["s"], s["v"])
            res["y8"] = s["v"]
        return res
    if s["op"] == "norm_backward":
        ops.rms_norm_backward(s["dy"], s["h"], s["g"], s["dh"], s["dg"], dres=s["r"], eps=EPS)
        return {"dh": s["dh"], "dg": s["dg"]}
    ops.pack8(s["z"], s["q"], s["s"])
    ops.unpack8(s["q"], s["s"], s["v"])
    ops.unpack8(s["q"], s["s"], s["a"], act=act)
    ops.act_backward(s["dy"], s["q"], s["s"], s["dz"], act=act)
    return {"v": s["v"], "a": s["a"], "dz": s["dz"]}


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    M, K, N = case["tokens"], case["n_in"], case["n_out"]
    t = 4 if case["dtype"] == "f32" else 2
    packed = lambda n: M * (n + _groups(n))  # noqa: E731
    if case["op"] == "linear":
        b = t * (M * K + N * K + M * N * (2 if case["residual"] else 1)) + 4 * N
        # the checkpoint is written, then read back and returned as values
        return {"bytes": b + (2 * packed(N) + t * M * N if case["ckpt"] else 0), "flops": 2 * M * N * K}
    if case["op"] == "linear_backward":
        gw = 4 if case["act"] in ("none", "relu") else t
        return {"bytes": t * (M * N + N * K + M * K) + gw * N * K + 4 * N + packed(K), "flops": 4 * M * N * K}
    if case["op"] == "norm":
        b = t * M * K * (4 if case["residual"] else 2) + 4 * K
        return {"bytes": b + (2 * packed(K) + t * M * K if case["ckpt"] else 0), "flops": 5 * M * K}
    if case["op"] == "norm_backward":
        return {"bytes": t * M * K * (4 if case["residual"] else 3) + 8 * K, "flops": 10 * M * K}
    # z and dy are read, the packed form is written once and read once, three results are written
    return {"bytes": 5 * t * M * K + 2 * packed(K), "flops": 20 * M * K}


# ---- the definitions in 64 bits -------------------------------------------------------------------

def _exact_act(z, kind):
    """(act(z), act'(z)) in 64 bits; the derivatives are written from tanh, apart from the form above."""
    one = torch.ones_like(z)
    if kind == "tanh":
        a = torch.tanh(z)
        return a, one - a * a
    if kind == "relu":
        return torch.where(z > 0, z, 0.0 * one), torch.where(z > 0, one, 0.0 * one)
    if kind == "none":
        return z, one
    u, du = (math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3), math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z ** 2)) if kind == "gelu" else (z / 2, 0.5 * one)
    t = torch.tanh(u)                       # sigmoid(2 u) = (1 + tanh u) / 2
    a, da = (1 + t) / 2, (1 - t * t) / 2 * du
    return (a, da) if kind == "sigmoid" else (z * a, a + z * da)


def exact(case, seed):
    s = prepare(case, seed)
    D, act = torch.float64, case["act"]
    if case["op"] == "linear":
        z = torch.mm(s["x"].to(D), s["w"].to(D).t()).add_(s["b"].to(D))
        y = _exact_act(z, act)[0]
        res = {"y": y + s["r"].to(D) if case["residual"] else y}
        if case["ckpt"]:
            res["z8"] = z          # what the 8-bit values stand for
        return res
    if case["op"] == "linear_backward":
        dz, z = s["dz"].to(D), _from_8_bits(s["q"], s["s"], D)
        a, da = _exact_act(z, act)
        return {"dx": torch.mm(dz, s["w"].to(D)).mul_(da), "gw": torch.mm(dz.t(), a), "gb": dz.sum(0)}
    if case["op"] == "norm":
        h = s["x"].to(D)
        if case["residual"]:
            h = h + s["r"].to(D)
        y = h / torch.sqrt(h.square().mean(1, keepdim=True) + EPS) * s["g"].to(D)
        res = {"y": y}
        if case["residual"]:
            res["h"] = h
        if case["ckpt"]:
            res["y8"] = y          # what the 8-bit values stand for
        return res
    if case["op"] == "norm_backward":
        # y_j = g_j h_j q^(-1/2), q = mean h^2 + eps:  dh_j = g_j dy_j q^(-1/2) - h_j q^(-3/2) / n * sum_i g_i dy_i h_i
        h, dy, g = s["h"].to(D), s["dy"].to(D), s["g"].to(D)
        q = h.square().mean(1, keepdim=True) + EPS
        dh = g * dy * q ** -0.5 - h * q ** -1.5 / h.shape[1] * (g * dy * h).sum(1, keepdim=True)
        return {"dh": dh + s["r"].to(D) if case["residual"] else dh, "dg": (dy * h * q ** -0.5).sum(0)}
    z = _from_8_bits(*_to_8_bits(s["z"].float()), D)
    a, da = _exact_act(z, act)
    return {"v": z, "a": a, "dz": s["dy"].to(D) * da}
