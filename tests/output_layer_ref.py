"""Plain 64-bit forms of layer norm, the 8-bit blocks of 128 and the loss against a teacher's top logits, and the bounds
their results are held to.  No code of the library is used here."""
from __future__ import annotations

import math

import torch

from operators_ref import D

U = 2.0 ** -24                 # half a unit of fp32, relative


def layer_norm(x, gain, bias, residual=None, eps=1e-5):
    h = x.to(D) if residual is None else x.to(D) + residual.to(D)
    m = h.mean(1, keepdim=True)
    r = 1 / torch.sqrt(((h - m) ** 2).mean(1, keepdim=True) + eps)
    y = (h - m) * r * gain.to(D)
    return h, m, r, y if bias is None else y + bias.to(D)


def layer_norm_err(h, m, r, y, gain, bias):
    """Errors before the last rounding of (mean, rstd, y).  A sum of n terms: at most 64 additions in a row (32 a thread, then trees), so
    64 U of the sum of magnitudes; h itself is one fp32 addition."""
    g = 64 * U
    m_err = g * h.abs().mean(1, keepdim=True) + U * h.abs().mean(1, keepdim=True)
    d_err = U * h.abs() + m_err + U * (h - m).abs()
    # the mean square of h - m: each term's error, the sum's, and eps is fp32 (rounded once)
    v = ((h - m) ** 2).mean(1, keepdim=True)
    v_err = 2 * ((h - m).abs() * d_err).mean(1, keepdim=True) + (g + 2 * U) * v + U / r ** 2
    r_err = r * (0.5 * v_err * r ** 2 + 3 * U)
    b = torch.zeros_like(gain) if bias is None else bias
    y_err = gain.abs().to(D) * (r * d_err + (h - m).abs() * r_err) + 3 * U * (y.abs() + b.abs().to(D))
    return m_err, r_err, y_err


def layer_norm_backward(dy, h, gain, mean, rstd, dres=None):
    """(dh, dgain, dbias) and their errors before the last rounding."""
    dy, h, g = dy.to(D), h.to(D), gain.to(D)
    m, r = mean.to(D)[:, None], rstd.to(D)[:, None]
    c, u = (h - m) * r, dy * g
    mu, mc = u.mean(1, keepdim=True), (u * c).mean(1, keepdim=True)
    dh = r * (u - mu - c * mc)
    if dres is not None:
        dh = dh + dres.to(D)
    # c = h r - m r: three roundings; sums of a row: 64 additions in a row at most
    c_err = 2 * U * ((m * r).abs() + (h * r).abs())
    mu_err = (66 * U) * u.abs().mean(1, keepdim=True)
    mc_err = (66 * U) * (u * c).abs().mean(1, keepdim=True) + (u.abs() * c_err).mean(1, keepdim=True)
    dh_err = r * (4 * U * (u.abs() + mu.abs() + (c * mc).abs()) + mu_err + c.abs() * mc_err + c_err * mc.abs()) + U * dh.abs()
    # sums over tokens: a thread adds its own rows (at least 148 blocks share many), then groups and blocks
    adds = (h.shape[0] / 100 + 64) * U
    dg, db = (dy * c).sum(0), dy.sum(0)
    return (dh, dg, db), (dh_err, adds * (dy * c).abs().sum(0) + (dy.abs() * c_err).sum(0), adds * dy.abs().sum(0))


# ---- blocks of 128 ------------------------------------------------------------------------------------

def _exponent(amax):
    """The smallest e >= -126 with amax <= 448 * 2^e, straight from the definition."""
    e = torch.full_like(amax, -126.0)
    for k in range(-125, 121):
        e = torch.where(amax > 448.0 * 2.0 ** (k - 1), torch.full_like(e, float(k)), e)
    return e


def spread(s, rows, n, tiles=False):
    """Scales as a [rows, n] matrix."""
    if tiles:
        return s.to(D).repeat_interleave(128, 0)[:rows].repeat_interleave(128, 1)[:, :n]
    return s.to(D).t().repeat_interleave(128, 1)[:, :n]


def pack(v, tiles=False):
    """(q, s) of the definition for finite values: blocks along rows, or tiles."""
    rows, n = v.shape
    br, bn = -(-rows // 128) if tiles else rows, -(-n // 128)
    pad = torch.zeros(br * 128 if tiles else rows, bn * 128, dtype=D, device=v.device)
    pad[:rows, :n] = v.to(D)
    if tiles:
        e = _exponent(pad.view(br, 128, bn, 128).abs().amax((1, 3)))
        s = torch.exp2(e)
    else:
        s = torch.exp2(_exponent(pad.view(rows, bn, 128).abs().amax(-1))).t()
    q = (v.to(D) / spread(s, rows, n, tiles)).float().to(torch.float8_e4m3fn)
    return q.view(torch.uint8), s.float().contiguous()


def values(q, s, tiles=False):
    return q.contiguous().view(torch.float8_e4m3fn).to(D) * spread(s, *q.shape, tiles)


def product(a, sa, b, sb, tiles):
    """a b^T and the error of its fp32 form.  An instruction aligns 33 summands (32 products and the accumulator) to the largest and
    drops what is below 2^-24 of it: four instructions a block, 4 * 33 U of the sum of magnitudes at most.  Two scales are
    multiplied and applied (2 U), the blocks and parts are added one after the other, and bias and residual."""
    va, vb = values(a, sa), values(b, sb, tiles)
    mags = va.abs() @ vb.abs().t()
    blocks = sa.shape[0]
    return va @ vb.t(), (4 * 33 + 2 + blocks + 24) * U * mags


# ---- loss ---------------------------------------------------------------------------------------------

def distill(z, index, value, weight, tau):
    """(loss, lse, dz) and their errors before the last rounding."""
    tokens, vocab = z.shape
    x = z.to(D) / tau
    m = x.amax(1, keepdim=True)
    lse = torch.logsumexp(x, 1)
    logq = x - lse[:, None]
    there = (index >= 0) & (value != -math.inf)
    at = index.clamp(min=0).long()
    t = torch.where(there, value.to(D) / tau, torch.full_like(value, -math.inf, dtype=D))
    lse_t = torch.logsumexp(t, 1, keepdim=True)
    logp = torch.where(there, t - lse_t, torch.zeros_like(t))
    p = torch.where(there, logp.exp(), torch.zeros_like(t))
    terms = torch.where(p > 0, p * (logp - logq.gather(1, at)), torch.zeros_like(p))
    w = weight.to(D) * there.any(1)
    loss = w * tau ** 2 * terms.sum(1)
    q = logq.exp()
    mass = torch.zeros_like(x).scatter_add_(1, at, p)
    dz = (w * tau)[:, None] * (q - mass)
    # e^x: the argument's roundings (three of its magnitude; where e^x counts it is at most 20) and 4 U of the function; the sum: a
    # thread's additions in a row, then trees
    adds = vocab / 256 + 64
    sum_err = (adds + 4 + 3 * 20) * U
    lse_err = sum_err + U * (m.abs().squeeze(1) * 3)
    arg = torch.where(q > 0, (logq.abs() + x.abs() + lse.abs()[:, None] + m.abs()) * 4 * U, torch.zeros_like(x))     # (masked: q is 0, exactly)
    p_err = p * (8 * U + 4 * U * (t.nan_to_num(neginf=0.0).abs() + lse_t.nan_to_num(neginf=0.0).abs()))
    picked = x.gather(1, at).nan_to_num(neginf=0.0)
    loss_err = w.abs() * tau ** 2 * (lse_err + (p_err * ((t.nan_to_num(neginf=0.0) - picked).abs() + 1)).sum(1) + 4 * U * lse.abs())
    dz_err = (w.abs() * tau)[:, None] * (q * (arg + sum_err + 8 * U) + torch.zeros_like(x).scatter_add_(1, at, p_err)) + 4 * U * dz.abs()
    return (loss, lse, dz), (loss_err, lse_err + U * lse.abs(), dz_err)
