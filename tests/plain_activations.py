"""The activation operators from their formulas, in 64 bits (torch.float64 on any device), and bounds on what binary32 may be off."""
import math

import torch

U = 2.0 ** -24                       # half a step of binary32 at 1


def half_step(t):
    return torch.finfo(t).eps / 2


def ckpt_fields(x):
    """x [rows, cols]: (codes uint8 [rows, pitch], scales uint8 [rows, pitch / 32], values float64 [rows, cols])."""
    rows, cols = x.shape
    pitch = (cols + 31) // 32 * 32
    v = torch.zeros(rows, pitch, dtype=torch.float64)
    v[:, :cols] = x.double().cpu()
    v = v.reshape(rows, -1, 32)
    top = v.abs().amax(2, keepdim=True)
    bad = ~torch.isfinite(top) | torch.isnan(v).any(2, keepdim=True)
    v = torch.where(bad, torch.zeros_like(v), v)
    top = torch.where(bad, torch.zeros_like(top), top)
    e = torch.where(top > 0, torch.frexp(top).exponent - 1 + 127 - 8, torch.zeros_like(top, dtype=torch.int32)).clamp(10, 246).to(torch.int64)
    power = ((e - 127 + 1023) << 52).view(torch.float64)
    w = v / power
    octave = torch.frexp(w).exponent - 1                                     # of each entry; steps stay those of 2^-6 below it
    step = ((octave.clamp(min=-6).to(torch.int64) - 3 + 1023) << 52).view(torch.float64)
    r = (torch.round(w / step) * step).clamp(-448.0, 448.0)
    m = r.abs()
    fr = torch.frexp(m)
    oct_r = fr.exponent.to(torch.int64) - 1
    code = torch.where(m < 2.0 ** -6, (m * 512).to(torch.int64), ((oct_r + 7) << 3) + ((fr.mantissa * 2 - 1) * 8).to(torch.int64))
    code = code + torch.where(torch.signbit(v), 128, 0)
    code = torch.where(bad, torch.full_like(code, 127), code)
    e = torch.where(bad, torch.full_like(e, 255), e)
    values = torch.where(bad, torch.full_like(r, math.nan), r * power)
    return code.to(torch.uint8).reshape(rows, pitch), e.to(torch.uint8).reshape(rows, -1), values.reshape(rows, pitch)[:, :cols].to(x.device)


def held(x):
    return ckpt_fields(x.reshape(-1, x.shape[-1]))[2].reshape(x.shape)


def layer_norm(x, weight, bias, eps):
    x = x.double()
    mean = x.mean(-1, keepdim=True)
    rstd = 1 / torch.sqrt((x - mean).square().mean(-1, keepdim=True) + eps)
    y = (x - mean) * rstd
    if weight is not None:
        y = y * weight.double()
    if bias is not None:
        y = y + bias.double()
    return y, mean, rstd


def depth(cols):
    """Additions that follow each other at most in a row's sum: a lane's own (64 lanes at least), then the lanes', then the waves'."""
    return cols / 64 + 40


def layer_norm_bound(x, weight, bias, eps, out):
    """How far y may be off, and the relative error of rstd and the absolute one of the mean."""
    y, mean, rstd = layer_norm(x, weight, bias, eps)
    x = x.double()
    dm = (depth(x.shape[-1]) + 2) * U * x.abs().mean(-1, keepdim=True)
    dk = (depth(x.shape[-1]) + 8) * U + (dm * rstd) ** 2 + dm * rstd * 2 * (dm * rstd + U)
    w = 1.0 if weight is None else weight.double().abs()
    n = (x - mean).abs() * rstd
    off = w * (rstd * (1 + dk) * (dm + U * (x.abs() + mean.abs())) + n * (dk + 3 * U))
    b = 0.0 if bias is None else bias.double().abs()
    return off + 2 * U * (w * n + b) + half_step(out) * (y.abs() + off), dk, dm


def layer_norm_grad(dy, xv, mean, rstd, weight):
    """dx, dweight, dbias from the checkpoint's values and the forward pass's statistics."""
    dy, n = dy.double(), (xv.double() - mean.double()[:, None]) * rstd.double()[:, None]
    q = dy if weight is None else dy * weight.double()
    dx = rstd.double()[:, None] * (q - q.mean(-1, keepdim=True) - n * (q * n).mean(-1, keepdim=True))
    return dx, (dy * n).sum(0), dy.sum(0)


def layer_norm_grad_bounds(dy, xv, mean, rstd, weight, out, weight_out):
    dx, dw, db = layer_norm_grad(dy, xv, mean, rstd, weight)
    k, dy = rstd.double()[:, None], dy.double()
    n = (xv.double() - mean.double()[:, None]).abs() * k
    q = dy.abs() if weight is None else (dy * weight.double()).abs()
    d, rows = depth(dy.shape[-1]), dy.shape[0]
    s, sn = q.mean(-1, keepdim=True), (q * n).mean(-1, keepdim=True)
    off = k * ((d + 4) * U * s + (d + 12) * U * n * sn + 8 * U * (q + s + n * sn))
    tw, tb = (rows + 8) * U * (dy.abs() * n).sum(0), (rows + 2) * U * dy.abs().sum(0)
    return (off + half_step(out) * (dx.abs() + off), tw + half_step(weight_out) * (dw.abs() + tw), tb + half_step(weight_out) * (db.abs() + tb))


def activation(z, kind):
    z = z.double()
    if kind == "silu":
        p = torch.sigmoid(z)
        return z * p, p + z * p * torch.sigmoid(-z)
    p = 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
    return z * p, p + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)


def activation_bounds(z, kind):
    """How far act and act' may be off in binary32.  The exponential, the reciprocal and erfc come within 8 half steps of their values;
    an argument's rounding moves e^-z by |z| half steps and erfc(z / sqrt 2) by z^2 of them."""
    z = z.double()
    a = z.abs()
    if kind == "silu":
        p, q = torch.sigmoid(z), torch.sigmoid(-z)
        rel = (20 + 2 * a) * U                                               # of p
        # e^-z passes the largest binary32, 2^128, at z = -88.72, where p is 2^-128: from 2^-125 down p may come out as zero
        none = torch.where(p < 2.0 ** -125, p, torch.zeros_like(p))
        return a * p * rel + a * p * U + a * none, p * (1 + a * q) * (rel + 4 * U) + p * a * (p * rel + U) + (1 + a) * none
    p = 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
    rel = (20 + 4 * a * a) * U
    density = a * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return a * p * (rel + U) + 1e-38, p * (rel + U) + density * (20 + 4 * a * a) * U + 1e-38


def weight_grad(dy, xv):
    return dy.double().t().contiguous() @ xv.double(), dy.double().sum(0)


def weight_grad_bounds(dy, xv, out):
    """A sum of n products in binary32, in any order, each addition off by a step of its result at most."""
    dw, db = weight_grad(dy, xv)
    n = dy.shape[0] + 8
    parts = 3 if dy.dtype == torch.float32 else 1
    tw = 2 * parts * n * U * (dy.double().abs().t().contiguous() @ xv.double().abs())
    tb = 2 * parts * n * U * dy.double().abs().sum(0)
    return tw + half_step(out) * (dw.abs() + tw) + 1e-38, tb + half_step(out) * (db.abs() + tb) + 1e-38
