"""Plain 64-bit forms of the normalisation and of the head's loss, with bounds on what float32 arithmetic may be off by.

E = 2^-24 is half a step of float32.  A sum of n rounded terms is off by at most n E times the sum of their sizes, and with
independent roundings by 4 sqrt(n) E times it with near certainty; blocks' shares of at most 256 terms a thread and a tree over
them are taken as 300 E.  A result rounded to a type of spacing eps is off by eps / 2 of its size (of the least normal number
below that).
"""
import math

import torch

E = 2.0 ** -24
TINY = {torch.float64: 2.0 ** -1022, torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -14, torch.bfloat16: 2.0 ** -126}


def rounding(t, dtype):
    return torch.finfo(dtype).eps / 2 * t.abs().clamp_min(TINY[dtype])


def norm_reference(x, groups, w, b, eps, act, dy=None):
    """(y, its bound) and, with dy, (dx, dw, db, their bounds); x [batch, points, channels], everything in float64."""
    dtype = x.dtype
    x = x.double()
    N, S, C = x.shape
    Cg = C // groups
    w = torch.ones(C, dtype=torch.float64, device=x.device) if w is None else w.double()
    b = torch.zeros(C, dtype=torch.float64, device=x.device) if b is None else b.double()

    def mean(t):
        return t.view(N, S, groups, Cg).mean((1, 3), keepdim=True).expand(N, S, groups, Cg).reshape(N, S, C)
    dev = x - mean(x)
    rstd = 1.0 / torch.sqrt(mean(dev * dev) + eps)
    xhat = dev * rstd
    v = xhat * w + b
    # the scale from squares summed in float32 (300 E of the variance, half of it in its root) and a few roundings, on
    # differences that carry a rounding of their own; and the mean, from differences summed in float32 over runs of at most 128
    # values: 4 sqrt(128) E = 45 E of the differences' mean size, which two values of one spread have at sqrt(2) spreads: 64 E
    d_xhat = 160 * E * xhat.abs() + 64 * E
    d_v = d_xhat * w.abs() + 4 * E * (v.abs() + b.abs())
    sig = torch.sigmoid(v)
    y = {"none": v, "relu": v.clamp_min(0.0), "silu": v * sig}[act]
    # the exponential's argument is rounded (|v| log2 e), then three results to an ulp each
    d_y = 1.1 * d_v + (8 + 2 * v.abs()) * E * y.abs() + rounding(y, dtype)
    if dy is None:
        return y, d_y
    dy = dy.double()
    slope = {"none": torch.ones_like(v), "relu": (v > 0).double(), "silu": sig * (1 + v * (1 - sig))}[act]
    dv = dy * slope
    if act == "relu":  # on which side of 0 such an element falls is open
        d_dv = torch.where(v.abs() <= d_v, dy.abs(), torch.zeros_like(dy))
    elif act == "silu":
        d_dv = dy.abs() * (0.5 * d_v + (16 + 4 * v.abs()) * E * (1 + v.abs()) * sig)
    else:
        d_dv = torch.zeros_like(dy)
    d_dv = d_dv + 2 * E * dv.abs()
    db, dw = dv.sum((0, 1)), (dv * xhat).sum((0, 1))
    d_db = d_dv.sum((0, 1)) + 300 * E * dv.abs().sum((0, 1)) + 1e-30
    d_dw = (d_dv * xhat.abs() + dv.abs() * d_xhat).sum((0, 1)) + 300 * E * (dv * xhat).abs().sum((0, 1)) + 1e-30
    t, d_t = dv * w, d_dv * w.abs()
    m1, m2 = mean(t), mean(t * xhat)
    d_m1 = mean(d_t) + 300 * E * mean(t.abs())
    d_m2 = mean(d_t * xhat.abs() + t.abs() * d_xhat) + 300 * E * mean((t * xhat).abs())
    dx = rstd * (t - m1 - xhat * m2)
    parts = t.abs() + m1.abs() + (xhat * m2).abs()
    d_dx = rstd * (d_t + d_m1 + xhat.abs() * d_m2 + d_xhat * m2.abs() + 200 * E * parts) + rounding(dx, dtype)
    return y, d_y, dx, d_dx, dw, d_dw, db, d_db


def xent_reference(h, W, labels, ignore, reduction, up=None):
    """(loss, its bound) and, with up (a float or [rows]), (dh, dW, their bounds), in float64."""
    dtype = h.dtype
    h, W = h.double(), W.double()
    n, d = h.shape
    V = W.shape[0]
    keep = labels != ignore
    h = torch.where(keep[:, None], h, torch.zeros_like(h))
    at = torch.where(keep, labels, torch.zeros_like(labels))[:, None]
    z = h @ W.t()
    # float32 products of at most 24 + 24 bits, summed in some order
    d_z = (4 * math.sqrt(d) + 4) * E * (h.abs() @ W.abs().t())
    # float32 with more than 128 rows, 128 classes and 2^28 products: two float16 planes, each value good to 2^-23 of itself and 2^-39
    # of the largest, products of the second planes (2^-11 each, at most) left out: 2 2^-23 + 2^-22 = 8 E of a product
    planes = dtype == torch.float32 and min(n, V) > 128 and n * d * V > 2 ** 28
    floor = 2.0 ** -39 * planes
    top_h, top_w, extra = h.abs().max(), W.abs().max(), 8 * E * planes
    d_z = d_z + extra * (h.abs() @ W.abs().t()) + floor * (top_h * W.abs().sum(1)[None, :] + top_w * h.abs().sum(1, keepdim=True))
    lse = torch.logsumexp(z, 1, keepdim=True)
    top_d = d_z.amax(1, keepdim=True)
    rows = (lse - z.gather(1, at))[:, 0]
    d_rows = (2 * top_d + (16 + 2 * math.log(V + 1)) * E * (1 + lse.abs()) + 4 * E * z.abs().amax(1, keepdim=True))[:, 0]
    zero = torch.zeros_like(rows)
    rows, d_rows = torch.where(keep, rows, zero), torch.where(keep, d_rows, zero)
    count = max(1, int(keep.sum()))
    by = {"mean": 1.0 / count, "sum": 1.0}.get(reduction)
    loss, d_loss = (rows, d_rows) if by is None else (rows.sum() * by, d_rows.sum() * by)
    d_loss = d_loss + 4 * E * loss.abs() + 1e-30
    if up is None:
        return loss, d_loss
    g = up.double() if by is None else torch.full_like(rows, float(up) * by)
    g = torch.where(keep, g, zero)[:, None]
    p = torch.exp(z - lse)
    hit = torch.zeros_like(p).scatter_(1, at, 1.0)
    dz = (p - hit) * g
    # exp of a difference that is off by d_z + what lse is off by; then held in the type (float32: whole)
    off = d_z + top_d + 8 * E * (1 + z.abs() + lse.abs())
    d_dz = (p * torch.expm1(off) + 4 * E * (p + hit)) * g.abs() + rounding(dz, torch.float32 if dtype == torch.float32 else dtype) * (dz != 0)
    d_dz = d_dz + planes * (2 * E * dz.abs() + floor * g.abs().max() * (g != 0))
    d_dz = d_dz + 4 * 2.0 ** -126 * g.abs()  # (what is below the least normal number may be taken as 0)
    if dtype == torch.float16:  # held as a multiple of the largest upstream gradient by 2^-14
        d_dz = d_dz.clamp_max(1e30) - rounding(dz, dtype) * (dz != 0) + torch.finfo(dtype).eps / 2 * (
            dz.abs() + g.abs().max() * 2.0 ** -28) * (dz != 0)
    sums_v, sums_n = (4 * math.sqrt(V) + 8) * E, (4 * math.sqrt(n) + 8) * E
    dh, dW = dz @ W, dz.t() @ h
    d_dh = d_dz @ W.abs() + (sums_v + extra) * (dz.abs() @ W.abs()) + floor * top_w * dz.abs().sum(1, keepdim=True) + rounding(dh, dtype)
    d_dW = d_dz.t() @ h.abs() + (sums_n + extra) * (dz.abs().t() @ h.abs()) + floor * top_h * dz.abs().sum(0)[:, None] + rounding(dW, dtype)
    return loss, d_loss, dh, d_dh, dW, d_dW


def within(got, want, bound, name=""):
    got = got.double()
    assert got.shape == want.shape, (name, got.shape, want.shape)
    assert bool(torch.isfinite(got).all()), f"{name}: not finite"
    over = ((got - want).abs() / bound.clamp_min(1e-300)).max()
    assert float(over) <= 1.0, f"{name}: off by {float(over):.3g} times its bound, {float((got - want).abs().max()):.3g}"
