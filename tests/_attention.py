"""Attention in 64 bits on the CPU, with bounds of what fp32 sums and bf16
operands may change.  Nothing here uses the library."""
import math

import torch

F64 = torch.float64
H = 2.0 ** -8    # a rounding to bf16, relative
E = 2.0 ** -24   # to fp32


def starts(lengths, first=0):
    out = [first]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def seen(lq, lk, causal):
    i, j = torch.arange(lq)[:, None], torch.arange(lk)[None, :]
    return j <= i + (lk - lq) if causal else torch.ones(lq, lk, dtype=torch.bool)


def forward(q, k, v, mask, scale):
    """One head: (out, lse, bound of out, bound of lse).  A score's error is that
    of dim products summed in fp32 and scaled; a weight's, twice that of a score
    (its own and the maximum's), two roundings of the exponent (relative to the
    scores' size) and the exponential's 2^-22; a weight is rounded to bf16
    where it enters the product, the result where it is written."""
    q, k, v = q.to(F64), k.to(F64), v.to(F64)
    n, dim = k.shape[0], q.shape[1]
    s = torch.where(mask, (q @ k.t()) * scale, -math.inf)
    lse = torch.logsumexp(s, 1) if n else torch.full((q.shape[0],), -math.inf, dtype=F64)
    base = torch.where(lse.isinf(), 0.0, lse)
    p = torch.exp(s - base[:, None])
    out = p @ v
    size = ((q.abs() @ k.abs().t()) * scale * mask).amax(1) if n else torch.zeros_like(lse)
    ds = (dim + 8) * E * size
    dp = 2 * ds + 4 * E * size + 2.0 ** -22 + 2 * n * E
    tol = H * out.abs() + (p @ v.abs()) * ((1 + H) * (H + dp))[:, None]
    return out, lse, 1.01 * tol + 1e-37, ds + n * E + 4 * E * (base.abs() + size) + 2.0 ** -21


def backward(q, k, v, out, lse, do, mask, scale):
    """One head: (dq, dk, dv) and the bounds of the sums (not yet of the final
    rounding): weights as above from the given lse; dS = p (dP - D) has the
    errors of dP and D, sums of dim products, and its own rounding to bf16."""
    q, k, v, out, do = (x.to(F64) for x in (q, k, v, out, do))
    lse = lse.to(F64)
    n, m, dim = k.shape[0], q.shape[0], q.shape[1]
    s = torch.where(mask, (q @ k.t()) * scale, -math.inf)
    base = torch.where(lse.isinf(), 0.0, lse)
    p = torch.exp(s - base[:, None])
    size = (q.abs() @ k.abs().t()) * scale + base.abs()[:, None]
    dp = (dim + 16) * E * size + 2.0 ** -22
    delta = (do * out).sum(1, keepdim=True)
    ds = p * (do @ v.t() - delta)
    eps = p * (dim + 4) * E * (do.abs() @ v.abs().t() + (do * out).abs().sum(1, keepdim=True))
    err = (ds.abs() + eps) * ((1 + H) * (H + dp) + (n + m) * E) + eps
    perr = p * ((1 + H) * (H + dp) + m * E)
    return ((scale * ds @ k, scale * ds.t() @ q, p.t() @ do),
            (scale * err @ k.abs(), scale * err.t() @ q.abs(), perr.t() @ do.abs()))
