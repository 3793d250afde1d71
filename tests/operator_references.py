"""Definitions of the token-model operators in 64 bits, and error bounds of a 32-bit evaluation.

The bounds hold for any kernel that computes in binary32 (u = 2^-24) with sums
of chains of at most n / 32 additions followed by a tree, whatever its order:
they are derived from the formulas, not from runs."""
from __future__ import annotations

import math

import torch

U = 2.0 ** -24
# half the spacing of a type's values relative to the value, and half of its smallest spacing
ROUND = {torch.float32: (U, 2.0 ** -126), torch.bfloat16: (2.0 ** -8, 2.0 ** -126), torch.float16: (2.0 ** -11, 2.0 ** -25)}


def chain(n):
    """Relative error of a sum of n terms against the sum of their magnitudes."""
    return (n / 32 + 24) * U


def rounded(y, dtype):
    """The error of rounding y to dtype."""
    rel, least = ROUND[dtype]
    return rel * y.abs() + least


def within(got, want, tol, what):
    got = got.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    same = (got == want) | (got.isnan() & want.isnan())
    bad = ~same & ~((got - want).abs() <= tol)
    if bad.any():
        i = tuple(int(x) for x in bad.nonzero()[0])
        t = tol.expand(want.shape)[i] if isinstance(tol, torch.Tensor) else tol
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {i}: {float(got[i])!r} for "
                             f"{float(want[i])!r}, allowed {float(t):.3g}")


def norm_forward(x, weight, bias, eps):
    """y, mean, rstd and the bounds of their errors; x, weight, bias broadcast to (rows, width), 64 bits."""
    n = x.shape[-1]
    mean = x.mean(-1, keepdim=True)
    d = x - mean
    var = (d * d).mean(-1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    e_mean = chain(n) * x.abs().mean(-1, keepdim=True) + 2 * U * mean.abs()
    # d is off by e_mean + u |d|; (sum of) squares by 2 |d| (e_mean + u |d|) + e_mean^2, and the chain
    e_var = 2 * d.abs().mean(-1, keepdim=True) * e_mean + e_mean ** 2 + (chain(n) + 6 * U) * var
    e_rstd = rstd * (0.5 * e_var / (var + eps) + (e_var / (var + eps)) ** 2 + 6 * U)
    h = d * rstd
    e_h = e_mean * rstd + d.abs() * e_rstd + 3 * U * h.abs()
    y = h * weight + bias
    e_y = e_h * weight.abs() + 3 * U * ((h * weight).abs() + bias.abs())
    return y, mean, rstd, e_y, e_mean, e_rstd


def norm_backward(dy, x, weight, mean, rstd):
    """dx, the terms of dweight and dbias, and the bound of dx's error, at the given statistics."""
    n = x.shape[-1]
    h = (x - mean) * rstd
    a = dy * weight
    c1 = a.mean(-1, keepdim=True)
    c2 = (a * h).mean(-1, keepdim=True)
    dx = rstd * (a - c1 - h * c2)
    e1 = (chain(n) + 4 * U) * a.abs().mean(-1, keepdim=True)
    e2 = (chain(n) + 8 * U) * (a * h).abs().mean(-1, keepdim=True)
    e = rstd * (e1 + h.abs() * e2 + 8 * U * (a.abs() + c1.abs() + (h * c2).abs()))
    return dx, dy * h, dy, e


def distillation(z, ids, values, teacher_lse, weights, temperature, scale, lse=None):
    """loss, lse, dlogits and the bounds of their errors.  z (rows, vocab) and values (rows, k) in 64 bits;
    lse: as given to the gradient alone."""
    R, V = z.shape
    T = temperature
    there = (ids >= 0) & (ids < V) & (values != -math.inf)
    counts = there.any(1) & (weights != 0)
    t = torch.where(there, values / T, torch.full_like(values, -math.inf))
    if teacher_lse is None:
        lse_t = torch.where(there.any(1), torch.logsumexp(t, 1), torch.zeros(R, dtype=t.dtype, device=t.device))
    else:
        lse_t = teacher_lse
    p = torch.where(there, torch.exp(t - lse_t[:, None]), torch.zeros_like(t))
    z = torch.where(counts[:, None], z, torch.zeros_like(z))  # rows that do not count are not read
    zt = z / T
    given = lse is not None
    if not given:
        lse = torch.logsumexp(zt, 1)
    at = ids.clamp(0, V - 1).long()
    logp = t - lse_t[:, None]
    logq = zt.gather(1, at) - lse[:, None]
    terms = torch.where(p > 0, p * (logp - logq), torch.zeros_like(p))
    c = torch.where(counts, weights, torch.zeros_like(weights))
    c = torch.where(counts, c, torch.zeros_like(c))
    zero = torch.zeros_like(lse)
    loss = torch.where(counts, c * T * T * terms.sum(1), zero)
    q = torch.exp(zt - lse[:, None])
    mass = p.sum(1, keepdim=True)
    pv = torch.zeros_like(z).scatter_add_(1, at, p)
    dz = torch.where(counts[:, None], scale * T * c[:, None] * (mass * q - pv), torch.zeros_like(z))

    finite = torch.where(zt.isfinite(), zt.abs(), torch.zeros_like(zt))
    tf = torch.where(there, t, torch.zeros_like(t))
    # an exponent's error: two roundings of each argument (and of the maximum), two of the constants
    # log2 e and 1 / T, and the exponential's and logarithm's own few units
    e_t = 8 * U * (tf.abs().amax(1) + lse_t.abs()) + 16 * U + chain(t.shape[1])
    e_z = 8 * U * (finite.amax(1) + torch.where(lse.isfinite(), lse.abs(), zero)) + 16 * U
    e_lse = e_z + (0 if given else chain(V))
    e_loss = c * T * T * ((p * (e_t + e_lse + e_z)[:, None]).sum(1)
                          + torch.where(p > 0, terms.abs() * (2 * e_t[:, None] + chain(t.shape[1])), 0 * p).nan_to_num(0, 0, 0).sum(1))
    e_dz = (scale * T * c).abs()[:, None] * (mass * q * (e_z + e_lse + e_t + chain(t.shape[1]))[:, None]
                                             + pv * (2 * e_t + chain(t.shape[1]))[:, None])
    return loss, torch.where(counts, lse, zero), dz, e_loss, e_lse + U * lse.abs().nan_to_num(0, 0, 0), e_dz
