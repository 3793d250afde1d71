"""Definitions of the linear layers, the token loss and the clipping in 64 bits, and error bounds of products of
16-bit parts with fp32 sums.

What a product's operands lose before they are multiplied: nothing where they lie in 16 bits, 2^-8 of the value in one
bf16 part, 2^-16 in two, 2^-24 in three (eps / 2 of bf16 is 2^-8, and each part holds what the ones before leave); of
pairs of parts those are left out that are below the last part's rounding, and there are at most three of them.  The
sums: up to 1024 products (8192 where the result is bf16, 2048 in f16) at a time in the tensor cores, 16 to a step,
each step within two units (2^-23) of the magnitudes so far; then additions rounded to nearest.  All relative to the
sum of the magnitudes."""
from __future__ import annotations

import math

import torch

from operator_references import U, rounded

DTYPES = {0: torch.float32, 1: torch.bfloat16, 2: torch.float16}


def parts_error(parts):
    return 2.0 ** (-8 * parts)


def sum_error(depth, terms=1, result=0):
    """Of a product's sum over `depth` with `terms` pairs of parts, relative to the sum of the magnitudes (the smaller
    pairs' own sums are at most 2^-7 of the first's)."""
    chunk = {0: 1024, 1: 8192, 2: 2048}[result]
    steps = min(math.ceil(depth / 64) * 4 * terms, chunk // 16)
    return steps * 2 * 2 ** -23 + (math.ceil(depth * terms / chunk) + 152) * U


def product_error(a_abs, b_abs, depth, a_loss, b_loss, terms, result=0):
    """Bound of the error of a @ b from the magnitudes, where a and b are off by a_loss and b_loss of themselves."""
    left_out = 3 * max(a_loss, b_loss) if terms > 1 else 0
    return (a_abs @ b_abs) * (a_loss + b_loss + a_loss * b_loss + left_out + sum_error(depth, terms, result))


def activation(u, kind):
    F = torch.nn.functional
    return {0: lambda v: v, 1: F.relu, 2: F.gelu, 3: F.silu}[kind](u)


def slope(u, kind):
    if kind == 0:
        return torch.ones_like(u)
    with torch.enable_grad():
        u = u.detach().requires_grad_()
        return torch.autograd.grad(activation(u, kind).sum(), u)[0]


def act_parts(dtype):
    return {0: 3, 1: 1, 2: 2}[dtype]


def forward_loss(dtype, weight_dtype):
    """What x and the weights lose in a linear layer's forward product, and the pairs of parts."""
    if dtype == weight_dtype and dtype != 0:
        return 0.0, 0.0, 1
    return (parts_error(3) if dtype == 0 else 0.0), parts_error({0: 3, 1: 1, 2: 2}[dtype]), {0: 6, 1: 1, 2: 3}[dtype]


def linear_forward(x, weight, bias, residual, kind, dtype, weight_dtype):
    """y, u and the bounds of their errors; one worker, 64 bits."""
    lx, lw, terms = forward_loss(dtype, weight_dtype)
    u = x @ weight.t() + bias
    e_u = product_error(x.abs(), weight.t().abs(), x.shape[1], lx, lw, terms, dtype) + 2 * U * (u.abs() + bias.abs())
    y = activation(u, kind)
    # slopes are at most 1.13; the functions' own errors are a few units of their arguments and results
    e_y = 1.13 * e_u + 16 * U * (y.abs() + u.abs().clamp(max=8))
    y = y + residual
    T = DTYPES[dtype]
    e_y = e_y + 2 * U * (y.abs() + residual.abs())
    return y, u, e_y + rounded(y.abs() + e_y, T), e_u + rounded(u.abs() + e_u, T)


def linear_backward(dy, x, weight, pre, kind, dtype, weight_dtype):
    """dx, dweight, dbias and the bounds of their errors; one worker, 64 bits."""
    s = slope(pre, kind)
    du = dy * s
    # the slopes' own errors: a few units of values of up to 1.13 (and of u^2 in the exponential)
    e_du = 32 * U * dy.abs() * (1 + pre.abs().clamp(max=8)) if kind > 1 else 0 * dy
    loss_d = {0: parts_error(3), 1: 0.0 if kind < 2 else parts_error(2), 2: 0.0 if kind < 2 else parts_error(2)}[dtype]
    loss_dx = {0: parts_error(3), 1: 0.0 if kind < 2 else parts_error(1), 2: 0.0 if kind < 2 else parts_error(2)}[dtype]
    if dtype == 2 and loss_d == 0:
        loss_d = loss_dx = parts_error(2)  # an f16 value in two bf16 parts is exact; the pairs left out are not
    lw = 0.0 if weight_dtype == 1 else parts_error({0: 3, 1: 1, 2: 2}[dtype])
    lx = {0: parts_error(3), 1: 0.0, 2: parts_error(2)}[dtype]
    terms = {0: 6, 1: 2, 2: 3}[dtype]
    dx = du @ weight
    e_dx = product_error(du.abs(), weight.abs(), du.shape[1], loss_dx, lw, 1 if dtype == 1 else terms, dtype) + e_du @ weight.abs()
    dw = du.t() @ x
    e_dw = product_error(du.abs().t(), x.abs(), len(x), loss_d, lx, terms) + e_du.t() @ x.abs()
    db = du.sum(0)
    e_db = (du.abs() * (len(x) / 8 + 24) * U + e_du).sum(0)
    T = DTYPES[dtype]
    return dx, dw, db, e_dx + rounded(dx.abs() + e_dx, T), e_dw + U * dw.abs(), e_db + U * db.abs()


def token_loss(x, weight, targets, weights, scale, dtype, weight_dtype, lse=None):
    """loss, lse, dx, dweight and the bounds of their errors; one worker, 64 bits.  lse: as given to the gradient."""
    V = len(weight)
    counts = (targets >= 0) & (targets < V) & (weights != 0)
    x = torch.where(counts[:, None], x, 0)  # what rows that do not count hold does not matter
    z = x @ weight.t()
    half = dtype == weight_dtype and dtype != 0
    lx = parts_error(3) if dtype == 0 else 0.0
    lw = 0.0 if half else parts_error(3 if dtype == 0 else 2)
    e_z = product_error(x.abs(), weight.t().abs(), x.shape[1], lx, lw, {0: 6, 1: 1 if half else 2, 2: 1 if half else 3}[dtype])
    given = lse is not None
    if not given:
        lse = torch.logsumexp(z, 1)
    worst = e_z.amax(1)
    # the exponents' errors, the exponential's and the logarithm's own, and the sum's chain
    e_lse = 0 * worst if given else worst + (8 * z.abs().amax(1) + 16 + V / 32 + 24) * U + 2 * U * lse.abs()
    at = targets.clamp(0, V - 1)[:, None]
    c = torch.where(counts, weights, 0)
    loss = c * (lse - z.gather(1, at)[:, 0])
    e_loss = c * (e_lse + e_z.gather(1, at)[:, 0] + 4 * U * (lse.abs() + z.gather(1, at)[:, 0].abs()))
    q = torch.exp(z - lse[:, None])
    e_q = q * (e_z + e_lse[:, None] + 8 * U * (z.abs() + lse.abs()[:, None]) + 16 * U)
    one = torch.zeros_like(q).scatter_(1, at, 1.0)
    d = (scale * c)[:, None] * (q - one)
    e_d = (scale * c)[:, None].abs() * e_q + 4 * U * d.abs()
    loss_d = parts_error(3 if dtype == 0 else 2)
    loss_dx = parts_error(1) if dtype == 1 else loss_d
    lw = {0: parts_error(3), 1: 0.0 if weight_dtype == 1 else parts_error(1), 2: parts_error(2)}[dtype]
    terms = {0: 6, 1: 1, 2: 3}[dtype]
    dx = d @ weight
    pieces = 4 * U * (d.abs() @ weight.abs())
    e_dx = product_error(d.abs(), weight.abs(), V, loss_dx, lw, terms, dtype) + e_d @ weight.abs() + pieces
    dw = d.t() @ x
    e_dw = product_error(d.abs().t(), x.abs(), len(x), loss_d, parts_error(act_parts(dtype)) if dtype != 1 else 0.0,
                         {0: 6, 1: 2, 2: 3}[dtype]) + e_d.t() @ x.abs()
    zero = torch.zeros_like(lse)
    T = DTYPES[dtype]
    return (torch.where(counts, loss, zero), torch.where(counts, lse, zero), dx, dw, e_loss, e_lse,
            e_dx + rounded(dx.abs() + e_dx, T), e_dw + U * dw.abs())
