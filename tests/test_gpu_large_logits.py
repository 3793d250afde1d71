"""The token loss of logits of any size: the exponents are differences, so that their error is that of the logits' sums
and of lse, not one that grows with the logits.

Where the logits are exact (x has a single one, the weights are the logits, in the type's own values): the loss is off
by the rounding of lse to 32 bits (and of the terms of its sum), the probabilities by what that rounding makes of them.
"""
from __future__ import annotations

import math

import pytest

from operator_references import U, rounded, within
from product_references import sum_error
from test_gpu_products import DTYPES, P, gen, stream  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

ROWS = [3, 9, 40, 300]  # without tiles, and on them


def step(P, z, targets, dtype, weight_dtype, rows):  # noqa: F811
    """Loss, lse, dx and dweight of `rows` equal rows with the logits z (one row of the table each)."""
    V, C, T = len(z), 8, DTYPES[dtype]
    w = torch.zeros((V, C), dtype=DTYPES[weight_dtype], device="cuda")
    w[:, 0] = z
    w[:, 1] = 1
    x = torch.zeros((rows, C), dtype=T, device="cuda")
    x[:, 0] = 1
    op = P.TokenLoss(vocab=V, width=C, max_rows=rows, dtype=dtype, weight_dtype=weight_dtype, cuda_stream=stream())
    loss, lse = torch.full((2, rows), math.nan, device="cuda")
    dx, dw = torch.full_like(x, math.nan), torch.full((V, C), math.nan, device="cuda")
    op.step(rows, x, C, w, 0, targets, None, 1.0, loss, lse, dx, C, dw, 0)
    op.synchronize()
    op.destroy()
    return w[:, 0].double(), loss, lse, dx, dw


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("types", [(0, 0), (1, 1), (1, 0), (2, 2), (2, 0)], ids=str)
@pytest.mark.parametrize("size", [40.0, 150.0, 15000.0, 1.5e6, 1.5e8, 6e9, 1e30])
def test_one_logit_far_above_the_others(P, size, types, rows):  # noqa: F811
    """Loss, gradients: 0, and never below; of another target the difference of the logits, and -1 and 1."""
    dtype, weight_dtype = types
    if dtype == 2:
        size = min(size, 3e4)  # f16's range
    V = 700
    for seed in range(3):
        z = size * (0.2 * torch.rand(V, generator=gen(seed), device="cuda") - 0.1)
        top = int(torch.randint(0, V, (1,), generator=gen(seed + 9), device="cuda"))
        other = (top + 1 + seed) % V
        z[top] = size * (1 + 0.03 * seed)
        targets = torch.full((rows,), top, dtype=torch.int32, device="cuda")
        targets[rows // 2] = other
        z, loss, lse, dx, dw = step(P, z, targets, dtype, weight_dtype, rows)
        with_top = targets == top
        tail = float(torch.exp(z - z[top]).sum() - 1)  # e^-32 of 700 others at least
        assert tail < 1e-11
        # fp32 logits pass through parts and sums
        near = 4 * U * z.abs() if weight_dtype == 0 else 0 * z
        assert bool((loss[with_top] >= 0).all()) and float(loss[with_top].max()) <= tail
        within(lse, z[top].expand(rows), U * z[top].abs() + near[top] + tail, "lse")
        gap = z[top] - z[other]
        within(loss[rows // 2], gap, 4 * U * (z[top].abs() + gap) + near[top] + near[other] + tail, "another target's loss")
        assert float(dx[with_top].abs().max()) <= tail * max(1.0, float(z.abs().max()))
        want = torch.zeros(V, dtype=torch.float64, device="cuda")
        want[top], want[other] = 1, -1
        within(dw[:, 0], want, 1e-8 + 4 * U * want.abs(), "dweight")
        assert float(dx[rows // 2, 1].abs()) <= 1e-6  # 1 - 1
        grad = z[top] - z[other]
        e = 2.0 ** -14 * (z[top].abs() + z[other].abs()) + tail * z.abs().sum()
        within(dx[rows // 2, 0], grad, e + rounded(grad.abs() + e, DTYPES[dtype]), "dx")


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("size", [30.0, 1e3, 1e5, 1e6])
@pytest.mark.parametrize("dtype", [1, 0])
def test_probabilities_of_large_logits_that_lie_together(P, dtype, size, rows):  # noqa: F811
    """Logits of size + 0 to 7: the probabilities go by their differences; lse is rounded to its own last bit."""
    V = 300
    spacing = 2.0 ** (math.floor(math.log2(size)) - (7 if dtype == 1 else 22))
    z = size + torch.randint(0, 8, (V,), generator=gen(1), device="cuda") * max(1.0, spacing)
    if dtype == 1:
        z = z.bfloat16().float()
    targets = torch.randint(0, V, (rows,), generator=gen(2), device="cuda").int()
    z, loss, lse, dx, dw = step(P, z, targets, dtype, dtype, rows)
    want = torch.logsumexp(z, 0)
    # fp32 logits pass through parts and sums: whole numbers of up to 21 bits are exact in three parts
    e_lse = 2 * U * want.abs() + 64 * U
    within(lse, want.expand(rows), e_lse, "lse")
    at = targets.long()
    within(loss, want - z[at], 2 * e_lse, "loss")
    assert bool((loss >= 0).all())
    p = torch.exp(z - lse.double()[0])
    count = torch.zeros(V, dtype=torch.float64, device="cuda").index_add_(0, at, torch.ones(rows, dtype=torch.float64, device="cuda"))
    # exponentials below 2^-126 may be taken as 0: here they are down to e^-4000, which no fp32 value is
    e_p = rows * (p * 32 * U + 2.0 ** -126) + (4 * U + sum_error(rows, 6)) * (rows * p + count)
    within(dw[:, 0], rows * p - count, e_p, "dweight")
    assert float(((dw[:, 0].double() + count) / rows).max()) <= 1 + 2.0 ** -15


def test_both_passes_sum_a_logit_alike(P):  # noqa: F811
    """Rows whose target's logit is far above the others, in a vocabulary of two pieces: nothing is left of the gradient
    unless the second pass has other sums than lse was made of.  The targets are the last columns, in tiles that do not
    fill the GPU and are cut along the width where a pass takes the whole vocabulary at once."""
    n, V, C = 20_000, 13_000, 2048
    w = torch.randn((V, C), generator=gen(1), device="cuda").bfloat16()
    targets = torch.randint(12_800, V, (n,), generator=gen(2), device="cuda").int()
    x = (40 * w[targets.long()].float()).bfloat16()  # logits of 8e4, and of at most 1e4 elsewhere
    op = P.TokenLoss(vocab=V, width=C, max_rows=n, dtype=P.BF16, weight_dtype=P.BF16, cuda_stream=stream())
    loss, lse = torch.full((2, n), math.nan, device="cuda")
    dx, dw = torch.full_like(x, math.nan), torch.full((V, C), math.nan, device="cuda")
    op.step(n, x, C, w, 0, targets, None, 1.0, loss, lse, dx, C, dw, 0)
    op.synchronize()
    assert not loss.any() and float(lse.min()) > 7e4
    assert not dx.any() and not dw.any()
    op.destroy()
