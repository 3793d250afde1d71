"""Rows that do not count have no loss and no gradient, whatever they hold and whatever the weights are."""
from __future__ import annotations

import math

import pytest

from test_gpu_products import DTYPES, P, gen, rows_of, stream  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("shape", [  # workers, rows, vocab, width, dtype, weight dtype, pad
    (2, 3, 50, 24, 1, 1, 0),
    (1, 8, 50, 17, 0, 0, 3),
    (2, 40, 300, 64, 1, 1, 0),
    (1, 300, 300, 33, 1, 0, 3),
    (2, 140, 200, 40, 2, 2, 0),
    (1, 65536, 5000, 16, 1, 1, 0),  # the gradient in pieces of the vocabulary
], ids=str)
def test_weights_that_are_not_finite(P, shape):  # noqa: F811
    workers, rows, vocab, width, dtype, weight_dtype, pad = shape
    n, T = workers * rows, DTYPES[dtype]
    w = torch.randn((workers, vocab * width), generator=gen(1), device="cuda").to(DTYPES[weight_dtype])
    w[:, 3], w[:, width + 1] = math.inf, math.nan
    x, _ = rows_of(torch.randn((n, width), generator=gen(2), device="cuda"), pad, T)
    targets = torch.randint(0, vocab, (n,), generator=gen(3), device="cuda").int()
    weights = torch.ones(n, device="cuda")
    gone = torch.arange(n, device="cuda") % 3 == 1
    targets[gone] = -1
    weights[torch.arange(n, device="cuda") % 6 == 2] = 0
    gone |= weights == 0
    op = P.TokenLoss(vocab=vocab, width=width, max_rows=rows, workers=workers, dtype=dtype, weight_dtype=weight_dtype,
                     cuda_stream=stream())
    loss, lse = torch.full((2, n), 7.0, device="cuda")
    dx, _ = rows_of(torch.full((n, width), 7.0), pad, T)
    op.step(rows, x, x.stride(0), w, w.stride(0), targets, weights, 1.0, loss, lse, dx, dx.stride(0), None, 0)
    for t in (loss, lse, dx):
        assert not t[gone].any()
        assert not t[~gone].isfinite().any()
    op.destroy()
