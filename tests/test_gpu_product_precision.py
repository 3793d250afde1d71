"""What the products keep of operands that have more than 16 bits: sums whose large parts cancel, so that what an operand
would lose shows beside the one rounding that a 16-bit result has.

Two bf16 parts keep 2^-16 of a value, three 2^-24 (eps / 2 of bf16 is 2^-8, and each part holds what the ones before
leave); a pair of parts that is left out is at most as large.  Each step of 16 products in the tensor cores is within
2^-22 of the magnitudes; here all products are in one step of each pair of parts, the others add zeros.
"""
from __future__ import annotations

import pytest

from operator_references import U, rounded, within
from test_gpu_products import P, gen, rows_of, stream  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TYPES = {1: torch.bfloat16, 2: torch.float16}
STEP = 2.0 ** -22


def nearby(shape, seed, spread):
    """Values of 24 bits from 1 to 1 + spread."""
    return 1 + spread * torch.rand(shape, generator=gen(seed), device="cuda")


@pytest.mark.parametrize("pad", [0, 3])  # rows that TMA reads, and rows that it does not
@pytest.mark.parametrize("dtype", [1, 2])
@pytest.mark.parametrize("rows", [3, 20, 200])
def test_weights_that_differ_by_less_than_a_16_bit_step(P, rows, dtype, pad):  # noqa: F811
    """fp32 weights of 16-bit rows, as a lookahead point has them: steps of less than 2^-8 of the weights count, in the
    forward pass and in dx."""
    W, K, N, T = 2, 16, 16, TYPES[dtype]
    signs = torch.tensor([1.0, -1.0], device="cuda").repeat(8)
    x, _ = rows_of(signs.expand(W * rows, K), pad, T)
    weight = nearby((W, N * K), rows, 2.0 ** -9)
    op = P.Linear(inputs=K, outputs=N, max_rows=rows, workers=W, dtype=dtype, cuda_stream=stream())
    y, _ = rows_of(torch.zeros((W * rows, N)), pad, T)
    op.forward(rows, x, x.stride(0), weight, N * K, None, 0, None, 0, y, y.stride(0))
    dx, _ = rows_of(torch.zeros((W * rows, K)), pad, T)
    op.backward(rows, x, x.stride(0), x, x.stride(0), weight, N * K, None, 0, dx, dx.stride(0), None, None, 0)
    w = weight.double().view(W, N, K)
    for got, want in ((y, w @ signs.double()), (dx, signs.double() @ w)):
        want = want.repeat_interleave(rows, 0)
        e = 16 * (2.0 ** -16 * (1 + 3) + 3 * STEP)
        within(got, want, e + rounded(want.abs() + e, T), "cancelling sums")
        assert float(want.abs().max()) > 2 * e
    op.destroy()


def lost_most(values, count):
    """The indices of the values of which two bf16 parts lose most, and what they lose."""
    first = values.bfloat16().float()
    left = values - first - (values - first).bfloat16().float()
    at = left.abs().argsort(descending=True)[:count]
    return at, left[at]


def gelu_slopes():
    """bf16 values between 1 and 3 and GELU's slopes there, in 64 bits and in 32."""
    u = torch.arange(1, 3, 2.0 ** -6, dtype=torch.float64, device="cuda")
    s = 0.5 * torch.erfc(-u / 2 ** 0.5) + u * torch.exp(-0.5 * u * u) / (2 * torch.pi) ** 0.5
    return u, s, s.float()


# A slope's error in 32 bits: erfc's approximation 1.5e-7, halved, and some ten roundings of values up to 1.
SLOPE = 10 * U


@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("dtype", [1, 2])
@pytest.mark.parametrize("rows", [3, 16])
def test_slopes_keep_more_than_a_16_bit_result(P, rows, dtype, pad):  # noqa: F811
    """dx of slopes whose roundings to 16 bits all point one way."""
    K, T = 8, TYPES[dtype]
    u, s, s32 = gelu_slopes()
    off = s32 - s32.to(torch.bfloat16).float()
    at = off.abs().argsort(descending=True)[:16]
    u, s, off = u[at], s[at], off[at]
    N = len(u)
    pre, _ = rows_of(u.float().expand(rows, N), pad, T)
    dy, _ = rows_of(torch.ones((rows, N)), pad, T)
    weight = off.sign()[:, None].expand(N, K).to(T).contiguous()
    weight[:, 1] = 1
    op = P.Linear(inputs=K, outputs=N, max_rows=rows, dtype=dtype, weight_dtype=dtype, activation=P.GELU, cuda_stream=stream())
    dx, _ = rows_of(torch.zeros((rows, K)), pad, T)
    op.backward(rows, dy, dy.stride(0), dy, dy.stride(0), weight, 0, pre, pre.stride(0), dx, dx.stride(0), None, None, 0)
    want = (s @ weight.double()).expand(rows, K)
    e = N * (2.0 ** -16 * (1 + 3) + 3 * STEP + SLOPE)
    within(dx, want, e + rounded(want.abs() + e, T), "dx")
    op.destroy()


@pytest.mark.parametrize("dtype", [1, 2])
@pytest.mark.parametrize("rows", [3, 16])
def test_slopes_keep_24_bits_in_fp32_gradients(P, rows, dtype):  # noqa: F811
    """dweight of slopes of which two bf16 parts lose most, all one way."""
    K, N, T = 8, 16, TYPES[dtype]
    u, s, s32 = gelu_slopes()
    at, left = lost_most(s32, rows)
    pre = u[at].to(T)[:, None].expand(rows, N).contiguous()
    dy = torch.ones((rows, N), dtype=T, device="cuda")
    x = left.sign().to(T)[:, None].expand(rows, K).contiguous()
    op = P.Linear(inputs=K, outputs=N, max_rows=rows, dtype=dtype, weight_dtype=dtype, activation=P.GELU, cuda_stream=stream())
    dw = torch.zeros((N, K), device="cuda")
    op.backward(rows, dy, N, x, K, None, 0, pre, N, None, K, dw, None, 0)
    want = (s[at] @ x.double()).expand(N, K)
    e = 1.13 * rows * (2.0 ** -24 * (1 + 3) + 3 * STEP) + rows * SLOPE
    within(dw, want, e + U * want.abs(), "dweight")
    if rows == 16:
        assert float(left.abs().sum()) > 2 * e
    op.destroy()
