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


def loss_of_one_row(P, z, columns, dtype, weight_dtype, rows, factor):  # noqa: F811
    """The step of `rows` equal rows over as many logits as z has, each column's weights [columns, z]: x = (0, 1), so that
    the logits are z.  Targets: the last column."""
    V, C, T = len(z), 8, TYPES[dtype]
    w = torch.zeros((V, C), device="cuda", dtype=torch.float32 if weight_dtype == 0 else T)
    w[:, 0], w[:, 1] = columns, z
    x = torch.zeros((rows, C), dtype=T, device="cuda")
    x[:, 1] = 1
    targets = torch.full((rows,), V - 1, dtype=torch.int32, device="cuda")
    op = P.TokenLoss(vocab=V, width=C, max_rows=rows, dtype=dtype, weight_dtype=weight_dtype, cuda_stream=stream())
    loss, lse = torch.zeros((2, rows), device="cuda")
    dx, dw = torch.zeros_like(x), torch.zeros((V, C), device="cuda")
    op.step(rows, x, C, w, 0, targets, factor, 1.0, loss, lse, dx, C, dw, 0)
    op.synchronize()
    op.destroy()
    return loss, lse, dx, dw, w.double()


@pytest.mark.parametrize("weight_dtype", [0, None])
@pytest.mark.parametrize("dtype", [1, 2])
@pytest.mark.parametrize("rows", [3, 16])
def test_the_logits_gradient_keeps_more_than_a_16_bit_result(P, rows, dtype, weight_dtype):  # noqa: F811
    """dx where the gradient's parts cancel: what is left are the probabilities' and the weights' last bits."""
    weight_dtype = dtype if weight_dtype is None else weight_dtype
    z = torch.tensor([0.0, 1.125, -30.0], device="cuda")  # p = 0.245, 0.755
    columns = torch.tensor([1.0, 1.0, 1.0], device="cuda")
    if weight_dtype == 0:
        columns = torch.tensor([1 + 2.0 ** -10 + 2.0 ** -12, 1 + 2.0 ** -9 - 2.0 ** -13, 1.0], device="cuda")
    _, _, dx, _, w = loss_of_one_row(P, z, columns, dtype, weight_dtype, rows, None)
    p = torch.softmax(z.double(), 0)
    want = (p @ w[:, 0] - w[2, 0]).expand(rows)
    # the magnitudes add up to 2; q is off by a few units
    e = 2 * (2.0 ** -16 * (2 + 3) + 3 * STEP + 32 * U)
    within(dx[:, 0], want, e + rounded(want.abs() + e, TYPES[dtype]), "dx")


@pytest.mark.parametrize("dtype", [1, 2])
def test_the_logits_gradient_keeps_24_bits_in_fp32_gradients(P, dtype):  # noqa: F811
    """dweight at a target whose probability is 0: the rows' weights, of which two bf16 parts lose most, all one way."""
    V, C, T = 2, 8, TYPES[dtype]
    lost = 2.0 ** -17 - 2.0 ** -22  # of 2^-9 (1 + 2^-8 - 2^-13), rounded to eight bits
    for rows in (3, 16):
        factor = torch.full((rows,), 1 + 2.0 ** -9, device="cuda") + lost * (torch.arange(rows, device="cuda") % 2)
        w = torch.zeros((V, C), dtype=T, device="cuda")
        w[0, 1], w[1, 1] = 200, -200
        x = torch.zeros((rows, C), dtype=T, device="cuda")
        x[:, 0] = 1 - 2.0 * (torch.arange(rows, device="cuda") % 2)
        x[:, 1] = 1
        targets = torch.ones(rows, dtype=torch.int32, device="cuda")
        op = P.TokenLoss(vocab=V, width=C, max_rows=rows, dtype=dtype, weight_dtype=dtype, cuda_stream=stream())
        loss, lse = torch.zeros((2, rows), device="cuda")
        dw = torch.zeros((V, C), device="cuda")
        op.step(rows, x, C, w, 0, targets, factor, 1.0, loss, lse, None, C, dw, 0)
        want = -(factor.double() @ x[:, 0].double())
        e = 1.01 * rows * (2.0 ** -24 * (1 + 3) + 5 * STEP)
        assert abs(float(dw[1, 0]) - float(want)) <= e + U * abs(float(want))
        assert abs(float(dw[0, 0]) + float(want)) <= e + U * abs(float(want))
        if rows == 16:
            assert rows / 2 * lost > 2 * e
        op.destroy()


@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("dtype", [1, 2])
@pytest.mark.parametrize("rows", [3, 20, 300])
def test_a_loss_of_fp32_weights_keeps_24_bits(P, rows, dtype, pad):  # noqa: F811
    """Logits that are the differences of weights, of which two bf16 parts lose most."""
    V, C, T = 70, 16, TYPES[dtype]
    signs = torch.tensor([1.0, -1.0], device="cuda").repeat(8)
    x, _ = rows_of(signs.expand(rows, C), pad, T)
    w = torch.full((V, C), 1 + 2.0 ** -9, device="cuda")
    w[0, ::2] += 2.0 ** -17 - 2.0 ** -22  # the first column's logit is 8 of them, the others' 0
    targets = torch.zeros(rows, dtype=torch.int32, device="cuda")
    op = P.TokenLoss(vocab=V, width=C, max_rows=rows, dtype=dtype, cuda_stream=stream())
    loss, lse = torch.zeros((2, rows), device="cuda")
    op.forward(rows, x, x.stride(0), w, 0, targets, None, loss, lse)
    z = w.double() @ signs.double()
    want = torch.logsumexp(z, 0)
    e = 1.01 * 16 * (2.0 ** -24 * (1 + 3) + 5 * STEP)
    within(lse, want.expand(rows), e + 16 * U * want, "lse")
    want = want - z[0]
    within(loss, want.expand(rows), 2 * e + 24 * U * want, "loss")
    assert float(z[0]) > 2 * e + 24 * U * float(want)
    op.destroy()


def test_small_parts_are_summed_before_large_ones(P):  # noqa: F811
    """320 rows whose gradient at the target is -(1.5 + d), d below 2^-9 of what 24 bits leave: the 1.5 add up exactly, and
    what lies below them is lost once, when the sum grows past it, not at every step of its own."""
    rows, V, C, T = 320, 2, 8, torch.bfloat16
    factor = 1.5 + 2.0 ** -9 * torch.rand(rows, generator=gen(4), device="cuda")
    w = torch.zeros((V, C), dtype=T, device="cuda")
    w[0, 1], w[1, 1] = 200, -200
    x = torch.zeros((rows, C), dtype=T, device="cuda")
    x[:, :2] = 1
    targets = torch.ones(rows, dtype=torch.int32, device="cuda")
    op = P.TokenLoss(vocab=V, width=C, max_rows=rows, dtype=P.BF16, weight_dtype=P.BF16, cuda_stream=stream())
    loss, lse = torch.zeros((2, rows), device="cuda")
    dw = torch.zeros((V, C), device="cuda")
    op.step(rows, x, C, w, 0, targets, factor, 1.0, loss, lse, None, C, dw, 0)
    want = float(factor.double().sum())
    # one accumulator: its last unit is 2^-15, those that it grew through add up to as much, each lost twice at most; the
    # small parts' sums are below 1, in 20 steps each
    e = 2 * 2 * 2.0 ** -15 + 40 * STEP
    assert abs(float(dw[1, 0]) + want) <= e, (float(dw[1, 0]), want, e)
    assert abs(float(dw[0, 0]) - want) <= e
    op.destroy()
