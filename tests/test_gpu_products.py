"""Linear layers, token loss and gradient clipping against their definitions in 64 bits, with bounds derived from the
formulas (product_references): every type, one row to several tiles of everything, odd sizes, rows that are not aligned,
shared and missing parameters, rows that do not count."""
from __future__ import annotations

import math

import pytest

from operator_references import U, rounded, within
from product_references import DTYPES, linear_backward, linear_forward, token_loss

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def P():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2010_13359_gb300 as P
    return P


def stream():
    return torch.cuda.current_stream().cuda_stream


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rows_of(values, pad, dtype, shift=0):
    """The values as rows of a larger buffer, `pad` values between them and `shift` before the first; the unused ones
    are NaN."""
    R, C = values.shape
    flat = torch.full((shift + R * (C + pad),), math.nan, dtype=dtype, device="cuda")
    view = flat[shift:].view(R, C + pad)[:, :C]
    view.copy_(values)
    return view, flat


def untouched(flat, R, C, pad, shift=0):
    return bool(flat[:shift].isnan().all()) and bool(flat[shift:].view(R, C + pad)[:, C:].isnan().all())


# ---------------------------------------------------------------------------
# linear layers
# ---------------------------------------------------------------------------

LINEAR = [  # workers, rows, inputs, outputs, dtype, weight dtype, activation, pad, shift, shared
    (1, 1, 1, 1, 0, 0, 0, 0, 0, False),
    (1, 1, 8, 8, 1, 1, 0, 0, 0, False),
    (1, 128, 64, 64, 1, 1, 0, 0, 0, False),
    (2, 3, 17, 5, 1, 1, 2, 0, 0, False),
    (3, 5, 33, 7, 2, 2, 3, 1, 1, True),
    (2, 7, 64, 129, 0, 0, 1, 3, 1, False),
    (1, 130, 65, 100, 2, 0, 2, 0, 0, False),
    (4, 4, 512, 512, 1, 0, 2, 0, 0, False),
    (1, 1, 4096, 1000, 1, 1, 0, 0, 0, False),
    (2, 129, 200, 260, 1, 1, 1, 8, 0, True),
    (2, 300, 513, 255, 2, 2, 1, 0, 0, False),
    (1, 77, 1030, 515, 0, 0, 3, 5, 0, False),
    (1, 2000, 72, 40, 1, 1, 2, 0, 0, False),
    (2, 1300, 640, 1300, 1, 1, 2, 0, 0, False),
    (3, 700, 328, 2056, 1, 0, 0, 0, 0, False),
    (1, 1281, 2049, 2050, 2, 0, 3, 0, 0, False),
    (2, 900, 300, 2100, 0, 0, 2, 0, 0, True),
    (16, 33, 96, 160, 2, 2, 0, 0, 0, False),
    (1, 20000, 48, 24, 1, 1, 0, 0, 0, False),
    (2, 70, 61, 125, 1, 1, 2, 3, 0, False),
    (1, 300, 509, 1021, 2, 2, 0, 3, 0, False),
    (1, 1400, 1021, 2301, 1, 1, 1, 3, 0, False),
    (2, 8, 4104, 77, 1, 0, 3, 0, 0, False),
    (1, 9, 2050, 130, 0, 0, 0, 2, 0, False),
    (1, 20, 65536, 9, 1, 1, 0, 0, 0, False),
    (1, 20, 9, 65536, 1, 1, 2, 0, 0, False),
    (200, 10, 16, 24, 1, 1, 2, 0, 0, False),
    (2, 600, 130, 1301, 1, 1, 3, 3, 1, False),
    (3, 100, 77, 203, 0, 0, 2, 3, 3, False),
    (2, 8, 1300, 2101, 1, 1, 2, 3, 1, True),
    (5, 6, 2052, 500, 2, 0, 1, 0, 0, False),
    (1, 2, 4096, 1024, 0, 0, 3, 0, 0, False),
]


def linear_data(workers, rows, inputs, outputs, dtype, weight_dtype, act, pad, shift, shared):
    g = gen(rows * 1000 + outputs)
    T, E = DTYPES[dtype], DTYPES[weight_dtype]
    held = 1 if shared else workers
    n = workers * rows
    x, _ = rows_of(torch.randn((n, inputs), generator=g, device="cuda") * torch.exp(
        torch.randn(inputs, generator=g, device="cuda")), pad, T, shift)
    stride = inputs * outputs + (0 if outputs % 8 == 0 else 3)
    weight = torch.full((held, stride), math.nan, dtype=E, device="cuda")
    weight[:, :inputs * outputs] = torch.randn((held, inputs * outputs), generator=g, device="cuda") / math.sqrt(inputs)
    bias = torch.randn((held, outputs + 1), generator=g, device="cuda")
    residual, _ = rows_of(torch.randn((n, outputs), generator=g, device="cuda"), pad, T, shift)
    dy, _ = rows_of(torch.randn((n, outputs), generator=g, device="cuda") * 1e-2, pad, T, shift)
    pre, _ = rows_of(torch.randn((n, outputs), generator=g, device="cuda") * 2, pad, T, shift)
    return x, weight, bias, residual, dy, pre


def linear_operator(P, shape):
    workers, rows, inputs, outputs, dtype, weight_dtype, act = shape[:7]
    return P.Linear(inputs=inputs, outputs=outputs, max_rows=rows, workers=workers, dtype=dtype, weight_dtype=weight_dtype,
                    activation=act, cuda_stream=stream())


@pytest.mark.parametrize("shape", LINEAR, ids=str)
def test_linear_forward(P, shape):
    workers, rows, inputs, outputs, dtype, weight_dtype, act, pad, shift, shared = shape
    x, weight, bias, residual, _, _ = linear_data(*shape)
    T, n = DTYPES[dtype], workers * rows
    op = linear_operator(P, shape)
    y, y_flat = rows_of(torch.full((n, outputs), math.nan), pad, T, shift)
    pre, pre_flat = rows_of(torch.full((n, outputs), math.nan), pad, T, shift)
    plain, _ = rows_of(torch.full((n, outputs), math.nan), pad, T, shift)
    p_stride, b_stride = (0, 0) if shared else (weight.stride(0), bias.stride(0))
    op.forward(rows, x, x.stride(0), weight, p_stride, bias, b_stride, residual, residual.stride(0), y, y.stride(0), pre,
               pre.stride(0))
    op.forward(rows, x, x.stride(0), weight, p_stride, None, 0, None, 0, plain, plain.stride(0))
    op.synchronize()
    for m in range(workers):
        part, held = slice(m * rows, (m + 1) * rows), 0 if shared else m
        w = weight[held, :inputs * outputs].double().view(outputs, inputs)
        b = bias[held, :outputs].double()
        want, u, e_y, e_u = linear_forward(x[part].double(), w, b, residual[part].double(), act, dtype, weight_dtype)
        within(pre[part], u, e_u, "pre")
        within(y[part], want, e_y, "y")
        want, _, e_y, _ = linear_forward(x[part].double(), w, 0 * b, 0 * residual[part].double(), act, dtype, weight_dtype)
        within(plain[part], want, e_y, "y without bias and residual")
    assert untouched(y_flat, n, outputs, pad, shift) and untouched(pre_flat, n, outputs, pad, shift)
    # the residual's place as y's: the same bits
    op.forward(rows, x, x.stride(0), weight, p_stride, bias, b_stride, residual, residual.stride(0), residual,
               residual.stride(0))
    assert torch.equal(residual, y)
    op.destroy()


@pytest.mark.parametrize("shape", LINEAR, ids=str)
def test_linear_backward(P, shape):
    workers, rows, inputs, outputs, dtype, weight_dtype, act, pad, shift, shared = shape
    x, weight, _, _, dy, pre = linear_data(*shape)
    T, n = DTYPES[dtype], workers * rows
    op = linear_operator(P, shape)
    dx, dx_flat = rows_of(torch.full((n, inputs), math.nan), pad, T, shift)
    d = inputs * outputs
    g = torch.full((workers, d + outputs + 5), math.nan, device="cuda")
    args = (rows, dy, dy.stride(0), x, x.stride(0), weight, 0 if shared else weight.stride(0), pre if act else None,
            pre.stride(0))
    op.backward(*args, dx, dx.stride(0), g, g[:, d:], g.stride(0))
    op.synchronize()
    for m in range(workers):
        part, held = slice(m * rows, (m + 1) * rows), 0 if shared else m
        w = weight[held, :d].double().view(outputs, inputs)
        want, dw, db, e_dx, e_dw, e_db = linear_backward(dy[part].double(), x[part].double(), w, pre[part].double(), act,
                                                         dtype, weight_dtype)
        within(dx[part], want, e_dx, "dx")
        within(g[m, :d].view(outputs, inputs), dw, e_dw, "dweight")
        within(g[m, d:d + outputs], db, e_db, "dbias")
    assert untouched(dx_flat, n, inputs, pad, shift) and bool(g[:, d + outputs:].isnan().all())
    # added to what is there, and each result alone: the same values
    base = torch.randn((workers, g.shape[1]), generator=gen(1), device="cuda")
    added, alone = base.clone(), base.clone()
    op.backward(*args, None, 0, added, added[:, d:], g.stride(0), accumulate=True)
    op.backward(*args, None, 0, alone, None, g.stride(0))
    assert torch.equal(alone[:, :d], g[:, :d]) and torch.equal(alone[:, d:], base[:, d:])
    total = base[:, :d + outputs].double() + g[:, :d + outputs].double()
    within(added[:, :d + outputs], total, 2 * U * (total.abs() + g[:, :d + outputs].double().abs()), "added")
    assert torch.equal(added[:, d + outputs:], base[:, d + outputs:])
    op.destroy()


# ---------------------------------------------------------------------------
# token loss
# ---------------------------------------------------------------------------

LOSS = [  # workers, rows, vocab, width, dtype, weight dtype, token bits, pad, shift, shared, masked
    (1, 1, 1, 1, 0, 0, 32, 0, 0, False, 0.0),
    (1, 1, 2, 8, 1, 1, 64, 0, 0, False, 0.0),
    (2, 3, 10, 17, 1, 1, 32, 1, 1, False, 0.3),
    (1, 129, 257, 64, 1, 1, 32, 0, 0, False, 0.2),
    (3, 40, 500, 33, 2, 2, 64, 3, 1, True, 0.3),
    (2, 33, 1000, 129, 0, 0, 32, 1, 0, False, 0.1),
    (1, 4, 5003, 256, 1, 0, 64, 0, 0, False, 0.0),
    (4, 100, 777, 96, 2, 0, 32, 0, 0, False, 0.5),
    (2, 300, 3001, 200, 1, 1, 32, 8, 0, True, 0.1),
    (1, 1000, 9000, 320, 1, 1, 32, 0, 0, False, 0.05),
    (1, 700, 8200, 72, 0, 0, 32, 0, 0, False, 0.05),
    (2, 600, 4100, 136, 2, 2, 32, 0, 0, False, 0.05),
    (1, 257, 20000, 104, 1, 0, 32, 0, 0, False, 1.0),
    (100, 5, 40, 24, 1, 1, 32, 0, 0, False, 0.2),
    (1, 33, 70, 65536, 1, 1, 32, 0, 0, False, 0.0),
    (1, 300, 600, 4096, 1, 1, 32, 0, 0, False, 0.1),  # few tiles: their logits' sums in pieces
    (2, 600, 2000, 3000, 0, 0, 32, 0, 0, False, 0.1),
    (1, 300, 600, 2048, 2, 0, 32, 0, 0, False, 0.1),
    (3, 8, 5001, 260, 1, 1, 32, 3, 1, False, 0.4),
    (2, 6, 3000, 1001, 0, 0, 64, 0, 0, True, 0.3),
    (1, 2, 20011, 512, 2, 2, 32, 0, 0, False, 0.0),
]


def loss_data(workers, rows, vocab, width, dtype, weight_dtype, bits, pad, shift, shared, masked):
    g = gen(rows * 1000 + vocab)
    n, held = workers * rows, 1 if shared else workers
    stride = vocab * width + (0 if width % 8 == 0 and vocab % 2 else 5)
    weight = torch.full((held, stride), math.nan, dtype=DTYPES[weight_dtype], device="cuda")
    weight[:, :vocab * width] = torch.randn((held, vocab * width), generator=g, device="cuda") / math.sqrt(width) * 2
    targets = torch.randint(0, vocab, (n,), generator=g, device="cuda")
    x = torch.randn((n, width), generator=g, device="cuda")
    out = torch.rand(n, generator=g, device="cuda") < masked
    weights = 0.5 + torch.rand(n, generator=g, device="cuda")
    weights[out & (torch.rand(n, generator=g, device="cuda") < 0.5)] = 0
    gone = out & (weights != 0)
    targets[gone] = torch.where(torch.rand(n, generator=g, device="cuda") < 0.5, -1, vocab)[gone]
    x[out] = math.nan  # what rows that do not count hold does not matter
    x, _ = rows_of(x, pad, DTYPES[dtype], shift)
    return x, weight, targets.to(torch.int32 if bits == 32 else torch.int64), weights


@pytest.mark.parametrize("shape", LOSS, ids=str)
def test_token_loss(P, shape):
    workers, rows, vocab, width, dtype, weight_dtype, bits, pad, shift, shared, masked = shape
    x, weight, targets, weights = loss_data(*shape)
    T, n, d = DTYPES[dtype], workers * rows, vocab * width
    scale = 1024.0 / rows if dtype == 2 else 1.0 / rows
    op = P.TokenLoss(vocab=vocab, width=width, max_rows=rows, workers=workers, dtype=dtype, weight_dtype=weight_dtype,
                     token_bits=bits, cuda_stream=stream())
    loss, lse, loss_step, lse_step = torch.full((4, n), math.nan, device="cuda")
    data = (rows, x, x.stride(0), weight, 0 if shared else weight.stride(0), targets, weights)
    op.forward(*data, loss, lse)
    dx, dx_flat = rows_of(torch.full((n, width), math.nan), pad, T, shift)
    g = torch.full((workers, d + 3), math.nan, device="cuda")
    op.backward(*data, lse, scale, dx, dx.stride(0), g, g.stride(0))
    dx_step, _ = rows_of(torch.full((n, width), math.nan), pad, T, shift)
    g_step = torch.full((workers, d + 3), math.nan, device="cuda")
    op.step(*data, scale, loss_step, lse_step, dx_step, dx_step.stride(0), g_step, g_step.stride(0))
    op.synchronize()
    for m in range(workers):
        part = slice(m * rows, (m + 1) * rows)
        w = weight[0 if shared else m, :d].double().view(vocab, width)
        args = (x[part].double(), w, targets[part].long(), weights[part].double(), scale, dtype, weight_dtype)
        w_loss, w_lse, _, _, e_loss, e_lse, _, _ = token_loss(*args)
        within(loss[part], w_loss, e_loss, "loss")
        within(lse[part], w_lse, e_lse, "lse")
        _, _, w_dx, w_dw, _, _, e_dx, e_dw = token_loss(*args, lse=lse[part].double())
        within(dx[part], w_dx, e_dx, "dx")
        within(g[m, :d].view(vocab, width), w_dw, e_dw, "dweight")
    assert untouched(dx_flat, n, width, pad, shift) and bool(g[:, d:].isnan().all())
    # the step is the two calls
    assert torch.equal(dx_step, dx) and torch.equal(g_step[:, :d], g[:, :d])
    assert torch.equal(loss_step, loss) and torch.equal(lse_step, lse)
    # added to what is there; no lse and no dx asked for
    base = torch.randn((workers, d + 3), generator=gen(1), device="cuda")
    added = base.clone()
    op.step(*data, scale, loss_step, None, None, 0, added, added.stride(0), accumulate=True)
    total = base[:, :d].double() + g[:, :d].double()
    within(added[:, :d], total, 2 * U * (total.abs() + g[:, :d].double().abs()), "added")
    assert torch.equal(added[:, d:], base[:, d:])
    op.destroy()


# ---------------------------------------------------------------------------
# gradient clipping
# ---------------------------------------------------------------------------

CLIP = [  # workers, sizes, dtype, out dtype, pad, shift
    (1, (1,), 0, 0, 0, 0),
    (3, (5, 0, 1, 17), 0, 0, 0, 0),
    (2, (16384, 16385, 40000, 3), 1, 0, 0, 0),
    (4, (100_003, 7, 65_536), 2, 0, 1, 1),
    (8, (1_000_000, 33), 0, 0, 3, 1),
    (1, tuple(range(1, 700)), 1, 0, 0, 0),
    (700, (50, 20_000), 1, 1, 0, 0),
    (2, tuple(37 * (i % 11) for i in range(1500)), 2, 2, 1, 0),
    (1, (30_000_001,), 0, 0, 0, 1),
    (3, (40_001, 20_000, 8, 15, 16_385), 0, 0, 3, 2),
    (2, (70_003, 33_333, 5), 1, 0, 5, 3),
    (2, (70_003, 33_333, 9), 2, 2, 7, 5),
]


@pytest.mark.parametrize("shape", CLIP, ids=lambda s: str(s)[:60])
@pytest.mark.parametrize("share", [0.25, 4.0])
def test_gradient_clip(P, shape, share):
    workers, sizes, dtype, out_dtype, pad, shift = shape
    g = gen(len(sizes) + workers)
    T, O = DTYPES[dtype], DTYPES[out_dtype]
    tensors = [rows_of(torch.randn((workers, n), generator=g, device="cuda") * math.exp(i % 5 - 2), pad, T, shift)[0]
               for i, n in enumerate(sizes)]
    total = sum(sizes)
    out = torch.full((workers, total + 4), math.nan, dtype=O, device="cuda")
    at, places = 0, []
    for n in sizes:
        places.append((out[:, at:], n, out.stride(0)))
        at += n
    values = torch.cat([t.double() for t in tensors], 1)
    want = values.square().sum(1).sqrt()
    op = P.GradientClip(workers=workers, dtype=dtype, out_dtype=out_dtype, eps=1e-6, cuda_stream=stream())
    lists = P.TensorList([(t, n, t.stride(0)) for t, n in zip(tensors, sizes)]), P.TensorList(places)
    norms, again = torch.full((2, workers), math.nan, device="cuda")
    op.norm(lists[0], norms)
    # a thread's fp32 sums have at most 64 terms, each rounded; then fp64; the square root halves the error
    e_norm = want * 34 * U
    within(norms, want, e_norm, "norms")
    max_norm = float(share * want.median())
    op.clip(*lists, max_norm, again)
    op.synchronize()
    assert torch.equal(norms, again)
    import numpy as np
    limit = float(np.float32(max_norm))
    factor = (limit / (want + float(np.float32(1e-6)))).clamp(max=1)
    clipped = values * factor[:, None]
    within(out[:, :total], clipped, 40 * U * clipped.abs() + rounded(clipped.abs() * (1 + 40 * U), O), "clipped")
    if out_dtype == dtype:
        keep = torch.cat(tensors, 1)
        assert torch.equal(out[factor == 1][:, :total], keep[factor == 1])  # below the limit: the same bits
        # in place
        op.clip(lists[0], lists[0], max_norm)
        assert torch.equal(torch.cat(tensors, 1), out[:, :total])
    assert bool(out[:, total:].isnan().all())
    op.destroy()
