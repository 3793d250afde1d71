"""The token-model operators against their definitions in 64 bits, with bounds derived from the
formulas (operator_references): every type, odd sizes, rows that are not aligned, shared and missing
parameters, masks that leave nothing, gradients against the formula and against differences."""
from __future__ import annotations

import math

import numpy as np
import pytest

from operator_references import U, chain, distillation, norm_backward, norm_forward, rounded, within

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DTYPES = {0: torch.float32, 1: torch.bfloat16, 2: torch.float16}


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
    """The values as rows of a larger buffer, `pad` values between them and `shift` before the first; the
    unused ones are NaN."""
    R, C = values.shape
    flat = torch.full((shift + R * (C + pad),), math.nan, dtype=dtype, device="cuda")
    view = flat[shift:].view(R, C + pad)[:, :C]
    view.copy_(values)
    return view, flat


def untouched(flat, R, C, pad, shift=0):
    """Whether the unused values of rows_of's buffer are still NaN."""
    return bool(flat[:shift].isnan().all()) and bool(flat[shift:].view(R, C + pad)[:, C:].isnan().all())


# ---------------------------------------------------------------------------
# layer norm
# ---------------------------------------------------------------------------

NORM = [  # workers, rows, width, dtype, pad, shift, shared
    (1, 1, 1, 0, 0, 0, False),
    (1, 3, 2, 1, 0, 0, False),
    (2, 5, 31, 2, 1, 0, False),
    (3, 7, 33, 0, 3, 1, True),
    (1, 9, 64, 1, 8, 0, False),
    (2, 4, 127, 1, 0, 1, False),
    (4, 4, 512, 1, 0, 0, False),
    (1, 1000, 128, 0, 0, 0, False),
    (2, 65, 1000, 2, 8, 0, False),
    (2, 33, 1024, 1, 0, 0, True),
    (3, 37, 1537, 0, 3, 0, False),
    (1, 300, 1536, 1, 8, 0, False),
    (2, 129, 2048, 0, 0, 0, False),
    (1, 50, 2056, 1, 0, 0, False),
    (16, 20, 4096, 1, 0, 0, False),
    (1, 700, 4100, 0, 4, 0, True),
    (2, 11, 5001, 1, 0, 0, False),
    (1, 333, 8192, 2, 0, 0, False),
    (1, 40, 8200, 0, 0, 0, False),
    (2, 21, 12289, 1, 3, 0, False),
    (1, 200, 16384, 1, 0, 0, False),
    (1, 9, 16384, 0, 0, 0, False),
    (1, 6, 16392, 1, 0, 0, False),
    (2, 3, 40001, 0, 0, 0, False),
    (1, 2, 65536, 1, 0, 0, False),
]


def norm_data(workers, rows, width, dtype, pad, shift, shared):
    g = gen(width * 1000 + rows)
    x = torch.randn((workers * rows, width), generator=g, device="cuda") * torch.exp(
        torch.randn(width, generator=g, device="cuda")) + torch.randn((workers * rows, 1), generator=g, device="cuda")
    dy = torch.randn((workers * rows, width), generator=g, device="cuda") * 1e-2
    stride = 2 * width + 5
    params = torch.randn((1 if shared else workers, stride), generator=g, device="cuda")
    x, x_flat = rows_of(x, pad, DTYPES[dtype], shift)
    dy, _ = rows_of(dy, pad, DTYPES[dtype], shift)
    return x, dy, params, 0 if shared else stride


def per_row(params, workers, rows, first, width):
    p = params[:, first:first + width].double().expand(workers, width)
    return p.repeat_interleave(rows, 0)


@pytest.mark.parametrize("shape", NORM, ids=str)
def test_layer_norm_forward(P, shape):
    workers, rows, width, dtype, pad, shift, shared = shape
    x, _, params, p_stride = norm_data(*shape)
    T = DTYPES[dtype]
    op = P.LayerNorm(width=width, workers=workers, dtype=dtype, eps=1e-5, cuda_stream=stream())
    n = workers * rows
    y, y_flat = rows_of(torch.full((n, width), math.nan), pad, T, shift)
    mean, rstd = torch.full((2, n), math.nan, device="cuda")
    op.forward(rows, x, x.stride(0), params, params[:, width:], p_stride, y, y.stride(0), mean, rstd)
    want, w_mean, w_rstd, e_y, e_mean, e_rstd = norm_forward(
        x.double(), per_row(params, workers, rows, 0, width), per_row(params, workers, rows, width, width),
        float(np.float32(1e-5)))
    within(y, want, e_y + rounded(want.abs() + e_y, T), "y")
    within(mean, w_mean[:, 0], e_mean[:, 0], "mean")
    within(rstd, w_rstd[:, 0], e_rstd[:, 0], "rstd")
    assert untouched(y_flat, n, width, pad, shift)
    # without parameters and statistics; and in place: the same bits as beside
    plain, _ = rows_of(torch.zeros((n, width)), pad, T, shift)
    op.forward(rows, x, x.stride(0), None, None, 0, plain, plain.stride(0))
    ones = torch.ones(1, dtype=torch.float64, device="cuda")
    want, _, _, e_y, _, _ = norm_forward(x.double(), ones, 0 * ones, float(np.float32(1e-5)))
    within(plain, want, e_y + rounded(want.abs() + e_y, T), "y without parameters")
    op.forward(rows, x, x.stride(0), params, params[:, width:], p_stride, x, x.stride(0))
    assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))
    op.destroy()


@pytest.mark.parametrize("shape", NORM, ids=str)
def test_layer_norm_backward(P, shape):
    workers, rows, width, dtype, pad, shift, shared = shape
    x, dy, params, p_stride = norm_data(*shape)
    T, n = DTYPES[dtype], workers * rows
    op = P.LayerNorm(width=width, workers=workers, dtype=dtype, eps=1e-5, cuda_stream=stream())
    xd = x.double()
    mean = xd.mean(1).float()
    rstd = (1 / torch.sqrt((xd - mean.double()[:, None]).square().mean(1) + 1e-5)).float()
    dx, dx_flat = rows_of(torch.full((n, width), math.nan), pad, T, shift)
    g = torch.full((workers, 2 * width + 3), math.nan, device="cuda")
    args = (rows, dy, dy.stride(0), x, x.stride(0), params, p_stride, mean, rstd)
    op.backward(*args, dx, dx.stride(0), g, g[:, width:], g.stride(0))
    want, tw, tb, e = norm_backward(dy.double(), xd, per_row(params, workers, rows, 0, width), mean.double()[:, None],
                                    rstd.double()[:, None])
    within(dx, want, e + rounded(want.abs() + e, T), "dx")
    assert untouched(dx_flat, n, width, pad, shift)
    for what, terms, got in (("dweight", tw, g[:, :width]), ("dbias", tb, g[:, width:2 * width])):
        terms = terms.view(workers, rows, width)
        # a sum over the rows, each term off by a few u
        within(got, terms.sum(1), (rows + 24) * U * terms.abs().sum(1), what)
    assert bool(g[:, 2 * width:].isnan().all())
    # twice: the same bits; added to; each output alone; dx in dy's place
    g2 = torch.full_like(g, math.nan)
    op.backward(*args, None, 0, g2, None, g.stride(0))
    op.backward(*args, None, 0, None, g2[:, width:], g.stride(0))
    assert torch.equal(g2[:, :2 * width], g[:, :2 * width])
    g2[:, :2 * width] = torch.randn((workers, 2 * width), generator=gen(1), device="cuda")
    before = g2.clone()
    op.backward(*args, dy, dy.stride(0), g2, g2[:, width:], g.stride(0), accumulate=True)
    assert torch.equal(g2[:, :2 * width], (before + g)[:, :2 * width])
    assert torch.equal(dy.contiguous().view(torch.uint8), dx.contiguous().view(torch.uint8))
    op.destroy()


def test_layer_norm_of_constant_and_huge_rows(P):
    """A row of one value has variance 0 and y = bias; values whose plain sum of squares would overflow after the
    mean is taken do not appear in 16 bits, but a large offset must not cost the small deviations."""
    op = P.LayerNorm(width=1024, dtype=0, eps=1e-5, cuda_stream=stream())
    x = torch.randn((3, 1024), generator=gen(3), device="cuda")
    x[0] = 7.25
    x[1] = 3e4 + x[1]
    y = torch.empty_like(x)
    mean, rstd = torch.empty((2, 3), device="cuda")
    bias = torch.randn(1024, generator=gen(4), device="cuda")
    op.forward(3, x, 1024, None, bias, 0, y, 1024, mean, rstd)
    assert torch.equal(y[0], bias)
    want, _, w_rstd, e_y, _, e_rstd = norm_forward(x.double(), torch.ones(1, device="cuda").double(), bias.double()[None],
                                                   float(np.float32(1e-5)))
    within(y, want, e_y + rounded(want, torch.float32), "y")
    within(rstd, w_rstd[:, 0], e_rstd[:, 0], "rstd")
    op.destroy()


def test_layer_norm_nan_stays_in_its_row(P):
    op = P.LayerNorm(width=300, dtype=0, cuda_stream=stream())
    x = torch.randn((5, 300), generator=gen(5), device="cuda")
    x[1, 17], x[3, 299] = math.nan, math.inf
    y = torch.empty_like(x)
    op.forward(5, x, 300, None, None, 0, y, 300)
    assert y[1].isnan().all() and y[3].isnan().any() and not y[[0, 2, 4]].isnan().any()
    op.destroy()


@pytest.mark.parametrize("width", [5, 48])
def test_layer_norm_gradient_is_the_differences(P, width):
    """dx, dweight, dbias against central differences of the definition in 64 bits."""
    rows = 3
    g = gen(width)
    x, dy = torch.randn((2, rows, width), generator=g, device="cuda")
    w, b = torch.randn((2, width), generator=g, device="cuda")
    op = P.LayerNorm(width=width, dtype=0, cuda_stream=stream())
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty((2, rows), device="cuda")
    grads = torch.empty(2 * width, device="cuda")
    op.forward(rows, x, width, w, b, 0, y, width, mean, rstd)
    op.backward(rows, dy, width, x, width, w, 0, mean, rstd, dx, width, grads, grads[width:], 0)

    def loss(x, w, b):
        return float((norm_forward(x, w, b, float(np.float32(1e-5)))[0] * dy.double()).sum())

    inputs = [x.double(), w.double(), b.double()]
    for i, got in enumerate((dx, grads[:width], grads[width:])):
        flat = inputs[i].view(-1)
        diff = torch.empty(flat.numel(), dtype=torch.float64)
        for j in range(flat.numel()):
            keep = float(flat[j])
            step = 1e-5
            flat[j] = keep + step
            up = loss(*inputs)
            flat[j] = keep - step
            diff[j] = (up - loss(*inputs)) / (2 * step)
            flat[j] = keep
        # 32-bit gradient of values of order 1 over sums of `width` terms; differences good to 1e-8
        size = float(diff.abs().max())
        assert float((got.double().cpu().view(-1) - diff).abs().max()) <= 64 * U * (size + 1) + 1e-7


# ---------------------------------------------------------------------------
# embedding
# ---------------------------------------------------------------------------

EMBED = [  # workers, tokens, vocab, width, dtype, table, bits, pad, shared, how the tokens fall
    (1, 1, 1, 1, 0, 0, 32, 0, False, "uniform"),
    (2, 3, 7, 5, 1, 0, 64, 1, False, "uniform"),
    (2, 333, 1009, 129, 0, 0, 32, 0, False, "zipf"),
    (3, 100, 50, 64, 2, 1, 32, 8, True, "zipf"),
    (1, 257, 1000, 1024, 1, 0, 64, 0, False, "zipf"),
    (2, 1000, 3, 48, 1, 2, 32, 0, False, "uniform"),
    (1, 3000, 40, 100, 0, 0, 32, 3, False, "one"),
    (1, 5000, 100, 256, 1, 0, 32, 0, False, "one"),
    (8, 4096, 2000, 64, 1, 0, 32, 0, False, "zipf"),
    (1, 4097, 100_003, 16, 0, 0, 64, 0, False, "uniform"),
    (2, 20_001, 30_011, 40, 2, 0, 32, 8, False, "zipf"),
    (1, 150_000, 131_072, 8, 0, 0, 64, 0, False, "zipf"),
    (1, 150_000, 200_003, 24, 1, 1, 32, 0, False, "none"),
    (1, 70_000, 1, 33, 0, 0, 32, 0, False, "uniform"),
    (2, 300, 17, 8192, 1, 0, 32, 0, False, "zipf"),
    (1, 40, 11, 20_001, 0, 0, 32, 0, False, "uniform"),
    (1, 33, 5, 65_536, 2, 2, 32, 0, False, "uniform"),
    (300, 5, 20, 12, 0, 0, 32, 0, False, "uniform"),
    (5, 20_000, 700, 20, 0, 0, 32, 0, False, "sorted"),
]


def tokens_of(workers, tokens, vocab, bits, how, seed, masked=0.1):
    g = gen(seed)
    shape = (workers, tokens)
    if how == "zipf":
        p = 1 / (torch.arange(vocab, device="cuda", dtype=torch.float64) + 2.7)
        r = torch.rand(shape, generator=g, device="cuda", dtype=torch.float64)
        ids = torch.searchsorted(torch.cumsum(p / p.sum(), 0), r).clamp_(max=vocab - 1)
        ids = torch.randperm(vocab, generator=g, device="cuda")[ids]
    elif how == "one":
        ids = torch.full(shape, vocab // 2, device="cuda")
        other = torch.rand(shape, generator=g, device="cuda") < 0.05
        ids[other] = torch.randint(0, vocab, (int(other.sum()),), generator=g, device="cuda")
    else:
        ids = torch.randint(0, vocab, shape, generator=g, device="cuda")
        if how == "sorted":
            ids = ids.sort(1).values
    no = torch.rand(shape, generator=g, device="cuda") < (1.0 if how == "none" else masked)
    outside = torch.tensor([-1, vocab, -(2 ** 31), 2 ** 31 - 1] + ([2 ** 32, -(2 ** 32), 2 ** 40] if bits == 64 else []),
                           device="cuda")
    ids[no] = outside[torch.randint(0, len(outside), (int(no.sum()),), generator=g, device="cuda")]
    return ids.to(torch.int32 if bits == 32 else torch.int64)


@pytest.mark.parametrize("case", EMBED, ids=str)
def test_embedding_forward(P, case):
    workers, tokens, vocab, width, dtype, table, bits, pad, shared, how = case
    ids = tokens_of(workers, tokens, vocab, bits, how, tokens)
    p_stride = vocab * width + 7
    params = torch.randn((1 if shared else workers, p_stride), generator=gen(2), device="cuda").to(DTYPES[table])
    op = P.Embedding(vocab=vocab, width=width, max_tokens=tokens + 3, workers=workers, table_dtype=table, dtype=dtype,
                     token_bits=bits, scale=1.7, cuda_stream=stream())
    n = workers * tokens
    y, flat = rows_of(torch.full((n, width), math.nan), pad, DTYPES[dtype])
    op.forward(tokens, ids, params, 0 if shared else p_stride, y, y.stride(0))
    there = (ids >= 0) & (ids < vocab)
    at = ids.long().clamp(0, vocab - 1)
    for m in range(workers):
        rows = params[0 if shared else m, :vocab * width].view(vocab, width)[at[m]].float() * np.float32(1.7).item()
        want = torch.where(there[m][:, None], rows, torch.zeros((), device="cuda")).to(DTYPES[dtype])
        assert torch.equal(y[m * tokens:(m + 1) * tokens], want)  # one product, rounded once
    assert untouched(flat, n, width, pad)
    op.destroy()


@pytest.mark.parametrize("case", EMBED, ids=str)
def test_embedding_backward(P, case):
    workers, tokens, vocab, width, dtype, table, bits, pad, shared, how = case
    ids = tokens_of(workers, tokens, vocab, bits, how, tokens)
    n, scale = workers * tokens, float(np.float32(1.7))
    there = (ids >= 0) & (ids < vocab)
    dy = torch.randn((n, width), generator=gen(7), device="cuda")
    dy[~there.view(-1)] = math.nan  # not read
    dy, _ = rows_of(dy, pad, DTYPES[dtype])
    op = P.Embedding(vocab=vocab, width=width, max_tokens=tokens, workers=workers, table_dtype=table, dtype=dtype,
                     token_bits=bits, scale=1.7, cuda_stream=stream())
    g_stride = vocab * width + 5
    g = torch.full((workers, g_stride), math.nan, device="cuda")
    op.backward(tokens, ids, dy, dy.stride(0), g, g_stride)
    want, size = torch.zeros((2, workers * vocab, width), dtype=torch.float64, device="cuda")
    at = (ids.long() + vocab * torch.arange(workers, device="cuda")[:, None])[there]
    values = dy[there.view(-1)].double()
    want.index_add_(0, at, values)
    size.index_add_(0, at, values.abs())
    count = torch.bincount(at, minlength=workers * vocab).double()[:, None]
    got = g[:, :vocab * width].reshape(workers * vocab, width)
    # a sum of `count` terms in any order, the scale's product
    within(got, want * scale, scale * (count + 2) * U * size, "dtable")
    assert bool(g[:, vocab * width:].isnan().all())
    # the same bits again; added to: only rows with tokens change
    again = torch.full_like(g, math.nan)
    op.backward(tokens, ids, dy, dy.stride(0), again, g_stride)
    assert torch.equal(again[:, :vocab * width], g[:, :vocab * width])
    base = torch.randn((workers, g_stride), generator=gen(8), device="cuda")
    base[:, 0] = math.nan
    added = base.clone()
    op.backward(tokens, ids, dy, dy.stride(0), added, g_stride, accumulate=True)
    rows = lambda t: t[:, :vocab * width].reshape(workers * vocab, width)  # noqa: E731
    expected = torch.where(count > 0, rows(base) + rows(g), rows(base))
    assert torch.equal(rows(added).nan_to_num(5.0), expected.nan_to_num(5.0))
    assert torch.equal(added[:, vocab * width:], base[:, vocab * width:])
    # fewer tokens than the operator was made for, down to none
    for less in {0, 1, tokens // 2}:
        part = torch.full_like(g, math.nan)
        op.backward(less, ids.view(-1)[:workers * less].contiguous(), dy, dy.stride(0), part, g_stride)
        sub = ids.view(-1)[:workers * less].view(workers, less).long()
        ok = (sub >= 0) & (sub < vocab)
        want = torch.zeros((workers * vocab, width), dtype=torch.float64, device="cuda")
        size = torch.zeros_like(want)
        at = (sub + vocab * torch.arange(workers, device="cuda")[:, None])[ok]
        if at.numel():
            values = dy[:workers * less][ok.view(-1)].double()  # some rows are NaN at these places
            want.index_add_(0, at, values)
            size.index_add_(0, at, values.abs())
        within(rows(part), want * scale, scale * (less + 2) * U * size, f"dtable of {less}")
    op.destroy()


def test_embedding_offsets_past_32_bits(P):
    """A table of more than 2^31 values, a gradient row beyond 2^31 floats, rows of dy beyond 2^31 elements."""
    vocab, width = 70_000, 32_768
    table = torch.empty(vocab * width, dtype=torch.float16, device="cuda")
    ids = torch.tensor([[69_999, 0, 65_537, 69_999, 1]], dtype=torch.int32, device="cuda")
    values = torch.randn((5, width), generator=gen(9), device="cuda").half()
    rows = table.view(vocab, width)
    for i in (1, 2, 3, 4):
        rows[int(ids[0, i])] = values[i]
    op = P.Embedding(vocab=vocab, width=width, max_tokens=5, table_dtype=2, dtype=2, cuda_stream=stream())
    ld = 600_000_000
    y = torch.zeros(4 * ld + width, dtype=torch.float16, device="cuda")
    op.forward(5, ids, table, 0, y, ld)
    view = torch.as_strided(y, (5, width), (ld, 1))
    assert torch.equal(view, rows[ids[0].long()])
    del table
    g = torch.full((vocab * width,), math.nan, device="cuda")
    op.backward(5, ids, y, ld, g, vocab * width)
    g = g.view(vocab, width)
    assert torch.equal(g[69_999], view[0].float() + view[3].float())
    for i in (1, 2, 4):
        assert torch.equal(g[int(ids[0, i])], view[i].float())
    assert int((g != 0).any(1).sum()) == 4
    op.destroy()


@pytest.mark.parametrize("in_shift,out_shift,width,dtype", [(0, 0, 64, 1), (3, 0, 64, 1), (0, 1, 64, 1), (5, 2, 64, 2),
                                                            (0, 0, 41, 0), (1, 3, 41, 0), (7, 1, 300, 1), (0, 1, 1032, 0),
                                                            (1, 0, 1032, 1), (2, 2, 7, 1)])
def test_embedding_backward_alignments(P, in_shift, out_shift, width, dtype):
    """Rows of dy and of the table's gradient that start anywhere, with unused values between them."""
    tokens, vocab, pad = 700, 60, 5
    ids = tokens_of(1, tokens, vocab, 32, "zipf", width)
    dy, _ = rows_of(torch.randn((tokens, width), generator=gen(21), device="cuda"), pad, DTYPES[dtype], in_shift)
    op = P.Embedding(vocab=vocab, width=width, max_tokens=tokens, dtype=dtype, scale=0.5, cuda_stream=stream())
    flat = torch.full((out_shift + vocab * width + 3,), math.nan, device="cuda")
    g = flat[out_shift:out_shift + vocab * width]
    op.backward(tokens, ids, dy, dy.stride(0), g, 0)
    there = (ids[0] >= 0) & (ids[0] < vocab)
    at, values = ids[0].long()[there], dy[there].double()
    want, size = torch.zeros((2, vocab, width), dtype=torch.float64, device="cuda")
    want.index_add_(0, at, values)
    size.index_add_(0, at, values.abs())
    count = torch.bincount(at, minlength=vocab).double()[:, None]
    within(g.view(vocab, width), want * 0.5, 0.5 * (count + 2) * U * size, "dtable")
    assert flat[:out_shift].isnan().all() and flat[out_shift + vocab * width:].isnan().all()
    base = torch.randn(vocab * width, generator=gen(22), device="cuda")
    added = torch.full_like(flat, math.nan)
    added[out_shift:out_shift + vocab * width] = base
    op.backward(tokens, ids, dy, dy.stride(0), added[out_shift:], 0, accumulate=True)
    assert torch.equal(added[out_shift:out_shift + vocab * width], base + g)
    op.destroy()


def test_embedding_backward_of_more_places_than_are_sorted_at_once(P):
    """Written and added to, each over several sections; no places at all in a worker's later ones."""
    workers, tokens, vocab, width = 2, 400_001, 5003, 12
    ids = tokens_of(workers, tokens, vocab, 64, "zipf", 31)
    ids[1, 170_000:] = -1
    dy = torch.randn((workers * tokens, width), generator=gen(32), device="cuda")
    op = P.Embedding(vocab=vocab, width=width, max_tokens=tokens, workers=workers, token_bits=64, cuda_stream=stream())
    g = torch.full((workers, vocab * width), math.nan, device="cuda")
    op.backward(tokens, ids, dy, width, g, vocab * width)
    there = (ids >= 0) & (ids < vocab)
    at, values = (ids + vocab * torch.arange(workers, device="cuda")[:, None])[there], dy[there.view(-1)].double()
    want, size = torch.zeros((2, workers * vocab, width), dtype=torch.float64, device="cuda")
    want.index_add_(0, at, values)
    size.index_add_(0, at, values.abs())
    count = torch.bincount(at, minlength=workers * vocab).double()[:, None]
    within(g.view(workers * vocab, width), want, (count + 2) * U * size, "dtable")
    added = torch.ones_like(g)
    op.backward(tokens, ids, dy, width, added, vocab * width, accumulate=True)
    within(added.view(workers * vocab, width), want + 1, (count + 8) * U * (size + 1), "dtable added to")
    assert torch.equal(added.view(-1, width)[count[:, 0] == 0], torch.ones_like(added).view(-1, width)[count[:, 0] == 0])
    op.destroy()


# ---------------------------------------------------------------------------
# distillation
# ---------------------------------------------------------------------------

DISTILL = [  # rows, vocab, k, dtype, teacher, temperature, pad, given
    (1, 1, 1, 0, 0, 1.0, 0, False),
    (3, 2, 4, 1, 1, 2.0, 1, False),
    (5, 33, 7, 2, 2, 0.7, 0, True),
    (4, 1000, 8, 1, 0, 1.0, 0, False),
    (7, 1001, 1, 0, 1, 1.0, 3, False),
    (200, 4096, 16, 1, 0, 2.0, 8, False),
    (33, 8200, 64, 2, 0, 1.5, 0, False),
    (1023, 5001, 33, 0, 0, 1.0, 3, True),
    (2, 32_000, 256, 1, 0, 1.0, 0, False),
    (9, 50_001, 100, 0, 2, 3.0, 0, False),
    (1, 131_072, 128, 1, 1, 2.0, 0, False),
    (40, 128_000, 128, 1, 0, 1.0, 0, True),
    (3, 128_001, 50, 1, 0, 1.0, 7, False),
    (3, 300_001, 50, 0, 0, 1.0, 0, False),
    (2, 1_000_003, 1024, 1, 0, 2.0, 5, False),
    (400, 700, 1024, 0, 0, 1.0, 0, False),
    (160, 65_536, 20, 2, 0, 1.0, 0, False),
]


def distill_data(rows, vocab, k, dtype, teacher, temperature, pad, given):
    """Ids with repetitions and outside the vocabulary, NaN in entries left out, rows of weight 0 full of NaN,
    rows without entries, logits of -inf."""
    g = gen(rows * 7 + vocab)
    z = 3 * torch.randn((rows, vocab), generator=g, device="cuda")
    ids = torch.randint(-(vocab // 8) - 1, vocab + vocab // 8 + 1, (rows, k), generator=g, device="cuda")
    values = 4 + 3 * torch.randn((rows, k), generator=g, device="cuda")
    if k > 2:
        ids[::3, 2] = ids[::3, 0]  # an id twice
        values[::5, 1] = -math.inf
    outside = (ids < 0) | (ids >= vocab)
    values[outside] = math.nan
    weights = 0.5 + torch.rand(rows, generator=g, device="cuda")
    if vocab > 8:
        no = torch.arange(0, vocab, 5, device="cuda")
        z[:, no] = torch.where(torch.rand((rows, len(no)), generator=g, device="cuda") < 0.5, -math.inf, z[:, no])
        z.scatter_(1, ids.clamp(0, vocab - 1), 2.0 + torch.zeros_like(values))
        z[:, 3] = 1.5
    if rows > 2:
        weights[1] = 0
        z[1] = math.nan
        ids[2] = -1
        z[2, 0] = math.nan
    z, flat = rows_of(z, pad, DTYPES[dtype])
    lse = (6 + torch.randn(rows, generator=g, device="cuda")) if given else None
    return z, ids.int(), values.to(DTYPES[teacher]), lse, weights


@pytest.mark.parametrize("case", DISTILL, ids=str)
def test_distillation(P, case):
    rows, vocab, k, dtype, teacher, temperature, pad, given = case
    T = DTYPES[dtype]
    z, ids, values, lse_t, weights = distill_data(*case)
    scale = 0.37
    op = P.Distillation(vocab=vocab, k=k, dtype=dtype, teacher_dtype=teacher, temperature=temperature,
                        cuda_stream=stream())
    args = (ids, values, k, lse_t, weights)
    loss, lse = torch.full((2, rows), math.nan, device="cuda")
    op.forward(rows, z, z.stride(0), *args, loss, lse)
    ref = distillation(z.double(), ids, values.double(), None if lse_t is None else lse_t.double(), weights.double(),
                       float(np.float32(temperature)), float(np.float32(scale)))
    within(loss, ref[0], ref[3] + 4 * U * ref[0].abs(), "loss")
    within(lse, ref[1], ref[4], "lse")
    # the gradient from the forward pass's lse
    dz, flat = rows_of(torch.full((rows, vocab), math.nan), pad, T)
    op.backward(rows, z, z.stride(0), lse, *args, scale, dz, dz.stride(0))
    want = distillation(z.double(), ids, values.double(), None if lse_t is None else lse_t.double(), weights.double(),
                        float(np.float32(temperature)), float(np.float32(scale)), lse=lse.double())
    within(dz, want[2], want[5] + rounded(want[2].abs() + want[5], T), "dlogits")
    assert untouched(flat, rows, vocab, pad)
    # both at once
    loss2, lse2 = torch.full((2, rows), math.nan, device="cuda")
    dz2, flat = rows_of(torch.full((rows, vocab), math.nan), pad, T)
    op.step(rows, z, z.stride(0), *args, scale, loss2, lse2, dz2, dz2.stride(0))
    within(loss2, ref[0], ref[3] + 4 * U * ref[0].abs(), "loss of the step")
    within(lse2, ref[1], ref[4], "lse of the step")
    within(dz2, ref[2], ref[5] + rounded(ref[2].abs() + ref[5], T), "dlogits of the step")
    assert untouched(flat, rows, vocab, pad)
    # in place, without lse: the same bits
    z2 = rows_of(z, pad, T)[0]
    loss3 = torch.full((rows,), math.nan, device="cuda")
    op.step(rows, z2, z2.stride(0), *args, scale, loss3, None, z2, z2.stride(0))
    assert torch.equal(z2.contiguous().view(torch.uint8), dz2.contiguous().view(torch.uint8))
    assert torch.equal(loss3, loss2)
    op.backward(rows, z, z.stride(0), lse, *args, scale, z, z.stride(0))
    assert torch.equal(z.contiguous().view(torch.uint8), dz.contiguous().view(torch.uint8))
    op.destroy()


@pytest.mark.parametrize("rows,vocab,k,dtype", [(6, 1003, 40, 1), (3, 40_001, 65, 0), (700, 333, 5, 2), (5, 129, 200, 1)])
def test_distillation_ids_in_steps_and_other_alignments(P, rows, vocab, k, dtype):
    """Ids a fixed step apart, all the same id, and a gradient whose rows are aligned differently from the logits'."""
    T = DTYPES[dtype]
    z = torch.randn((rows, vocab), generator=gen(41), device="cuda")
    steps = torch.tensor([1, 2, 3, 0, 16, 128, 64], device="cuda")[torch.arange(rows, device="cuda") % 7]
    ids = (5 + steps[:, None] * torch.arange(k, device="cuda")) % vocab
    values = torch.randn((rows, k), generator=gen(42), device="cuda")
    z, _ = rows_of(z, 1, T, 1)
    dz, flat = rows_of(torch.full((rows, vocab), math.nan), 4, T, 2)
    loss, lse = torch.full((2, rows), math.nan, device="cuda")
    op = P.Distillation(vocab=vocab, k=k, dtype=dtype, cuda_stream=stream())
    op.step(rows, z, z.stride(0), ids.int(), values, k, None, None, 1.0, loss, lse, dz, dz.stride(0))
    ref = distillation(z.double(), ids, values.double(), None, torch.ones(rows, device="cuda").double(), 1.0, 1.0)
    within(loss, ref[0], ref[3] + 4 * U * ref[0].abs(), "loss")
    within(dz, ref[2], ref[5] + rounded(ref[2].abs() + ref[5], T), "dlogits")
    assert untouched(flat, rows, vocab, 4, 2)
    op.destroy()


def test_distillation_extreme_logits(P):
    """The type's lowest value as a mask, large logits, an entry at a logit of -inf, a row of -inf, +inf and NaN."""
    rows, vocab = 8, 4099
    z = torch.randn((rows, vocab), generator=gen(11), device="cuda")
    z[0, 100:] = torch.finfo(torch.float32).min
    z[1] = 1e30 * z[1].sign()
    z[2, 7] = -math.inf
    z[3] = -math.inf
    z[4, 9] = math.nan
    z[5] = torch.finfo(torch.float32).min
    z[6] = -8e4 + z[6]
    ids = torch.tensor([[7, 11]] * rows, dtype=torch.int32, device="cuda")
    values = torch.tensor([[1.0, 0.0]] * rows, device="cuda")
    op = P.Distillation(vocab=vocab, k=2, cuda_stream=stream())
    loss, lse = torch.zeros((2, rows), device="cuda")
    dz = torch.full_like(z, 5.0)
    op.step(rows, z, vocab, ids, values, 2, None, None, 1.0, loss, lse, dz, vocab)
    ref = distillation(z.double(), ids, values.double(), None, torch.ones(rows, device="cuda").double(), 1.0, 1.0)
    for r in (0, 6, 7):
        within(loss[r:r + 1], ref[0][r:r + 1], ref[3][r:r + 1] + 4 * U * ref[0][r:r + 1].abs(), "loss")
        within(dz[r:r + 1], ref[2][r:r + 1], ref[5][r:r + 1] + rounded(ref[2][r:r + 1], torch.float32), "dlogits")
    assert loss[2] == math.inf and dz[2].isfinite().all()
    within(dz[2:3], ref[2][2:3], ref[5][2:3] + rounded(ref[2][2:3], torch.float32), "dlogits")
    assert loss[3].isnan() and dz[3].isnan().all()
    assert loss[4].isnan() and dz[4].isnan().all()
    # equal lowest values: a uniform distribution
    assert torch.allclose(dz[5, 20:], torch.full((vocab - 20,), 1 / vocab, device="cuda"), rtol=1e-5, atol=0)
    assert dz[1].isfinite().all() and loss[1].isfinite() and loss[1] >= 0
    op.destroy()


def test_distillation_of_one_entry_is_cross_entropy(P):
    rows, vocab = 50, 777
    z = torch.randn((rows, vocab), generator=gen(12), device="cuda", requires_grad=True)
    labels = torch.randint(0, vocab, (rows,), generator=gen(13), device="cuda")
    labels[3] = -100
    want = torch.nn.functional.cross_entropy(z.double(), labels, reduction="sum")
    want.backward()
    op = P.Distillation(vocab=vocab, k=1, cuda_stream=stream())
    loss, lse = torch.empty((2, rows), device="cuda")
    dz = torch.empty((rows, vocab), device="cuda")
    zero = torch.zeros((rows, 1), device="cuda")
    op.step(rows, z.detach(), vocab, labels.int(), zero, 1, None, None, 1.0, loss, lse, dz, vocab)
    assert abs(float(loss.double().sum()) - float(want.detach())) <= 64 * U * float(want.detach())
    assert float((dz - z.grad).abs().max()) <= 64 * U
    op.destroy()


def test_distillation_gradient_is_the_differences(P):
    rows, vocab, k, T = 2, 13, 4, 1.5
    g = gen(14)
    z = torch.randn((rows, vocab), generator=g, device="cuda")
    ids = torch.tensor([[3, 7, 3, -1], [0, 12, 5, 6]], dtype=torch.int32, device="cuda")
    values = torch.randn((rows, k), generator=g, device="cuda")
    weights = torch.tensor([0.7, 1.3], device="cuda")
    op = P.Distillation(vocab=vocab, k=k, temperature=T, cuda_stream=stream())
    loss, lse = torch.empty((2, rows), device="cuda")
    dz = torch.empty_like(z)
    op.step(rows, z, vocab, ids, values, k, None, weights, 2.0, loss, lse, dz, vocab)
    at = z.double()
    step = 1e-5
    for i in range(rows):
        for j in range(vocab):
            up, down = at.clone(), at.clone()
            up[i, j] += step
            down[i, j] -= step
            d = [float(distillation(v, ids, values.double(), None, weights.double(), T, 2.0)[0].sum()) * 2.0 for v in (up, down)]
            assert abs((d[0] - d[1]) / (2 * step) - float(dz[i, j])) <= 64 * U * 4 + 1e-7
    op.destroy()


# ---------------------------------------------------------------------------
# refusals, streams, graphs, allocation
# ---------------------------------------------------------------------------


def refused(P, call, needle):
    with pytest.raises(P.DqganError) as ei:
        call()
    assert ei.value.status == P.dqgan.ERR_INVALID_ARG
    assert needle in str(ei.value), str(ei.value)


def test_refusals(P):
    x = torch.zeros(64, device="cuda")
    norm = P.LayerNorm(width=8, workers=2, cuda_stream=stream())
    refused(P, lambda: norm.forward(-1, x, 8, x, x, 8, x, 8), "rows")
    refused(P, lambda: norm.forward(1 << 40, x, 8, x, x, 8, x, 8), "rows")
    refused(P, lambda: norm.forward(1, None, 8, x, x, 8, x, 8), "NULL")
    refused(P, lambda: norm.forward(1, x, 7, x, x, 8, x, 8), "stride")
    refused(P, lambda: norm.forward(1, x, 8, x, x, 7, x, 8), "p_stride")
    refused(P, lambda: norm.forward(1, x, 8, x, x, 8, x, 8, x, None), "mean")
    refused(P, lambda: norm.forward(1, x.data_ptr() + 2, 8, x, x, 8, x, 8), "aligned")
    refused(P, lambda: norm.backward(1, x, 8, None, 8, x, 8, x, x, x, 8, x, x, 8), "NULL")
    refused(P, lambda: norm.backward(1, x, 8, x, 8, x, 8, x, x, x, 8, x, x, 7), "g_stride")
    refused(P, lambda: norm.backward(1, x, 8, x, 8, x, 8, x, x, x, 3, x, x, 8), "stride")
    norm.forward(0, None, 8, None, None, 0, None, 8)
    embed = P.Embedding(vocab=4, width=8, max_tokens=2, workers=2, cuda_stream=stream())
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    refused(P, lambda: embed.forward(3, ids, x, 32, x, 8), "tokens")
    refused(P, lambda: embed.forward(1, ids, x, 31, x, 8), "p_stride")
    refused(P, lambda: embed.forward(1, ids, None, 32, x, 8), "NULL")
    refused(P, lambda: embed.forward(1, ids, x, 32, x, 7), "stride")
    refused(P, lambda: embed.backward(1, ids, x, 8, x, 31), "g_stride")
    refused(P, lambda: embed.backward(1, ids, None, 8, x, 32), "NULL")
    refused(P, lambda: embed.backward(0, ids, None, 8, None, 32), "NULL")
    refused(P, lambda: embed.backward(1, ids.data_ptr() + 1, x, 8, x, 32), "aligned")
    distill = P.Distillation(vocab=8, k=2, cuda_stream=stream())
    refused(P, lambda: distill.forward(1, x, 7, ids, x, 2, None, None, x), "stride")
    refused(P, lambda: distill.forward(1, x, 8, ids, x, 1, None, None, x), "teacher_stride")
    refused(P, lambda: distill.forward(1, x, 8, ids, x, 2, None, None, None), "loss")
    refused(P, lambda: distill.backward(1, x, 8, None, ids, x, 2, None, None, 1.0, x, 8), "lse")
    refused(P, lambda: distill.step(1, x, 8, ids, x, 2, None, None, math.inf, x, x, x, 8), "scale")
    refused(P, lambda: distill.step(1, x, 8, ids, x, 2, None, None, 1.0, x, x, None, 8), "dlogits")
    distill.step(0, None, 8, None, None, 2, None, None, 1.0, None, None, None, 8)
    # another kind's operator
    L = P.dqgan.load_library()
    assert L.dqgan_layer_norm_forward(embed._h, 1, x.data_ptr(), 8, None, None, 0, x.data_ptr(), 8, None, None) == \
        P.dqgan.ERR_INVALID_ARG
    assert "layer norm" in embed.last_error()
    torch.cuda.synchronize()
    assert not x.any()


def test_allocation_failure(P, monkeypatch):
    monkeypatch.setenv("DQGAN_TEST_FAIL_ALLOC", "1")
    with pytest.raises(P.DqganError) as ei:
        P.Embedding(vocab=1000, width=8, max_tokens=100)
    assert ei.value.status == P.dqgan.ERR_OOM
    monkeypatch.delenv("DQGAN_TEST_FAIL_ALLOC")
    P.Embedding(vocab=1000, width=8, max_tokens=100).destroy()


def test_other_stream_and_graph(P):
    """On a stream of its own, captured once and replayed on new data."""
    s = torch.cuda.Stream()
    W, n, V, C, K = 2, 300, 500, 96, 5
    norm = P.LayerNorm(width=C, workers=W, dtype=1, cuda_stream=s.cuda_stream)
    embed = P.Embedding(vocab=V, width=C, max_tokens=n, workers=W, dtype=1, cuda_stream=s.cuda_stream)
    distill = P.Distillation(vocab=C, k=K, dtype=1, cuda_stream=s.cuda_stream)
    ids = torch.zeros((W, n), dtype=torch.int32, device="cuda")
    table = torch.randn((W, V * C), generator=gen(1), device="cuda")
    tid = torch.randint(0, C, (W * n, K), generator=gen(2), device="cuda").int()
    tv = torch.randn((W * n, K), generator=gen(3), device="cuda")
    x, y, dx = torch.zeros((3, W * n, C), dtype=torch.bfloat16, device="cuda")
    mean, rstd, loss = torch.zeros((3, W * n), device="cuda")
    g = torch.zeros((W, V * C + 2 * C), device="cuda")

    def step():
        embed.forward(n, ids, table, V * C, x, C)
        norm.forward(n, x, C, None, None, 0, y, C, mean, rstd)
        distill.step(W * n, y, C, tid, tv, K, None, None, 1.0, loss, None, y, C)
        norm.backward(n, y, C, x, C, None, 0, mean, rstd, dx, C, g[:, V * C:], g[:, V * C + C:], g.stride(0))
        embed.backward(n, ids, dx, C, g, g.stride(0))

    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        step()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            step()
        for seed in (5, 6):
            ids.copy_(tokens_of(W, n, V, 32, "zipf", seed))
            graph.replay()
            s.synchronize()
            replayed = [t.clone() for t in (x, mean, loss, dx, g)]
            step()
            s.synchronize()
            for a, b in zip(replayed, (x, mean, loss, dx, g)):
                assert torch.equal(a, b)
    assert norm.launch_count() > 0 and embed.launch_count() > 0 and distill.launch_count() > 0


@pytest.mark.parametrize("shape", [(2, 150, 1500, 1, 0, 0, False), (1, 77, 2999, 0, 1, 1, False), (3, 40, 6000, 1, 0, 0, True),
                                   (1, 30, 12000, 2, 0, 3, False), (1, 200, 5120, 1, 0, 0, False)], ids=str)
def test_layer_norm_between_powers_of_two(P, shape):
    test_layer_norm_forward(P, shape)
    test_layer_norm_backward(P, shape)


@pytest.mark.parametrize("width", [64, 1537, 20_000])
def test_layer_norm_gradient_of_no_rows(P, width):
    """Zeros, or what was there; the rows' pointers are not looked at."""
    op = P.LayerNorm(width=width, workers=3, cuda_stream=stream())
    g = torch.full((3, 2 * width), math.nan, device="cuda")
    op.backward(0, None, width, None, width, None, 0, None, None, None, width, g, g[:, width:], 2 * width)
    assert not g.any()
    g.fill_(2.5)
    op.backward(0, None, width, None, width, None, 0, None, None, None, width, g, g[:, width:], 2 * width, accumulate=True)
    assert (g == 2.5).all()
    op.destroy()


@pytest.mark.parametrize("rows", [1, 5, 400])
def test_distillation_of_rows_that_do_not_count(P, rows):
    """All weights 0, no entries, and every second row: zeros where nothing counts, the others as alone."""
    vocab, k = 9000, 12
    z = torch.randn((rows, vocab), generator=gen(51), device="cuda").bfloat16()
    ids = torch.randint(0, vocab, (rows, k), generator=gen(52), device="cuda").int()
    values = torch.randn((rows, k), generator=gen(53), device="cuda")
    op = P.Distillation(vocab=vocab, k=k, dtype=1, cuda_stream=stream())

    def step(ids, weights):
        loss, lse = torch.full((2, rows), math.nan, device="cuda")
        dz = torch.full_like(z, math.nan)
        op.step(rows, z, vocab, ids, values, k, None, weights, 1.0, loss, lse, dz, vocab)
        return loss, lse, dz

    for got in step(ids, torch.zeros(rows, device="cuda")) + step(torch.full_like(ids, -1), None):
        assert not got.any()
    weights = torch.ones(rows, device="cuda")
    weights[::2] = 0
    for part, whole in zip(step(ids, weights), step(ids, None)):
        assert not part[::2].any() and torch.equal(part[1::2], whole[1::2])
    op.destroy()
