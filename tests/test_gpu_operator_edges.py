"""The token-model operators at the ends of their types' ranges, against the definitions in 64 bits."""
from __future__ import annotations

import math

import numpy as np
import pytest

from operator_references import U, distillation, rounded, within
from test_gpu_operators import DTYPES, P, gen, rows_of, stream  # noqa: F401
from test_gpu_operators import test_layer_norm_backward as norm_backward_case
from test_gpu_operators import test_layer_norm_forward as norm_forward_case

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("vocab", [300, 40_000, 1_000_003])  # one block a row, a cluster, rows that do not fit on chip
@pytest.mark.parametrize("teacher", [0, 1])
@pytest.mark.parametrize("temperature", [0.5, 1.0, 2.0])
def test_distillation_of_extreme_teacher_values(P, vocab, teacher, temperature):  # noqa: F811
    """The type's lowest value is a number: entries of nothing else share the mass, whatever t / T overflows to.  The
    probabilities depend on differences, so the definition is evaluated at values moved to where they can be written."""
    least = torch.finfo(DTYPES[teacher]).min
    rows = [  # values as given, and with the same differences where those count
        ([least] * 4, [0.0] * 4),
        ([-least] * 4, [0.0] * 4),
        ([least, -least, 0.0, least], [-1e4, 0.0, -1e4, -1e4]),
        ([0.5 * -least, 0.5 * -least, least, -math.inf], [0.0, 0.0, -1e4, -math.inf]),
        ([least, 0.5, 0.25, -math.inf], [-1e4, 0.5, 0.25, -math.inf]),
        ([least, -math.inf, -math.inf, -math.inf], [0.0, -math.inf, -math.inf, -math.inf]),
        ([0.5, 1.0, -2.0, 3.0], [0.5, 1.0, -2.0, 3.0]),
    ]
    R, T32 = len(rows), float(np.float32(temperature))
    values = torch.tensor([r[0] for r in rows], device="cuda").to(DTYPES[teacher])
    moved = torch.tensor([r[1] for r in rows], device="cuda", dtype=torch.float64)
    ids = torch.tensor([[7, 250, 11, 0]] * R, dtype=torch.int32, device="cuda")
    z = torch.randn((R, vocab), generator=gen(vocab), device="cuda")
    op = P.Distillation(vocab=vocab, k=4, teacher_dtype=teacher, temperature=temperature, cuda_stream=stream())
    loss, lse, loss2, lse2 = torch.full((4, R), math.nan, device="cuda")
    dz, back = torch.full((2, R, vocab), math.nan, device="cuda")
    op.forward(R, z, vocab, ids, values, 4, None, None, loss, lse)
    op.step(R, z, vocab, ids, values, 4, None, None, 1.0, loss2, lse2, dz, vocab)
    op.backward(R, z, vocab, lse, ids, values, 4, None, None, 1.0, back, vocab)
    ones = torch.ones(R, dtype=torch.float64, device="cuda")
    ref = distillation(z.double(), ids, moved, None, ones, T32, 1.0)
    for got in (loss, loss2):
        within(got, ref[0], ref[3] + 4 * U * ref[0].abs(), "loss")
    for got in (lse, lse2):
        within(got, ref[1], ref[4], "lse")
    within(dz, ref[2], ref[5] + rounded(ref[2].abs() + ref[5], torch.float32), "dlogits of the step")
    want = distillation(z.double(), ids, moved, None, ones, T32, 1.0, lse=lse.double())
    within(back, want[2], want[5] + rounded(want[2].abs() + want[5], torch.float32), "dlogits")
    op.destroy()


@pytest.mark.parametrize("width,pad,shift,dtype", [(1, 0, 1, 1), (1, 2, 7, 2), (2, 0, 3, 0), (3, 0, 5, 1), (3, 1, 1, 0), (5, 0, 6, 2),
                                                   (7, 1, 0, 1), (9, 7, 0, 1), (6, 2, 0, 0), (21, 0, 3, 1)])
@pytest.mark.parametrize("workers,tokens", [(1, 1), (2, 3), (3, 40)])
def test_narrow_rows_at_both_ends_of_a_tensor(P, width, pad, shift, dtype, workers, tokens):  # noqa: F811
    """Rows whose first or last pack of 16 bytes reaches beyond the tensor, into memory that holds NaN."""
    n, vocab = workers * tokens, 4
    dy, _ = rows_of(torch.randn((n, width), generator=gen(width), device="cuda"), pad, DTYPES[dtype], shift)
    ids = torch.randint(0, vocab, (workers, tokens), generator=gen(tokens), device="cuda").int()
    op = P.Embedding(vocab=vocab, width=width, max_tokens=tokens, workers=workers, dtype=dtype, cuda_stream=stream())
    g = torch.full((workers, vocab * width), math.nan, device="cuda")
    op.backward(tokens, ids, dy, dy.stride(0), g, vocab * width)
    want, size = torch.zeros((2, workers * vocab, width), dtype=torch.float64, device="cuda")
    at = (ids.long() + vocab * torch.arange(workers, device="cuda")[:, None]).view(-1)
    want.index_add_(0, at, dy.double())
    size.index_add_(0, at, dy.double().abs())
    count = torch.bincount(at, minlength=workers * vocab).double()[:, None]
    within(g.view(workers * vocab, width), want, (count + 2) * U * size, "dtable")
    op.destroy()
    shape = (workers, tokens, width, dtype, pad, shift, False)
    norm_forward_case(P, shape)
    norm_backward_case(P, shape)


@pytest.mark.parametrize("vocab,k", [(500, 300), (32_000, 1024), (130_000, 200)])
def test_distillation_of_ids_that_come_again(P, vocab, k):  # noqa: F811
    """One id twice, pairs, ids of many entries, all the same: summed over their entries, and one of them does not make
    every other entry of the row dear (it did 20-fold; a few looks at k ids each cost a small part of the row)."""
    rows = 1024
    z = torch.randn((rows, vocab), generator=gen(k), device="cuda").bfloat16()
    step = vocab // k
    unique = (torch.randint(0, vocab, (rows, 1), generator=gen(vocab), device="cuda") + step * torch.arange(k, device="cuda")) % vocab
    one = unique.clone()
    one[:, k - 1] = one[:, 0]
    many = one.clone()
    many[0::4, 1::2] = many[0::4, 0::2]
    many[1::4] = many[1::4, k // 2:k // 2 + 1]
    many[2::4] = many[2::4, torch.arange(k, device="cuda") % 7]
    many[3::8, 5] = -1
    values = torch.randn((rows, k), generator=gen(63), device="cuda")
    op = P.Distillation(vocab=vocab, k=k, dtype=1, temperature=1.5, cuda_stream=stream())
    loss, lse = torch.full((2, rows), math.nan, device="cuda")
    dz = torch.full_like(z, math.nan)

    def call(ids):
        op.step(rows, z, vocab, ids, values, k, None, None, 1.0, loss, lse, dz, vocab)

    ones = torch.ones(rows, dtype=torch.float64, device="cuda")
    for ids in (one, many):
        call(ids.int())
        first = dz.clone()
        for at in range(0, rows, 256):
            part = slice(at, at + 256)
            ref = distillation(z[part].double(), ids[part], values[part].double(), None, ones[part], 1.5, 1.0)
            within(loss[part], ref[0], ref[3] + 4 * U * ref[0].abs(), "loss")
            within(dz[part], ref[2], ref[5] + rounded(ref[2].abs() + ref[5], torch.bfloat16), "dlogits")
        call(ids.int())
        assert torch.equal(first.view(torch.int16), dz.view(torch.int16))

    def time_of(ids):
        times = []
        for _ in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            torch.cuda.synchronize()
            a.record()
            for _ in range(4):
                call(ids)
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b))
        return min(times)

    if k > 1000:
        assert time_of(one.int()) < 4 * time_of(unique.int())
    op.destroy()
