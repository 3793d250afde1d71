"""The token-model operators with more rows than the GPU holds at once, so that clusters, rings of rows on
their way and kept weights go through several turns; and from two host threads at once.  Row counts follow the
number of SMs.  Bounds as in test_gpu_operators."""
from __future__ import annotations

import math
import threading

import numpy as np
import pytest

from operator_references import U, distillation, rounded, within
from test_gpu_operators import DTYPES, P, distill_data, gen, rows_of, stream, untouched  # noqa: F401
from test_gpu_operators import test_layer_norm_backward as norm_backward_case
from test_gpu_operators import test_layer_norm_forward as norm_forward_case

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


# rows an SM, vocab, k, dtype, teacher, temperature, pad, given
TURNS = [
    (4, 65_536, 40, 1, 0, 1.0, 0, False),      # clusters of several blocks, rows aligned
    (2, 128_001, 33, 1, 1, 2.0, 0, False),     # rows start anywhere
    (3, 50_001, 140, 0, 2, 1.5, 1, True),
    (8, 20_011, 9, 2, 0, 1.0, 2, False),       # one block a row
    (60, 2300, 100, 1, 0, 1.0, 1, False),
    (1280, 40, 3, 0, 0, 1.0, 0, False),        # more than 32 turns of up to 32 blocks an SM
]


@pytest.mark.parametrize("case", TURNS, ids=str)
def test_distillation_in_several_turns(P, case):  # noqa: F811
    rows, vocab, k, dtype, teacher, temperature, pad, given = (case[0] * sms() + 3,) + case[1:]
    T = DTYPES[dtype]
    z, ids, values, lse_t, weights = distill_data(rows, vocab, k, dtype, teacher, temperature, pad, given)
    # rows that do not count, alone and in long runs: a cluster passes over some and begins and ends with others
    no = torch.rand(rows, generator=gen(61), device="cuda") < 0.2
    no[:7] = no[-5:] = True
    no[rows // 2:rows // 2 + rows // 8] = True
    weights[no] = 0
    ids[torch.rand(rows, generator=gen(62), device="cuda") < 0.1] = -1
    scale, T32, s32 = 0.37, float(np.float32(temperature)), float(np.float32(0.37))
    op = P.Distillation(vocab=vocab, k=k, dtype=dtype, teacher_dtype=teacher, temperature=temperature,
                        cuda_stream=stream())
    args = (ids, values, k, lse_t, weights)
    loss, lse = torch.full((2, rows), math.nan, device="cuda")
    op.forward(rows, z, z.stride(0), *args, loss, lse)
    given64 = None if lse_t is None else lse_t.double()
    ref = distillation(z.double(), ids, values.double(), given64, weights.double(), T32, s32)
    within(loss, ref[0], ref[3] + 4 * U * ref[0].abs(), "loss")
    within(lse, ref[1], ref[4], "lse")
    loss2, lse2 = torch.full((2, rows), math.nan, device="cuda")
    dz, flat = rows_of(torch.full((rows, vocab), math.nan), pad, T)
    op.step(rows, z, z.stride(0), *args, scale, loss2, lse2, dz, dz.stride(0))
    within(loss2, ref[0], ref[3] + 4 * U * ref[0].abs(), "loss of the step")
    within(lse2, ref[1], ref[4], "lse of the step")
    within(dz, ref[2], ref[5] + rounded(ref[2].abs() + ref[5], T), "dlogits of the step")
    assert untouched(flat, rows, vocab, pad)
    del ref
    back, flat = rows_of(torch.full((rows, vocab), math.nan), pad, T)
    op.backward(rows, z, z.stride(0), lse, *args, scale, back, back.stride(0))
    want = distillation(z.double(), ids, values.double(), given64, weights.double(), T32, s32, lse=lse.double())
    within(back, want[2], want[5] + rounded(want[2].abs() + want[5], T), "dlogits")
    assert untouched(flat, rows, vocab, pad)
    # in place, and again: the same bits
    for _ in range(3):
        place = rows_of(z, pad, T)[0]
        loss3 = torch.full((rows,), math.nan, device="cuda")
        op.step(rows, place, place.stride(0), *args, scale, loss3, None, place, place.stride(0))
        assert torch.equal(place.contiguous().view(torch.uint8), dz.contiguous().view(torch.uint8))
        assert torch.equal(loss3, loss2)
        place = rows_of(z, pad, T)[0]
        op.backward(rows, place, place.stride(0), lse, *args, scale, place, place.stride(0))
        assert torch.equal(place.contiguous().view(torch.uint8), back.contiguous().view(torch.uint8))
    op.destroy()


# workers, rows an SM, width, dtype, pad, shift, shared: rows that do not start on 16-byte boundaries, and narrow ones
NORM_TURNS = [
    (1, 40, 1537, 0, 0, 0, False),
    (1, 14, 5001, 1, 0, 1, False),
    (3, 210, 31, 0, 0, 0, False),
    (1, 700, 30, 2, 2, 0, False),
    (1, 5, 12_289, 1, 0, 0, False),
    (2, 3, 8201, 0, 0, 1, True),
    (1, 24, 3001, 2, 0, 3, False),
    (1, 300, 256, 1, 0, 0, False),
]


@pytest.mark.parametrize("shape", NORM_TURNS, ids=str)
def test_layer_norm_in_several_turns(P, shape):  # noqa: F811
    shape = (shape[0], shape[1] * sms() + 5) + shape[2:]
    norm_forward_case(P, shape)
    norm_backward_case(P, shape)


def test_two_host_threads(P):  # noqa: F811
    """One kind of operator with different sizes from two threads on two streams: the bits of each alone."""
    sizes = [(37, 9001, 11), (400, 700, 80)]
    torch.cuda.synchronize()

    def make(rows, vocab, k):
        g = gen(rows)
        z = torch.randn((rows, vocab), generator=g, device="cuda").bfloat16()
        ids = torch.randint(0, vocab, (rows, k), generator=g, device="cuda").int()
        values = torch.randn((rows, k), generator=g, device="cuda")
        x = torch.randn((rows, vocab), generator=g, device="cuda")
        tokens = torch.randint(0, 50, (rows,), generator=g, device="cuda").int()
        s = torch.cuda.Stream()
        at = s.cuda_stream
        ops = (P.Distillation(vocab=vocab, k=k, dtype=1, cuda_stream=at), P.LayerNorm(width=vocab, cuda_stream=at),
               P.Embedding(vocab=50, width=vocab, max_tokens=rows, cuda_stream=at))
        return s, ops, (z, ids, values, x, tokens)

    def run(s, ops, data, out, times):
        z, ids, values, x, tokens = data
        rows, vocab = z.shape
        loss, dz, y, g, mean, rstd, dw = out
        for _ in range(times):
            ops[0].step(rows, z, vocab, ids, values, ids.stride(0), None, None, 1.0, loss, None, dz, vocab)
            ops[1].forward(rows, x, vocab, None, None, 0, y, vocab, mean, rstd)
            ops[1].backward(rows, x, vocab, x, vocab, None, 0, mean, rstd, y, vocab, dw, None, 0)
            ops[2].backward(rows, tokens, y, vocab, g, 0)
        s.synchronize()

    def buffers(rows, vocab):
        new = lambda *shape: torch.full(shape, math.nan, device="cuda")  # noqa: E731
        return (new(rows), new(rows, vocab).bfloat16(), new(rows, vocab), new(50 * vocab), new(rows), new(rows), new(vocab))

    made = [make(*size) for size in sizes]
    alone = [buffers(*size[:2]) for size in sizes]
    both = [buffers(*size[:2]) for size in sizes]
    torch.cuda.synchronize()
    for m, out in zip(made, alone):
        run(*m, out, 1)
    failures = []

    def body(m, out):
        try:
            torch.cuda.set_device(0)
            run(*m, out, 50)
        except Exception as error:  # reported by the test's own thread
            failures.append(error)

    threads = [threading.Thread(target=body, args=(m, out)) for m, out in zip(made, both)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failures, failures
    for a, b in zip(alone, both):
        for x, y in zip(a, b):
            assert torch.equal(x, y)
