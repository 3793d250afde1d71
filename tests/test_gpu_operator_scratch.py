"""What operators hold: not more than the calls of their sizes can use."""
from __future__ import annotations

import pytest

from test_gpu_products import P, stream  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def held(make):
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    op = make()
    taken = free - torch.cuda.mem_get_info()[0]
    op.destroy()
    return taken


@pytest.mark.parametrize("shape", [
    (64, 1 << 24, 8, 8),  # the largest vocabulary: few rows of it always take tiles
    (64, 1 << 24, 1, 4),  # a width that is rounded up to eight
    (8, 1 << 21, 64, 8),  # four rows a worker go without tiles
], ids=str)
def test_token_loss_of_a_large_vocabulary(P, shape):  # noqa: F811
    workers, vocab, width, rows = shape
    taken = held(lambda: P.TokenLoss(vocab=vocab, width=width, max_rows=rows, workers=workers, cuda_stream=stream()))
    few = min(rows, (80 << 20) // (vocab // 256 * workers * width * 4)) if vocab <= 65535 * 64 else 0
    # a gigabyte each of the weights' and the gradient's parts, 80 MB, the sums, and x and dx in fp32 and in parts
    sums = workers * rows * 2 * (vocab // 256) * 8
    assert taken <= (2 << 30) + (80 << 20) + sums + workers * (rows * (4 * width + 48) + few * vocab * 4) + (64 << 20)


def test_linear_of_large_sizes_and_many_workers(P):  # noqa: F811
    workers, inputs, outputs, rows = 512, 128, 65536, 8
    taken = held(lambda: P.Linear(inputs=inputs, outputs=outputs, max_rows=rows, workers=workers, dtype=P.BF16,
                                  weight_dtype=P.BF16, cuda_stream=stream()))
    # eight rows' sums of d W would not fit 80 MB; du in parts, x, the weights, the bias's blocks of sums
    few = 80 * 2 ** 20 // (256 * workers * inputs * 4)
    assert few == 1
    parts = workers * (rows * outputs * 2 + rows * inputs * 2 + outputs * inputs * 2)
    assert taken <= parts + workers * outputs * 4 * (few + 1) + (80 << 20) + (64 << 20)


@pytest.mark.parametrize("rows", [3, 4])
def test_rows_at_the_limit_of_what_goes_without_tiles(P, rows):  # noqa: F811
    """Six runs of 256 weights, 512 workers and 2048 inputs: sums of three rows fit 80 MB, of four not."""
    workers, inputs, outputs = 512, 2048, 1300
    dy = torch.ones((workers * rows, outputs), device="cuda")
    w = torch.full((outputs * inputs,), 0.5, device="cuda")
    op = P.Linear(inputs=inputs, outputs=outputs, max_rows=8, workers=workers, cuda_stream=stream())
    dx = torch.zeros((workers * rows, inputs), device="cuda")
    op.backward(rows, dy, outputs, None, inputs, w, 0, None, 0, dx, inputs, None, None, 0)
    assert bool((dx == outputs / 2).all())
    op.destroy()
