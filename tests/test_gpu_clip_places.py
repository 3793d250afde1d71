"""Clipping refuses lists in which an address comes twice, where two entries would write one place or one would read what
another writes."""
from __future__ import annotations

import math

import pytest

from operator_references import U, within
from test_gpu_products import P, gen, stream  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("count", [2, 3, 400, 4096])
def test_an_address_that_comes_twice_is_refused(P, count):  # noqa: F811
    workers, n = 2, 8
    stride = (count + 1) * n
    a, b = torch.ones((2, workers, stride), device="cuda")
    op = P.GradientClip(workers=workers, cuda_stream=stream())

    def entry(t, i):
        return t[:, i * n:], n, stride

    good = [entry(a, i) for i in range(count)]
    places = [entry(b, i) for i in reversed(range(count))]  # any order
    twice, across = good[:-1] + good[:1], good[:-2] + [entry(a, count), good[-2]]
    for tensors, to, needle in ((twice, twice, "the same address"), (good, places[:-1] + places[:1], "the same address"),
                                (good, across, "the address of tensor"), (places, places[1:] + [entry(b, count)], "the address of tensor")):
        with pytest.raises(P.DqganError) as ei:
            op.clip(P.TensorList(tensors), P.TensorList(to), 0.5)
        assert ei.value.status == P.dqgan.ERR_INVALID_ARG and needle in str(ei.value), str(ei.value)
    assert op.launch_count() == 0 and bool((a == 1).all()) and bool((b == 1).all())
    # tensors of no values have no place; one tensor may go to two places, and counts twice
    empty = [(None, 0, 0), (a, 0, 0), (a, 0, 0)]
    norms = torch.zeros(workers, device="cuda")
    op.clip(P.TensorList(good[:1] * 2 + empty), P.TensorList(places[:2] + empty), 1.0, norms)
    within(norms, torch.full((workers,), 4.0, dtype=torch.float64, device="cuda"), 8 * U, "norms")
    op.clip(P.TensorList(good), P.TensorList(places), 1e9)
    op.clip(P.TensorList(good), P.TensorList(good), 0.0)
    assert not a[:, :count * n].any() and bool((b[:, :count * n] == 1).all())
    op.destroy()


def test_a_norm_beyond_fp32_clips(P):  # noqa: F811
    """Finite values whose norm is not: clipped; a value that is not finite: passed on."""
    n = 100_000
    g = torch.full((2, n), 3e38, device="cuda")
    g[1, 5] = math.inf
    norms = torch.zeros(2, device="cuda")
    op = P.GradientClip(workers=2, eps=0.0, cuda_stream=stream())
    lists = P.TensorList([(g, n, n)])
    op.clip(lists, lists, 1.0, norms)
    assert bool(norms.isinf().all())
    within(g[0], torch.full((n,), 1 / math.sqrt(n), dtype=torch.float64, device="cuda"), 40 * U / math.sqrt(n), "clipped")
    assert float(g[1, 0]) == float(torch.tensor(3e38)) and bool(g[1, 5].isinf())
    op.destroy()
