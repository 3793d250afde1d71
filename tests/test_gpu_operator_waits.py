"""A bounded wait that gives up in an operator's kernels: the next synchronize says so, once, and the operator and the
context stay usable.  The wait is the self-test's, on a barrier at which nothing arrives."""
from __future__ import annotations

import pytest

from test_gpu_products import P, gen, stream  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("polls", [1, 4096, 0])
@pytest.mark.parametrize("make", [
    lambda P, s: P.Linear(inputs=64, outputs=96, max_rows=40, dtype=P.BF16, weight_dtype=P.BF16, cuda_stream=s),
    lambda P, s: P.TokenLoss(vocab=96, width=64, max_rows=40, dtype=P.BF16, weight_dtype=P.BF16, cuda_stream=s),
], ids=["linear", "token loss"])
def test_a_wait_that_gives_up_is_reported_once(P, make, polls):  # noqa: F811
    op, other = make(P, stream()), make(P, stream())
    x = torch.randn((40, 64), generator=gen(1), device="cuda").bfloat16()
    w = torch.randn((96, 64), generator=gen(2), device="cuda").bfloat16()
    targets = torch.arange(40, dtype=torch.int32, device="cuda")
    y, again = torch.zeros((2, 40, 96), dtype=torch.bfloat16, device="cuda")

    def call(out):
        if isinstance(op, P.Linear):
            op.forward(40, x, 64, w, 0, None, 0, None, 0, out, 96)
        else:
            op.forward(40, x, 64, w, 0, targets, None, out.view(-1)[:80].view(torch.float32))

    call(y)
    op.synchronize()
    launches = op.launch_count()
    op.selftest_wait_timeout(polls)
    assert op.launch_count() == launches + 1
    with pytest.raises(P.DqganError) as ei:
        op.synchronize()
    assert ei.value.status == P.ERR_TIMEOUT and "gave up" in str(ei.value)
    other.synchronize()  # each operator has its own word
    op.synchronize()  # and it was cleared
    call(again)
    op.synchronize()
    assert torch.equal(y.view(torch.int16), again.view(torch.int16)) and bool(y.any())
    op.destroy()
    other.destroy()


def test_refusals(P):  # noqa: F811
    op, norm = P.Linear(inputs=8, outputs=8, max_rows=1), P.LayerNorm(width=8)
    for o, polls, needle in ((op, (1 << 21) + 1, "polls"), (norm, 1, "do not wait")):
        with pytest.raises(P.DqganError) as ei:
            o.selftest_wait_timeout(polls)
        assert ei.value.status == P.dqgan.ERR_INVALID_ARG and needle in str(ei.value)
    op.destroy()
    norm.destroy()
