"""The token model through Algorithm 2: its gradient rows against automatic differentiation of the same
model in 64 bits, and a training run whose loss falls with every compressor."""
from __future__ import annotations

import math

import pytest

from operator_references import U

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def P():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2010_13359_gb300 as P
    return P


def data(M, n, V, C, k, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ids = torch.randint(0, V, (M, n), generator=g, device="cuda", dtype=torch.int32)
    ids[torch.rand((M, n), generator=g, device="cuda") < 0.1] = -1
    teacher = torch.randn((V, V), generator=g, device="cuda") * 2  # a bigram teacher: logits of the next token
    values, tid = teacher[ids.clamp(min=0).view(-1).long()].topk(k, 1)
    weights = (ids.view(-1) >= 0).float()
    return ids, tid.int(), values.contiguous(), weights


def loss64(w, V, C, ids, tid, values, weights, T):
    E, gamma, beta = w[:V * C].view(V, C), w[V * C:V * C + C], w[V * C + C:]
    x = torch.where((ids >= 0)[:, None], math.sqrt(C) * E[ids.clamp(min=0).long()], 0)
    x = torch.nn.functional.layer_norm(x, (C,), gamma, beta, 1e-5)
    logp = torch.log_softmax(values.double() / T, 1)
    logq = torch.log_softmax(x @ E.t() / T, 1).gather(1, tid.long())
    return (weights.double() * T * T * (logp.exp() * (logp - logq)).sum(1)).sum() / len(ids)


def test_gradient_rows(P):
    from paper_2010_13359_gb300.token_model import TokenModel
    M, n, V, C, k, T = 3, 40, 61, 33, 7, 1.5
    s = torch.cuda.current_stream().cuda_stream
    model = TokenModel(V, C, n, M, k, T, cuda_stream=s)
    ids, tid, values, weights = data(M, n, V, C, k, 1)
    ld = model.d + 9
    w = torch.zeros((M, ld), device="cuda")
    g0 = torch.Generator(device="cuda")
    g0.manual_seed(3)
    w[:, :model.d] = 0.2 * torch.randn((M, model.d), generator=g0, device="cuda")
    w[:, V * C:V * C + C] += 1
    g = torch.full((M, ld), math.nan, device="cuda")
    b = model.buffers("cuda")
    before = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    model.operator(w[:, :model.d], ids, tid, values, weights, g, b)
    torch.backends.cuda.matmul.allow_tf32 = before
    for m in range(M):
        p = w[m, :model.d].double().requires_grad_()
        rows = slice(m * n, (m + 1) * n)
        loss = loss64(p, V, C, ids[m], tid[rows], values[rows], weights[rows], T)
        loss.backward()
        # chains of products over width, vocabulary and tokens in 32 bits: a few hundred u of the largest
        assert float((g[m, :model.d].double() - p.grad).abs().max()) <= 1024 * U * float(p.grad.abs().max())
        assert abs(float(b["loss"][rows].double().mean()) - float(loss.detach())) <= 1024 * U * float(loss.detach())
    assert bool(g[:, model.d:].isnan().all())


@pytest.mark.parametrize("compressor", ["SIGN", "TOPK", "SQUANT", "IDENTITY"])
def test_training_lowers_the_loss(P, compressor):
    from paper_2010_13359_gb300.token_model import TokenModel, train
    M, n, V, C, k = 4, 256, 96, 32, 8
    s = torch.cuda.current_stream().cuda_stream
    model = TokenModel(V, C, n, M, k, cuda_stream=s)
    batch = data(M, n, V, C, k, 5)
    h = P.create(P.make_config(d=model.d, M=M, compressor=getattr(P, compressor), lr=0.2, bucket=64, k=model.d // 10,
                               bits=8, flags=P.KEEP_LOOKAHEAD, cuda_stream=s))
    w = torch.zeros(model.d, device="cuda")
    g0 = torch.Generator(device="cuda")
    g0.manual_seed(6)
    w[:V * C] = 0.1 * torch.randn(V * C, generator=g0, device="cuda")
    w[V * C:V * C + C] = 1
    losses = []
    train(h, model, w, lambda t: batch, 60, on_step=lambda t, loss: losses.append(loss.mean()))
    h.synchronize()
    first, last = float(losses[0]), float(torch.stack(losses[-5:]).mean())
    assert last < 0.7 * first, (first, last)
