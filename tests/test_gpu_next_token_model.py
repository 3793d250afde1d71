"""The model of linear layers and cross entropy through Algorithm 2: its gradient rows against automatic
differentiation of the same model in 64 bits, and training runs with clipping."""
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


def data(M, n, V, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ids = torch.randint(0, V, (M, n), generator=g, device="cuda", dtype=torch.int32)
    ids[torch.rand((M, n), generator=g, device="cuda") < 0.1] = -1
    targets = (ids * 7 + 3) % V
    targets[ids < 0] = -1
    weights = 0.5 + torch.rand(M * n, generator=g, device="cuda")
    return ids, targets, weights


def loss64(model, w, ids, targets, weights):
    F = torch.nn.functional
    V, C, H = model.vocab, model.width, model.hidden
    places = model.places()
    E = w[:V * C].view(V, C)
    x = torch.where((ids >= 0)[:, None], math.sqrt(C) * E[ids.clamp(min=0).long()], 0)
    for g, b, w1, b1, w2, b2 in places[:-1]:
        y = F.layer_norm(x, (C,), w[g:g + C], w[b:b + C], 1e-5)
        y = F.gelu(y @ w[w1:w1 + H * C].view(H, C).t() + w[b1:b1 + H])
        x = x + y @ w[w2:w2 + C * H].view(C, H).t() + w[b2:b2 + C]
    g, b = places[-1]
    logp = torch.log_softmax(F.layer_norm(x, (C,), w[g:g + C], w[b:b + C], 1e-5) @ E.t(), 1)
    picked = logp.gather(1, targets.clamp(min=0).long()[:, None])[:, 0]
    return -(torch.where(targets >= 0, weights.double(), 0) * picked).sum() / len(ids)


def parameters(model, rows, ld, seed):
    w = torch.zeros((rows, ld), device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    w[:, :model.d] = 0.2 * torch.randn((rows, model.d), generator=g, device="cuda")
    for layer in model.places():
        w[:, layer[0]:layer[0] + model.width] += 1
    return w


@pytest.mark.parametrize("n", [6, 40])
def test_gradient_rows(P, n):
    from paper_2010_13359_gb300.token_model import NextTokenModel
    M, V, C, H, L = 3, 61, 33, 70, 2
    model = NextTokenModel(V, C, H, L, n, M, cuda_stream=torch.cuda.current_stream().cuda_stream)
    ids, targets, weights = data(M, n, V, 1)
    w = parameters(model, M, model.d + 9, 3)
    g = torch.full_like(w, math.nan)
    b = model.buffers("cuda")
    model.operator(w[:, :model.d], ids, targets, weights, g, b)
    for m in range(M):
        p = w[m, :model.d].double().requires_grad_()
        part = slice(m * n, (m + 1) * n)
        loss = loss64(model, p, ids[m], targets[m], weights[part])
        loss.backward()
        # chains of products over widths, vocabulary and tokens in 32 bits: some thousand u of the largest
        assert float((g[m, :model.d].double() - p.grad).abs().max()) <= 4096 * U * float(p.grad.abs().max())
        assert abs(float(b["loss"][part].double().mean()) - float(loss.detach())) <= 1024 * U * float(loss.detach())
    assert bool(g[:, model.d:].isnan().all())


def test_gradient_rows_in_bf16(P):
    """bf16 activations: rounded at some ten places a layer, 2^-8 each, which the layers pass on."""
    from paper_2010_13359_gb300.token_model import NextTokenModel
    M, n, V, C, H, L = 2, 300, 500, 64, 128, 2
    model = NextTokenModel(V, C, H, L, n, M, dtype=P.BF16, cuda_stream=torch.cuda.current_stream().cuda_stream)
    ids, targets, weights = data(M, n, V, 2)
    w = parameters(model, M, model.d, 4)
    g = torch.full_like(w, math.nan)
    model.operator(w, ids, targets, weights, g, model.buffers("cuda"))
    for m in range(M):
        p = w[m].double().requires_grad_()
        loss64(model, p, ids[m], targets[m], weights[m * n:(m + 1) * n]).backward()
        assert float((g[m].double() - p.grad).norm()) <= 40 * 2.0 ** -8 * float(p.grad.norm())


@pytest.mark.parametrize("compressor,max_norm", [("SIGN", None), ("TOPK", 0.5), ("SQUANT", 0.5), ("IDENTITY", 1e-3)])
def test_training_runs(P, compressor, max_norm):
    from paper_2010_13359_gb300.token_model import NextTokenModel, train
    M, n, V, C, H, L = 3, 64, 48, 16, 32, 1
    s = torch.cuda.current_stream().cuda_stream
    model = NextTokenModel(V, C, H, L, n, M, cuda_stream=s)
    batch = data(M, n, V, 5)
    h = P.create(P.make_config(d=model.d, M=M, compressor=getattr(P, compressor), lr=0.1, bucket=64, k=model.d // 10, bits=8,
                               flags=P.KEEP_LOOKAHEAD, cuda_stream=s))
    w = parameters(model, 1, model.d, 6)[0]
    before = w.clone()
    losses = []
    train(h, model, w, lambda t: batch, 5, on_step=lambda t, loss: losses.append(loss), max_norm=max_norm)
    h.synchronize()
    assert len(losses) == 5 and bool(torch.stack(losses).isfinite().all()) and bool(w.isfinite().all())
    moved = float((w - before).double().norm())
    assert moved > 0
    if compressor == "IDENTITY":  # five steps of lr times a mean of gradients of at most that norm, each rounded
        assert moved <= 5 * 0.1 * max_norm * (1 + 1e-4) + 10 * U * float(w.norm())
