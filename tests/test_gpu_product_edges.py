"""Linear layers, token loss and clipping where they can go wrong: refusals, no rows, other streams and graphs, two host
threads, pieces of the vocabulary, places beyond 32 bits, values at the ends of the types' ranges, gradients against
differences."""
from __future__ import annotations

import math
import threading

import pytest

from operator_references import U, within
from product_references import activation, linear_backward, linear_forward, token_loss
from test_gpu_products import P, gen, rows_of, stream, test_token_loss as token_loss_case  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def refused(P, call, needle):  # noqa: F811
    with pytest.raises(P.DqganError) as ei:
        call()
    assert ei.value.status == P.dqgan.ERR_INVALID_ARG
    assert needle in str(ei.value), str(ei.value)


def test_refusals(P):  # noqa: F811
    x = torch.zeros(256, device="cuda")
    a = x.data_ptr()
    op = P.Linear(inputs=8, outputs=4, max_rows=3, workers=2, activation=P.SILU, cuda_stream=stream())

    def forward(rows=1, x=x, xs=8, w=x, ps=32, b=x, bs=4, r=None, rs=0, y=x, ys=4, pre=None, pres=0):
        return lambda: op.forward(rows, x, xs, w, ps, b, bs, r, rs, y, ys, pre, pres)

    for kw, needle in ((dict(rows=-1), "rows"), (dict(rows=4), "rows"), (dict(x=None), "NULL"), (dict(w=None), "NULL"),
                       (dict(y=None), "NULL"), (dict(xs=7), "stride"), (dict(ys=3), "stride"), (dict(ps=31), "p_stride"),
                       (dict(bs=3), "b_stride"), (dict(r=x, rs=3), "stride"), (dict(pre=x, pres=3), "stride"),
                       (dict(x=a + 2), "aligned"), (dict(w=a + 1), "aligned"), (dict(pre=a + 2, pres=4), "aligned"),
                       (dict(xs=1 << 41), "stride")):
        refused(P, forward(**kw), needle)

    def backward(rows=1, dy=x, dys=4, x=x, xs=8, w=x, ps=32, pre=x, pres=4, dx=x, dxs=8, dw=x, db=x, gs=36):
        return lambda: op.backward(rows, dy, dys, x, xs, w, ps, pre, pres, dx, dxs, dw, db, gs)

    for kw, needle in ((dict(rows=4), "rows"), (dict(dy=None), "NULL"), (dict(x=None), "NULL"), (dict(w=None), "NULL"),
                       (dict(pre=None), "NULL"), (dict(dys=3), "stride"), (dict(xs=7), "stride"), (dict(dxs=7), "stride"),
                       (dict(pres=3), "stride"), (dict(ps=31), "p_stride"), (dict(gs=31), "g_stride"),
                       (dict(dw=a + 2), "aligned"), (dict(dy=a + 3), "aligned")):
        refused(P, backward(**kw), needle)
    op.forward(0, None, 8, None, 32, None, 0, None, 0, None, 4)
    backward(dx=None, dw=None, db=None, dy=None)()

    loss = P.TokenLoss(vocab=4, width=8, max_rows=3, workers=2, cuda_stream=stream())
    ids = torch.zeros(6, dtype=torch.int32, device="cuda")

    def step(rows=1, x=x, xs=8, w=x, ps=32, t=ids, scale=1.0, loss_=x, dx=x, dxs=8, dw=x, gs=32):
        return lambda: loss.step(rows, x, xs, w, ps, t, None, scale, loss_, None, dx, dxs, dw, gs)

    for kw, needle in ((dict(rows=4), "rows"), (dict(rows=-1), "rows"), (dict(x=None), "NULL"), (dict(w=None), "NULL"),
                       (dict(t=None), "NULL"), (dict(loss_=None), "loss"), (dict(xs=7), "stride"), (dict(dxs=7), "stride"),
                       (dict(ps=31), "p_stride"), (dict(gs=31), "g_stride"), (dict(scale=math.inf), "scale"),
                       (dict(t=ids.data_ptr() + 2), "aligned"), (dict(dw=a + 1), "aligned")):
        refused(P, step(**kw), needle)
    refused(P, lambda: loss.backward(1, x, 8, x, 32, ids, None, None, 1.0, x, 8, x, 32), "lse")
    refused(P, lambda: op.forward(1, x, 8, x, 32, ids, 0, None, 0, x, 4), "torch.int32")
    loss.forward(0, None, 8, None, 32, None, None, None)

    clip = P.GradientClip(workers=2, dtype=P.F32, cuda_stream=stream())
    good = P.TensorList([(x, 8, 8)])
    for tensors, places, norm, needle in (
            ([(x, -1, 8)], [(x, -1, 8)], 1.0, "size"), ([(None, 8, 8)], [(x, 8, 8)], 1.0, "NULL"),
            ([(x, 8, 7)], [(x, 8, 8)], 1.0, "stride"), ([(x, 8, 8)], [(x, 7, 8)], 1.0, "size"),
            ([(a + 2, 8, 8)], [(x, 8, 8)], 1.0, "aligned"), ([(x, 8, 8)], [(x, 8, 16)], 1.0, "stride"),
            ([(x, 8, 8)], [(x, 8, 8)], -1.0, "max_norm"), ([(x, 8, 8)], [(x, 8, 8)], math.nan, "max_norm"),
            ([(x, 0, 0)] * 4097, [(x, 0, 0)] * 4097, 1.0, "count")):
        refused(P, lambda: clip.clip(P.TensorList(tensors), P.TensorList(places), norm, x), needle)
    refused(P, lambda: clip.norm(good, None), "norms")
    refused(P, lambda: clip.norm(good, a + 2), "aligned")
    mixed = P.GradientClip(workers=1, dtype=P.BF16, out_dtype=P.F32, cuda_stream=stream())
    refused(P, lambda: mixed.clip(P.TensorList([(a, 8, 8)]), P.TensorList([(a, 8, 8)]), 1.0), "another type")
    L = P.dqgan.load_library()
    assert L.dqgan_linear_forward(loss._h, 1, a, 8, a, 32, None, 0, None, 0, a, 4, None, 0) == P.dqgan.ERR_INVALID_ARG
    assert "linear layer" in loss.last_error()
    for o in (op, loss, clip, mixed):
        o.synchronize()
        assert o.launch_count() == 0
        o.destroy()
    assert not x.any()


@pytest.mark.parametrize("make", [lambda P: P.Linear(inputs=64, outputs=64, max_rows=10),
                                  lambda P: P.TokenLoss(vocab=64, width=64, max_rows=10), lambda P: P.GradientClip()])
def test_allocation_failure(P, monkeypatch, make):  # noqa: F811
    monkeypatch.setenv("DQGAN_TEST_FAIL_ALLOC", "1")
    with pytest.raises(P.DqganError) as ei:
        make(P)
    assert ei.value.status == P.dqgan.ERR_OOM
    monkeypatch.delenv("DQGAN_TEST_FAIL_ALLOC")
    make(P).destroy()


def test_too_large_a_scratch_is_an_error(P):  # noqa: F811
    with pytest.raises(P.DqganError) as ei:
        P.Linear(inputs=65536, outputs=65536, max_rows=1 << 16, workers=4096)
    assert ei.value.status == P.dqgan.ERR_OOM


def test_gradients_of_no_rows_and_no_tensors(P):  # noqa: F811
    """Zeros, or what was there; the rows' pointers are not looked at."""
    W, K, N = 3, 20, 12
    linear = P.Linear(inputs=K, outputs=N, max_rows=5, workers=W, activation=P.GELU, cuda_stream=stream())
    loss = P.TokenLoss(vocab=N, width=K, max_rows=5, workers=W, cuda_stream=stream())
    stride = K * N + N + 3
    for accumulate in (False, True):
        g = torch.full((W, stride), 2.5, device="cuda")
        linear.backward(0, None, N, None, K, None, 0, None, N, None, K, g, g[:, K * N:], stride, accumulate=accumulate)
        assert bool((g[:, :K * N + N] == (2.5 if accumulate else 0)).all()) and bool((g[:, K * N + N:] == 2.5).all())
        g.fill_(2.5)
        loss.step(0, None, K, None, 0, None, None, 1.0, None, None, None, K, g, stride, accumulate=accumulate)
        assert bool((g[:, :K * N] == (2.5 if accumulate else 0)).all()) and bool((g[:, K * N:] == 2.5).all())
    clip = P.GradientClip(workers=2, cuda_stream=stream())
    for tensors in ([], [(None, 0, 0)] * 3):
        norms = torch.full((2,), math.nan, device="cuda")
        clip.clip(P.TensorList(tensors), P.TensorList(tensors), 1.0, norms)
        assert not norms.any()
        norms.fill_(math.nan)
        clip.norm(P.TensorList(tensors), norms)
        assert not norms.any()


def test_other_stream_and_graph(P):  # noqa: F811
    """On a stream of its own, captured once and replayed on new data: the same bits as the calls."""
    s = torch.cuda.Stream()
    W, n, V, C, H = 2, 300, 1000, 64, 200
    kw = dict(workers=W, dtype=P.BF16, cuda_stream=s.cuda_stream)
    widen = P.Linear(inputs=C, outputs=H, max_rows=n, activation=P.GELU, **kw)
    narrow = P.Linear(inputs=H, outputs=C, max_rows=n, **kw)
    few = P.Linear(inputs=H, outputs=C, max_rows=4, **kw)
    loss_op = P.TokenLoss(vocab=V, width=C, max_rows=n, **kw)
    clip = P.GradientClip(workers=W, cuda_stream=s.cuda_stream)
    d = [H * C, H, C * H, C, V * C]
    at = [sum(d[:i]) for i in range(6)]
    params = torch.randn((W, at[5]), generator=gen(1), device="cuda") / 8
    g = torch.zeros_like(params)
    ps = params.stride(0)
    x = torch.zeros((W * n, C), dtype=torch.bfloat16, device="cuda")
    u, h, dh = torch.zeros((3, W * n, H), dtype=torch.bfloat16, device="cuda")
    y, dy, dx, z = torch.zeros((4, W * n, C), dtype=torch.bfloat16, device="cuda")
    targets = torch.zeros(W * n, dtype=torch.int32, device="cuda")
    loss, norms = torch.zeros(W * n, device="cuda"), torch.zeros(W, device="cuda")
    lists = P.TensorList([(g[:, a:], m, ps) for a, m in zip(at, d)])

    def step():
        w = [params[:, a:] for a in at[:5]]
        k = [g[:, a:] for a in at[:5]]
        widen.forward(n, x, C, w[0], ps, w[1], ps, None, 0, h, H, u, H)
        narrow.forward(n, h, H, w[2], ps, w[3], ps, x, C, y, C)
        few.forward(4, h, H, w[2], ps, w[3], ps, None, 0, z, C)
        loss_op.step(n, y, C, w[4], ps, targets, None, 1.0 / n, loss, None, dy, C, k[4], ps)
        narrow.backward(n, dy, C, h, H, w[2], ps, None, 0, dh, H, k[2], k[3], ps)
        widen.backward(n, dh, H, x, C, w[0], ps, u, H, dx, C, k[0], k[1], ps)
        clip.clip(lists, lists, 0.5, norms)

    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        step()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            step()
        for seed in (5, 6):
            x.copy_(torch.randn(x.shape, generator=gen(seed), device="cuda"))
            targets.copy_(torch.randint(-1, V, targets.shape, generator=gen(seed), device="cuda"))
            graph.replay()
            s.synchronize()
            replayed = [t.clone() for t in (y, z, loss, dx, g, norms)]
            step()
            s.synchronize()
            for a, b in zip(replayed, (y, z, loss, dx, g, norms)):
                assert torch.equal(a, b)
            assert float(norms.min()) > 0 and float(loss.max()) > 0
    for o in (widen, narrow, few, loss_op, clip):
        assert o.launch_count() > 0
        o.synchronize()


def test_two_host_threads(P):  # noqa: F811
    """Each with operators and a stream of its own: the results of one after another."""
    n, K, N = 700, 320, 640

    def work(seed, results):
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            g = torch.Generator(device="cuda")
            g.manual_seed(seed)
            x = torch.randn((n, K), generator=g, device="cuda").bfloat16()
            w = torch.randn(N * K, generator=g, device="cuda").bfloat16()
            y = torch.zeros((n, N), dtype=torch.bfloat16, device="cuda")
            dx, dw = torch.zeros_like(x), torch.zeros(N * K, device="cuda")
            op = P.Linear(inputs=K, outputs=N, max_rows=n, dtype=P.BF16, weight_dtype=P.BF16, cuda_stream=s.cuda_stream)
            for _ in range(20):
                op.forward(n, x, K, w, 0, None, 0, None, 0, y, N)
                op.backward(n, y, N, x, K, w, 0, None, 0, dx, K, dw, None, N * K)
            op.synchronize()
            op.destroy()
            results[seed] = [t.cpu() for t in (y, dx, dw)]

    alone, beside = {}, {}
    for seed in (1, 2):
        work(seed, alone)
    threads = [threading.Thread(target=work, args=(seed, beside)) for seed in (1, 2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for seed in (1, 2):
        for a, b in zip(alone[seed], beside[seed]):
            assert torch.equal(a, b)


@pytest.mark.parametrize("shape", [
    (1, 65536, 5000, 16, 1, 1, 32, 0, 0, False, 0.05),     # the gradient in two pieces of the vocabulary
    (2, 30000, 4500, 24, 2, 2, 32, 0, 0, False, 0.05),     # the same with operands of both 16-bit types
    (1, 10, 4200, 65536, 1, 0, 32, 0, 0, False, 0.0),       # the weights' parts in pieces
    (1, 40000, 4400, 40, 0, 0, 64, 0, 0, False, 0.05),
    # few rows of pieces that have few tiles, of a vocabulary too large for narrow ones' slots
    (1, 12, 20000, 14000, 1, 0, 32, 0, 0, False, 0.0),
], ids=str)
def test_token_loss_in_pieces(P, shape):  # noqa: F811
    token_loss_case(P, shape)


def test_weights_beyond_32_bits(P):  # noqa: F811
    """More than 2^31 values in the table and its gradient."""
    V, C, n = 140_000, 16_384, 20
    g = gen(3)
    weight = torch.empty(V * C, dtype=torch.bfloat16, device="cuda")
    for part in weight.split(1 << 28):
        part.copy_(torch.randn(part.shape, generator=g, device="cuda") / 64)
    x = torch.randn((n, C), generator=g, device="cuda").bfloat16()
    targets = torch.randint(V - 1000, V, (n,), generator=g, device="cuda").int()
    loss, lse = torch.zeros((2, n), device="cuda")
    dx = torch.zeros_like(x)
    dw = torch.full((V * C,), math.nan, device="cuda")
    op = P.TokenLoss(vocab=V, width=C, max_rows=n, dtype=P.BF16, weight_dtype=P.BF16, cuda_stream=stream())
    op.step(n, x, C, weight, 0, targets, None, 1.0, loss, lse, dx, C, dw, 0)
    op.synchronize()
    z = torch.cat([x.double() @ w.double().t() for w in weight.view(V, C).split(10_000)], 1)
    want = torch.logsumexp(z, 1)
    # one term of bf16 operands: the sums' errors and the exponentials'
    e_z = float((x.double().abs() @ weight.view(V, C)[:1000].double().abs().t()).amax()) * 2 * (64 * 2 * 2 ** -23 + 170 * U)
    assert float((lse.double() - want).abs().max()) <= e_z + (V / 32 + 200) * U * float(want.abs().max())
    at = targets.long()
    p = torch.exp(z - want[:, None])
    p[torch.arange(n, device="cuda"), at] -= 1
    first = torch.tensor([0, 1, 131_071, 131_072, 139_999, int(at[0])], device="cuda")  # 131,072 * 16,384 is 2^31
    got = dw.view(V, C)[first].double()
    ref = p[:, first].t() @ x.double()
    size = p[:, first].abs().t() @ x.double().abs()
    within(got, ref, size * (2 ** -16 + 3 * 2 ** -16 + 2 * e_z + 64 * 2 * 2 ** -23 + 400 * U), "dweight")
    assert bool(dw.isfinite().all())
    op.destroy()


def test_a_tensor_beyond_32_bits_is_clipped(P):  # noqa: F811
    n = (1 << 31) + 12345
    t = torch.full((n,), 2.0 ** -10, dtype=torch.bfloat16, device="cuda")
    t[-1] = 3.0
    want = math.sqrt((n - 1) * 2.0 ** -20 + 9)
    norms = torch.zeros(1, device="cuda")
    op = P.GradientClip(dtype=P.BF16, out_dtype=P.BF16, eps=0.0, cuda_stream=stream())
    lists = P.TensorList([(t, n, n)])
    op.clip(lists, lists, want / 4, norms)
    op.synchronize()
    assert abs(float(norms) - want) <= 40 * U * want
    assert float(t[0]) == 2.0 ** -12 and float(t[-2]) == 2.0 ** -12 and float(t[1 << 31]) == 2.0 ** -12 and float(t[-1]) == 0.75
    op.destroy()


def test_norms_at_the_ends_of_the_range(P):  # noqa: F811
    """Squares beyond fp32's range on both sides; a worker whose norm is not finite is passed on as it is."""
    n = 50_000
    g = torch.randn((8, n), generator=gen(9), device="cuda")
    g[0] *= 1e30
    g[1] *= 1e-30
    g[2] = 0
    g[3] *= 1e-42  # subnormal
    g[4, 77] = math.inf
    g[5, 78] = math.nan
    g[6] = 0
    g[6, 123] = 1e-25
    before = g.clone()
    norms = torch.zeros(8, device="cuda")
    op = P.GradientClip(workers=8, eps=0.0, cuda_stream=stream())
    lists = P.TensorList([(g, n, n)])
    op.clip(lists, lists, 1e-31, norms)
    want = before.double().square().sum(1).sqrt()
    ok = [0, 1, 2, 3, 6, 7]
    within(norms[ok], want[ok], 40 * U * want[ok] + 2.0 ** -149, "norms")
    assert norms[4] == math.inf and norms[5].isnan()
    assert torch.equal(g[4], before[4]) and torch.equal(g[5].isnan(), before[5].isnan())
    factor = (1e-31 / want[ok]).clamp(max=1).nan_to_num(1)
    after = before[ok].double() * factor[:, None]
    # a result below 2^-126 is rounded to 2^-150
    within(g[ok], after, 40 * U * after.abs() + 2.0 ** -149, "clipped")
    limit = torch.full((8, n), 5.0, device="cuda")
    op.clip(P.TensorList([(limit, n, n)]), P.TensorList([(limit, n, n)]), math.inf, norms)
    assert bool((limit == 5).all())
    op.clip(P.TensorList([(limit, n, n)]), P.TensorList([(limit, n, n)]), 0.0, norms)
    assert not limit.any()
    op.destroy()


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("rows", [3, 40])
def test_values_that_are_not_finite_stay_in_their_rows(P, dtype, rows):  # noqa: F811
    """A NaN or an infinity in one row of x changes that row of y alone; large finite values stay finite."""
    T = {0: torch.float32, 1: torch.bfloat16, 2: torch.float16}[dtype]
    K, N = 128, 96
    x = torch.randn((rows, K), generator=gen(5), device="cuda").to(T)
    w = torch.randn(N * K, generator=gen(6), device="cuda").to(T)
    op = P.Linear(inputs=K, outputs=N, max_rows=rows, dtype=dtype, weight_dtype=dtype, cuda_stream=stream())
    y, bad = torch.zeros((2, rows, N), dtype=T, device="cuda")
    op.forward(rows, x, K, w, 0, None, 0, None, 0, y, N)
    x[1, 7], x[2, 9] = math.nan, math.inf
    op.forward(rows, x, K, w, 0, None, 0, None, 0, bad, N)
    others = [r for r in range(rows) if r not in (1, 2)]
    assert torch.equal(bad[others], y[others]) and not bad[1:3].isfinite().any()
    # the type's largest value through an identity
    x.zero_()
    x[:, 0] = torch.finfo(T).max
    eye = torch.eye(N, K, device="cuda").to(T).view(-1).contiguous()
    op.forward(rows, x, K, eye, 0, None, 0, None, 0, y, N)
    # of three parts: the value to 24 bits; else exact
    assert float((y[:, 0].double() / torch.finfo(T).max - 1).abs().max()) <= (2.0 ** -22 if dtype == 0 else 0)
    assert not y[:, 1:].any()
    op.destroy()


def test_large_logits_and_equal_ones(P):  # noqa: F811
    """Logits of 1e4, all equal, and a vocabulary of one entry."""
    V, C, n = 3000, 64, 30
    x = torch.randn((n, C), generator=gen(1), device="cuda")
    w = torch.randn((V, C), generator=gen(2), device="cuda")
    x[0] *= 1000
    x[1] = 0
    targets = torch.randint(0, V, (n,), generator=gen(3), device="cuda").int()
    op = P.TokenLoss(vocab=V, width=C, max_rows=n, cuda_stream=stream())
    loss, lse = torch.zeros((2, n), device="cuda")
    dx, dw = torch.zeros_like(x), torch.zeros_like(w)
    op.step(n, x, C, w, 0, targets, None, 1.0, loss, lse, dx, C, dw, 0)
    ones = torch.ones(n, dtype=torch.float64, device="cuda")
    ref = token_loss(x.double(), w.double(), targets.long(), ones, 1.0, 0, 0)
    within(loss, ref[0], ref[4], "loss")
    within(lse, ref[1], ref[5], "lse")
    within(dx, ref[2], ref[6], "dx")
    within(dw, ref[3], ref[7], "dweight")
    assert abs(float(loss[1]) - math.log(V)) <= 16 * U * math.log(V)
    one = P.TokenLoss(vocab=1, width=C, max_rows=n, cuda_stream=stream())
    one.step(n, x, C, w, 0, torch.zeros_like(targets), None, 1.0, loss, lse, dx, C, dw, 0)
    z = x.double() @ w[0].double()
    assert float(loss.abs().max()) <= 8 * U * float(z.abs().max())
    within(lse, z, 1e-5 * (x.double().abs() @ w[0].double().abs()), "lse of one entry")
    op.destroy()
    one.destroy()


@pytest.mark.parametrize("kind", [0, 1, 2, 3])
def test_linear_gradient_is_the_differences(P, kind):  # noqa: F811
    n, K, N = 12, 5, 4
    g = gen(14)
    x, w, b = (torch.randn(s, generator=g, device="cuda") for s in ((n, K), (N, K), (N,)))
    dy = torch.randn((n, N), generator=g, device="cuda")
    op = P.Linear(inputs=K, outputs=N, max_rows=n, activation=kind, cuda_stream=stream())
    y, pre = torch.zeros((2, n, N), device="cuda")
    op.forward(n, x, K, w, 0, b, 0, None, 0, y, N, pre, N)
    dx, grads = torch.zeros_like(x), torch.zeros(N * K + N, device="cuda")
    op.backward(n, dy, N, x, K, w, 0, pre, N, dx, K, grads, grads[N * K:], 0)

    def f(x, w, b):
        return float((activation(x @ w.t() + b, kind) * dy.double()).sum())

    at = [t.double() for t in (x, w, b)]
    step = 1e-6
    for t, got in zip(range(3), (dx, grads[:N * K].view(N, K), grads[N * K:])):
        for i in range(at[t].numel()):
            up, down = [v.clone() for v in at], [v.clone() for v in at]
            up[t].view(-1)[i] += step
            down[t].view(-1)[i] -= step
            # the formula's values are some tens; differences lose 2^-53 of them over the step
            assert abs((f(*up) - f(*down)) / (2 * step) - float(got.reshape(-1)[i])) <= 1e-5
    op.destroy()


def test_token_loss_gradient_is_the_differences(P):  # noqa: F811
    n, V, C = 3, 7, 4
    g = gen(15)
    x, w = torch.randn((n, C), generator=g, device="cuda"), torch.randn((V, C), generator=g, device="cuda")
    targets = torch.tensor([2, -1, 6], dtype=torch.int32, device="cuda")
    weights = torch.tensor([0.7, 1.0, 1.3], device="cuda")
    op = P.TokenLoss(vocab=V, width=C, max_rows=n, cuda_stream=stream())
    loss, lse = torch.zeros((2, n), device="cuda")
    dx, dw = torch.zeros_like(x), torch.zeros_like(w)
    op.step(n, x, C, w, 0, targets, weights, 2.0, loss, lse, dx, C, dw, 0)

    def f(x, w):
        logp = torch.log_softmax(x @ w.t(), 1)
        return float(-2 * (0.7 * logp[0, 2] + 1.3 * logp[2, 6]))

    at, step = [x.double(), w.double()], 1e-6
    for t, got in zip(range(2), (dx, dw)):
        for i in range(at[t].numel()):
            up, down = [v.clone() for v in at], [v.clone() for v in at]
            up[t].view(-1)[i] += step
            down[t].view(-1)[i] -= step
            assert abs((f(*up) - f(*down)) / (2 * step) - float(got.view(-1)[i])) <= 1e-5
    op.destroy()


@pytest.mark.parametrize("weights", [None, "zeros"])
def test_nothing_counts(P, weights):  # noqa: F811
    n, V, C = 200, 900, 72
    x = torch.full((n, C), math.nan, dtype=torch.bfloat16, device="cuda")
    w = torch.randn(V * C, generator=gen(1), device="cuda").bfloat16()
    targets = torch.full((n,), -1 if weights is None else 5, dtype=torch.int32, device="cuda")
    op = P.TokenLoss(vocab=V, width=C, max_rows=n, dtype=P.BF16, weight_dtype=P.BF16, cuda_stream=stream())
    loss, lse = torch.full((2, n), math.nan, device="cuda")
    dx, dw = torch.full_like(x, 3), torch.full((V * C,), math.nan, device="cuda")
    op.step(n, x, C, w, 0, targets, None if weights is None else torch.zeros(n, device="cuda"), 1.0, loss, lse, dx, C, dw, 0)
    for t in (loss, lse, dx, dw):
        assert not t.any()
    op.destroy()


@pytest.mark.parametrize("rows", [8, 9, 128, 129, 257])
def test_the_same_bits_again_and_rows_apart(P, rows):  # noqa: F811
    """Twice the same call gives the same bits, and workers do not reach into one another."""
    W, K, N = 3, 96, 200
    x = torch.randn((W * rows, K), generator=gen(1), device="cuda").bfloat16()
    w = torch.randn((W, N * K), generator=gen(2), device="cuda").bfloat16()
    y = torch.zeros((2, W * rows, N), dtype=torch.bfloat16, device="cuda")
    g = torch.zeros((2, W, N * K), device="cuda")
    op = P.Linear(inputs=K, outputs=N, max_rows=rows, workers=W, dtype=P.BF16, weight_dtype=P.BF16, cuda_stream=stream())
    for i in range(2):
        op.forward(rows, x, K, w, N * K, None, 0, None, 0, y[i], N)
        op.backward(rows, y[0], N, x, K, w, N * K, None, 0, None, K, g[i], None, N * K)
    assert torch.equal(y[0], y[1]) and torch.equal(g[0], g[1])
    one = P.Linear(inputs=K, outputs=N, max_rows=rows, dtype=P.BF16, weight_dtype=P.BF16, cuda_stream=stream())
    alone = torch.zeros((rows, N), dtype=torch.bfloat16, device="cuda")
    for m in range(W):
        part = slice(m * rows, (m + 1) * rows)
        one.forward(rows, x[part], K, w[m], 0, None, 0, None, 0, alone, N)
        zero = torch.zeros(N, dtype=torch.float64, device="cuda")
        want, _, e, _ = linear_forward(x[part].double(), w[m].double().view(N, K), zero, zero, 0, 1, 1)
        within(alone, want, e, "one worker")
        within(y[0][part], want, e, "the same among three")
    op.destroy()
    one.destroy()


def test_backward_of_shared_weights_keeps_gradients_apart(P):  # noqa: F811
    W, rows, K, N = 4, 50, 40, 24
    x = torch.randn((W * rows, K), generator=gen(1), device="cuda")
    w = torch.randn((N, K), generator=gen(2), device="cuda")
    dy = torch.randn((W * rows, N), generator=gen(3), device="cuda")
    op = P.Linear(inputs=K, outputs=N, max_rows=rows, workers=W, cuda_stream=stream())
    dx, g = torch.zeros_like(x), torch.zeros((W, N * K), device="cuda")
    op.backward(rows, dy, N, x, K, w, 0, None, 0, dx, K, g, None, N * K)
    for m in range(W):
        part = slice(m * rows, (m + 1) * rows)
        want, dw, _, e_dx, e_dw, _ = linear_backward(dy[part].double(), x[part].double(), w.double(),
                                                     torch.zeros_like(dy[part]).double(), 0, 0, 0)
        within(dx[part], want, e_dx, "dx")
        within(g[m].view(N, K), dw, e_dw, "dweight")
    op.destroy()
