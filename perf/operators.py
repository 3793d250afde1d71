"""The operators a token model's workers run before the compressed step, and how long each takes.

A worker of Algorithm 2 needs its gradient row before it can compress it.  For a model over tokens
the memory-bound ends of that gradient are the embedding lookup and its gradient, layer norm and its
gradient, and the loss: here distillation from a teacher's top logits.  All of them are batched over
the workers, each with its own parameters (or shared ones) and its own gradient row.

`run` computes an operator from elementary torch operations in 32 bits, rounded once at the end, or
(where `own` is true) through the package's operators.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5


def _norm(name, way, workers, rows, width, **kw):
    """way: forward or backward.  pad: unused values between rows.  shared: one weight and bias for all workers."""
    case = dict(name=name, op="norm", way=way, workers=workers, rows=rows, width=width, dtype="bf16", pad=0, shared=False)
    case.update(kw)
    return case


def _embed(name, way, workers, tokens, vocab, width, **kw):
    """masked: share of the places that hold no token.  shared: one table for all workers."""
    case = dict(name=name, op="embed", way=way, workers=workers, tokens=tokens, vocab=vocab, width=width, dtype="bf16",
                table="f32", token_bits=32, pad=0, shared=False, masked=0.0)
    case.update(kw)
    return case


def _distill(name, way, rows, vocab, k, **kw):
    """way: forward, backward or step (both at once).  masked: share of the rows that do not count; with it some
    rows have fewer teacher entries and the vocabulary's last columns are padding.  given: the teacher's
    logsumexp over its whole vocabulary comes with its entries."""
    case = dict(name=name, op="distill", way=way, rows=rows, vocab=vocab, k=k, dtype="bf16", teacher="f32",
                temperature=1.0, pad=0, masked=0.0, given=False)
    case.update(kw)
    return case


def listed():
    return [
        # Four workers with a handful of rows each: launches and latency.
        _norm("norm_forward_few", "forward", 4, 4, 512),
        # One layer's activations of a small model, eight workers.
        _norm("norm_forward", "forward", 8, 2048, 1024),
        # The backward pass of a wide layer, weight and bias gradients of each worker.
        _norm("norm_backward_wide", "backward", 8, 2048, 4096),
        # Ragged: an odd width in 32 bits, rows that are not aligned, an odd number of workers.
        _norm("norm_backward_odd", "backward", 3, 777, 1537, dtype="f32", pad=3),
        # Every worker looks its batch up in its own parameters (its lookahead point).
        _embed("embed_forward", "forward", 8, 4096, 32000, 1024),
        # A small table, an odd width, masked places: latency of the sort.
        _embed("embed_backward_small", "backward", 2, 333, 1009, 129, dtype="f32", masked=0.1),
        # The same batch's gradient: most of a worker's gradient row is written, few of its rows are not zero.
        _embed("embed_backward", "backward", 8, 4096, 32000, 1024, masked=0.05),
        # One worker, long sequences, a large vocabulary: many tokens fall on few rows of the table.
        _embed("embed_backward_long", "backward", 1, 131072, 128000, 4096, token_bits=64),
        # A few rows of a small vocabulary: launches and latency.
        _distill("distill_step_few", "step", 4, 1000, 8),
        # A worker's batch.
        _distill("distill_step", "step", 4096, 32000, 64, temperature=2.0, masked=0.05),
        # A large vocabulary and a long batch.
        _distill("distill_step_large", "step", 8192, 128000, 128, teacher="bf16", temperature=2.0),
        # The gradient alone from a kept logsumexp, odd sizes in 32 bits.
        _distill("distill_backward_odd", "backward", 1023, 50001, 33, dtype="f32", pad=3, given=True),
    ]


def _log_uniform(rng, low, high):
    return int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))


def draw(rng):
    """Sizes over their whole range by their logarithm, odd ones among them, every direction and type."""
    dtype = rng.choice(("bf16", "bf16", "f32", "f16"))
    pad = rng.choice((0, 0, 0, 8, 3))
    op = rng.choice(("norm", "embed", "distill"))
    workers = rng.choice((1, 1, 2, 3, 4, 8, 16))
    even = rng.choice((1, 1, 8, 64))  # widths as models have them, or any
    size = SIZES[dtype]
    if op == "norm":
        width = -(-_log_uniform(rng, 32, 16384) // even) * even
        rows = _log_uniform(rng, 1, max(1, min(65536, 64 * 2 ** 20 * 2 // (size * workers * width))))
        case = _norm("", rng.choice(("forward", "backward")), workers, rows, width, dtype=dtype, pad=pad,
                     shared=rng.random() < 0.3)
    elif op == "embed":
        vocab = _log_uniform(rng, 100, 200_000)
        width = -(-_log_uniform(rng, 16, max(16, min(8192, 400_000_000 // (workers * vocab)))) // even) * even
        tokens = _log_uniform(rng, 1, max(1, min(200_000, 1_000_000_000 // (size * workers * width))))
        case = _embed("", rng.choice(("forward", "backward", "backward")), workers, tokens, vocab, width, dtype=dtype,
                      table=rng.choice(("f32", "f32", "bf16", "f16")), token_bits=rng.choice((32, 64)), pad=pad,
                      shared=rng.random() < 0.3, masked=rng.choice((0.0, 0.05, 0.3)))
    else:
        vocab = _log_uniform(rng, 64, 200_000)
        rows = _log_uniform(rng, 1, max(1, min(16384, 2_000_000_000 // (size * vocab))))
        case = _distill("", rng.choice(("forward", "backward", "step", "step")), rows, vocab,
                        _log_uniform(rng, 1, min(256, vocab // 2)), dtype=dtype, teacher=rng.choice(("f32", "bf16", "f16")),
                        temperature=rng.choice((1.0, 2.0, 0.7)), pad=pad, masked=rng.choice((0.0, 0.05, 0.3)),
                        given=rng.random() < 0.3)
    del case["name"]
    return case


def _generator(seed, *which):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(random.Random("%d %s" % (seed, which)).getrandbits(60))
    return gen


def _normal(shape, gen):
    return torch.randn(shape, generator=gen, device="cuda")


def _rows(values, pad, dtype):
    """The values as rows of `dtype`, `pad` unused values after each: a view of the rows."""
    out = torch.zeros((values.shape[0], values.shape[1] + pad), dtype=DTYPES[dtype], device="cuda")
    out[:, :values.shape[1]] = values
    return out[:, :values.shape[1]]


def _empty_rows(rows, width, pad, dtype):
    return torch.zeros((rows, width + pad), dtype=DTYPES[dtype], device="cuda")[:, :width]


def _norm_inputs(case, seed):
    """Activations with a few large channels and a mean of their own in each row; the weights and biases of the
    workers side by side in their parameter vectors; output gradients; the forward pass's statistics."""
    W, R, C = case["workers"], case["rows"], case["width"]
    gen = _generator(seed, "norm")
    x = _normal((W * R, C), gen)
    x *= torch.exp(0.5 * _normal((C,), gen))
    x += 0.3 * _normal((W * R, 1), gen)
    stride = (2 * C + 3) // 4 * 4
    params = 0.1 * _normal((1 if case["shared"] else W, stride), gen)
    params[:, :C] += 1
    state = dict(x=_rows(x, case["pad"], case["dtype"]), params=params)
    if case["way"] == "backward":
        state["dy"] = _rows(1e-3 * _normal((W * R, C), gen), case["pad"], case["dtype"])
        x = state["x"].double()
        mean = x.mean(1)
        state["mean"] = mean.float()
        state["rstd"] = (x.sub_(mean[:, None]).square_().mean(1) + EPS).rsqrt_().float()
    return state


def _shares(vocab):
    """How often each token comes, most frequent first, as in text: 1 / (rank + 2.7)."""
    p = 1.0 / (np.arange(vocab) + 2.7)
    return p / p.sum()


def _embed_inputs(case, seed):
    W, n, V, C = case["workers"], case["tokens"], case["vocab"], case["width"]
    gen = _generator(seed, "embed")
    ends = torch.from_numpy(np.cumsum(_shares(V))).cuda()
    rank = torch.searchsorted(ends, torch.rand((W, n), generator=gen, device="cuda", dtype=torch.float64))
    tokens = torch.randperm(V, generator=gen, device="cuda")[rank.clamp_(max=V - 1)]
    tokens[torch.rand((W, n), generator=gen, device="cuda") < case["masked"]] = -1
    state = dict(tokens=tokens.to(torch.int32 if case["token_bits"] == 32 else torch.int64))
    if case["way"] == "forward":
        table = torch.empty((1 if case["shared"] else W, V * C), dtype=DTYPES[case["table"]], device="cuda")
        for row in table:
            row.copy_(0.02 * _normal((V * C,), gen))
        state["table"] = table
    else:
        state["dy"] = _rows(1e-3 * _normal((W * n, C), gen), case["pad"], case["dtype"])
    return state


def _distill_inputs(case, seed):
    """Student logits that follow the teacher's entries in part."""
    R, V, K, T = case["rows"], case["vocab"], case["k"], case["temperature"]
    gen = _generator(seed, "distill")
    live = V - V // 50 if case["masked"] else V
    step = torch.randint(1, live // K + 1, (R, 1), generator=gen, device="cuda")
    start = torch.randint(0, live, (R, 1), generator=gen, device="cuda")
    ids = (start + step * torch.arange(K, device="cuda")) % live
    values = (6 + 2 * _normal((R, K), gen)).sort(1, descending=True).values.to(DTYPES[case["teacher"]])
    logits = _empty_rows(R, V, case["pad"], case["dtype"])
    chunk = max(1, 2 ** 28 // V)
    for at in range(0, R, chunk):
        z = 2 * _normal((min(chunk, R - at), V), gen)
        if live < V:
            z[:, live:] = -math.inf
        logits[at:at + chunk] = z.scatter_add_(1, ids[at:at + chunk], 0.7 * values[at:at + chunk].float())
    ids = ids.to(torch.int32)
    weights = torch.ones(R, device="cuda")
    if case["masked"]:
        count = torch.randint(0, 4 * K, (R, 1), generator=gen, device="cuda")  # a quarter of the rows have fewer than K
        ids[torch.arange(K, device="cuda") >= count] = -1
        weights = 0.5 + torch.rand(R, generator=gen, device="cuda")
        weights[torch.rand(R, generator=gen, device="cuda") < case["masked"]] = 0
    state = dict(logits=logits, ids=ids, values=values, weights=weights, scale=1.0 / R, teacher_lse=None)
    if case["given"]:
        t = torch.where(ids >= 0, values.double() / T, -math.inf)
        t = torch.cat([t, torch.zeros((R, 1), dtype=t.dtype, device="cuda")], 1)
        state["teacher_lse"] = torch.logsumexp(t, 1).float()
    if case["way"] == "backward":
        lse = torch.empty(R, device="cuda")
        for at in range(0, R, chunk):
            lse[at:at + chunk] = torch.logsumexp(logits[at:at + chunk].double() / T, 1).float()
        state["lse"] = torch.where((weights != 0) & (ids >= 0).any(1), lse, 0)
    return state


INPUTS = {"norm": _norm_inputs, "embed": _embed_inputs, "distill": _distill_inputs}


def _operator(case):
    """The package's operator, as a training program makes it once."""
    import paper_2010_13359_gb300 as P

    types = {"f32": P.F32, "bf16": P.BF16, "f16": P.F16}
    stream = torch.cuda.current_stream().cuda_stream
    if case["op"] == "norm":
        return P.LayerNorm(width=case["width"], workers=case["workers"], dtype=types[case["dtype"]], eps=EPS,
                           cuda_stream=stream)
    if case["op"] == "embed":
        return P.Embedding(vocab=case["vocab"], width=case["width"], workers=case["workers"], max_tokens=case["tokens"],
                           table_dtype=types[case["table"]], dtype=types[case["dtype"]], token_bits=case["token_bits"],
                           scale=math.sqrt(case["width"]), cuda_stream=stream)
    return P.Distillation(vocab=case["vocab"], k=case["k"], dtype=types[case["dtype"]],
                          teacher_dtype=types[case["teacher"]], temperature=case["temperature"], cuda_stream=stream)


def prepare(case, seed):
    """The inputs, the buffers of the outputs and the operator."""
    state = INPUTS[case["op"]](case, seed) | dict(case=case)
    if case["op"] == "norm":
        W, R, C = case["workers"], case["rows"], case["width"]
        state["out"] = _empty_rows(W * R, C, case["pad"], case["dtype"])
        if case["way"] == "forward":
            state["mean"], state["rstd"] = torch.zeros((2, W * R), device="cuda")
        else:
            state["g"] = torch.zeros((W, (2 * C + 3) // 4 * 4), device="cuda")
    elif case["op"] == "embed":
        W, n, V, C = case["workers"], case["tokens"], case["vocab"], case["width"]
        if case["way"] == "forward":
            state["out"] = _empty_rows(W * n, C, case["pad"], case["dtype"])
        else:
            state["g"] = torch.zeros((W, (V * C + 3) // 4 * 4), device="cuda")
    else:
        R, V = case["rows"], case["vocab"]
        if case["way"] != "forward":
            state["out"] = _empty_rows(R, V, case["pad"], case["dtype"])
        if case["way"] != "backward":
            state["loss"], state["lse"] = torch.zeros((2, R), device="cuda")
    if own:
        state["operator"] = _operator(case)
    return state


def _plain_norm(state):
    case = state["case"]
    W, R, C = case["workers"], case["rows"], case["width"]
    weight, bias = state["params"][:, None, :C], state["params"][:, None, C:2 * C]
    x = state["x"].float().view(W, R, C)
    if case["way"] == "forward":
        mean = x.sum(2, keepdim=True) / C
        d = x - mean
        rstd = ((d * d).sum(2, keepdim=True) / C + EPS).rsqrt()
        y = d * rstd * weight + bias
        return {"y": y.view(W * R, C).to(state["x"].dtype), "mean": mean.view(-1), "rstd": rstd.view(-1)}
    rstd = state["rstd"].view(W, R, 1)
    normal = (x - state["mean"].view(W, R, 1)) * rstd
    dy = state["dy"].float().view(W, R, C)
    a = dy * weight
    c1 = a.sum(2, keepdim=True) / C
    c2 = (a * normal).sum(2, keepdim=True) / C
    dx = rstd * (a - c1 - normal * c2)
    return {"dx": dx.view(W * R, C).to(state["x"].dtype), "dweight": (dy * normal).sum(1), "dbias": dy.sum(1)}


def _own_norm(state):
    case, op, params, out = state["case"], state["operator"], state["params"], state["out"]
    R, C, x = case["rows"], case["width"], state["x"]
    stride = 0 if case["shared"] else params.stride(0)
    if case["way"] == "forward":
        op.forward(R, x, x.stride(0), params, params[:, C:], stride, out, out.stride(0), state["mean"], state["rstd"])
        return {"y": out, "mean": state["mean"], "rstd": state["rstd"]}
    g, dy = state["g"], state["dy"]
    op.backward(R, dy, dy.stride(0), x, x.stride(0), params, stride, state["mean"], state["rstd"], out, out.stride(0),
                g, g[:, C:], g.stride(0))
    return {"dx": out, "dweight": g[:, :C], "dbias": g[:, C:2 * C]}


def _plain_embed(state):
    case, tokens = state["case"], state["tokens"].long()
    W, n, V, C = case["workers"], case["tokens"], case["vocab"], case["width"]
    scale = math.sqrt(C)
    counts = (tokens >= 0) & (tokens < V)
    if case["way"] == "forward":
        at = tokens.clamp(0, V - 1) + (0 if case["shared"] else V * torch.arange(W, device="cuda")[:, None])
        y = state["table"].view(-1, C)[at.view(-1)].float() * scale
        return {"y": torch.where(counts.view(-1, 1), y, 0).to(DTYPES[case["dtype"]])}
    at = (tokens + V * torch.arange(W, device="cuda")[:, None])[counts]
    g = torch.zeros((W * V, C), device="cuda").index_add_(0, at, state["dy"][counts.view(-1)].float())
    return {"dtable": (g * scale).view(W, V * C)}


def _own_embed(state):
    case, op, tokens = state["case"], state["operator"], state["tokens"]
    if case["way"] == "forward":
        table, out = state["table"], state["out"]
        op.forward(case["tokens"], tokens, table, 0 if case["shared"] else table.stride(0), out, out.stride(0))
        return {"y": out}
    g, dy = state["g"], state["dy"]
    op.backward(case["tokens"], tokens, dy, dy.stride(0), g, g.stride(0))
    return {"dtable": g[:, :case["vocab"] * case["width"]]}


def _plain_distill(state):
    case, weights = state["case"], state["weights"]
    V, T = case["vocab"], case["temperature"]
    ids = state["ids"].long()
    counts = (ids >= 0) & (ids < V)
    left_out = (weights == 0) | ~counts.any(1)
    t = torch.where(counts, state["values"].float() / T, -math.inf)
    if state["teacher_lse"] is None:
        most = torch.where(counts.any(1), t.amax(1), 0)[:, None]
        lse_t = most + (t - most).exp().sum(1, keepdim=True).log()
    else:
        lse_t = state["teacher_lse"][:, None]
    p = torch.where(counts & ~left_out[:, None], (t - lse_t).exp(), 0)
    z = state["logits"].float() / T
    if case["way"] == "backward":
        lse = state["lse"][:, None]
    else:
        most = z.amax(1, keepdim=True)
        lse = most + (z - most).exp().sum(1, keepdim=True).log()
    out = {}
    if case["way"] != "backward":
        terms = p * ((t - lse_t) - (z.gather(1, ids.clamp(0, V - 1)) - lse))
        loss = weights * T * T * torch.where(p > 0, terms, 0).sum(1)
        out = {"loss": torch.where(left_out, 0, loss), "lse": torch.where(left_out, 0, lse[:, 0])}
    if case["way"] != "forward":
        dz = (z - lse).exp() * p.sum(1, keepdim=True)
        dz.scatter_add_(1, ids.clamp(0, V - 1), -p)
        dz *= (state["scale"] * T * weights)[:, None]
        out["dlogits"] = torch.where(left_out[:, None], 0, dz).to(state["logits"].dtype)
    return out


def _own_distill(state):
    case, op, z = state["case"], state["operator"], state["logits"]
    teacher = (state["ids"], state["values"], state["ids"].stride(0), state["teacher_lse"], state["weights"])
    if case["way"] == "forward":
        op.forward(case["rows"], z, z.stride(0), *teacher, state["loss"], state["lse"])
        return {"loss": state["loss"], "lse": state["lse"]}
    out = state["out"]
    if case["way"] == "backward":
        op.backward(case["rows"], z, z.stride(0), state["lse"], *teacher, state["scale"], out, out.stride(0))
        return {"dlogits": out}
    op.step(case["rows"], z, z.stride(0), *teacher, state["scale"], state["loss"], state["lse"], out, out.stride(0))
    return {"loss": state["loss"], "lse": state["lse"], "dlogits": out}


PLAIN = {"norm": _plain_norm, "embed": _plain_embed, "distill": _plain_distill}
OWN = {"norm": _own_norm, "embed": _own_embed, "distill": _own_distill}


def run(state):
    return (OWN if own else PLAIN)[state["case"]["op"]](state)


def work(case):
    """Each input read once, each output written once.  Of a table only the rows that are looked up, as often as
    the tokens' shares say; of the logits only the rows that count."""
    size = SIZES[case["dtype"]]
    if case["op"] == "norm":
        W, R, C = case["workers"], case["rows"], case["width"]
        params = (1 if case["shared"] else W) * C * 4
        if case["way"] == "forward":
            return {"bytes": 2 * W * R * C * size + 8 * W * R + 2 * params, "flops": 8 * W * R * C}
        return {"bytes": 3 * W * R * C * size + 8 * W * R + params + 8 * W * C, "flops": 14 * W * R * C}
    if case["op"] == "embed":
        W, n, V, C = case["workers"], case["tokens"], case["vocab"], case["width"]
        total = W * n * case["token_bits"] // 8
        live = int(W * n * (1 - case["masked"]))
        if case["way"] == "backward":
            return {"bytes": total + live * C * size + W * V * C * 4, "flops": live * C}
        tables = 1 if case["shared"] else W
        looked_up = tables * float((1 - (1 - _shares(V)) ** (live / tables)).sum())
        return {"bytes": int(total + looked_up * C * SIZES[case["table"]] + W * n * C * size), "flops": live * C}
    R, V, K = case["rows"], case["vocab"], case["k"]
    live = R * (1 - case["masked"])
    total = live * V * size + R * K * (4 + SIZES[case["teacher"]]) + (4 if case["given"] else 0) * R + 4 * R
    total += {"forward": 8 * R, "backward": 4 * R + R * V * size, "step": 8 * R + R * V * size}[case["way"]]
    return {"bytes": int(total), "flops": int(live * V * {"forward": 5, "backward": 4, "step": 9}[case["way"]])}


def exact(case, seed):
    """The definitions in 64 bits."""
    return {"norm": _exact_norm, "embed": _exact_embed, "distill": _exact_distill}[case["op"]](case, seed)


def _exact_norm(case, seed):
    s = _norm_inputs(case, seed)
    W, R, C = case["workers"], case["rows"], case["width"]
    params = s["params"].double().expand(W, -1)
    out = {}
    for m in range(W):
        x = s["x"][m * R:(m + 1) * R].double()
        gamma, beta = params[m, :C], params[m, C:2 * C]
        if case["way"] == "forward":
            var, mean = torch.var_mean(x, 1, correction=0)
            rstd = 1 / torch.sqrt(var + EPS)
            part = {"y": (x - mean[:, None]) / torch.sqrt(var + EPS)[:, None] * gamma + beta, "mean": mean, "rstd": rstd}
        else:
            # the definition's own derivative, at the statistics that the call is given
            mean, rstd = s["mean"][m * R:(m + 1) * R].double(), s["rstd"][m * R:(m + 1) * R].double()
            h = (x - mean[:, None]) * rstd[:, None]
            dy = s["dy"][m * R:(m + 1) * R].double()
            inner = dy * gamma
            dx = (inner - inner.mean(1, keepdim=True) - h * (inner * h).mean(1, keepdim=True)) * rstd[:, None]
            part = {"dx": dx, "dweight": torch.einsum("rc,rc->c", dy, h)[None], "dbias": dy.sum(0)[None]}
        for key, value in part.items():
            out.setdefault(key, []).append(value)
    return {key: torch.cat(values) for key, values in out.items()}


def _exact_embed(case, seed):
    s = _embed_inputs(case, seed)
    W, n, V, C = case["workers"], case["tokens"], case["vocab"], case["width"]
    scale = math.sqrt(C)
    if case["way"] == "forward":
        y = torch.zeros((W, n, C), dtype=torch.float64, device="cuda")
        for m in range(W):
            live = s["tokens"][m] >= 0
            y[m, live] = scale * s["table"][0 if case["shared"] else m].view(V, C)[s["tokens"][m][live].long()].double()
        return {"y": y.view(W * n, C)}
    out = torch.zeros((W, V, C), dtype=torch.float64, device="cuda")
    for m in range(W):
        token, order = s["tokens"][m].long().sort()
        order = order[token >= 0]
        token = token[token >= 0]
        step = max(1, 2 ** 24 // C)
        for at in range(0, len(order), step):
            dy = s["dy"][m * n:(m + 1) * n][order[at:at + step]].double() * scale
            out[m].index_add_(0, token[at:at + step], dy)
    return {"dtable": out.view(W, V * C)}


def _exact_distill(case, seed):
    s = _distill_inputs(case, seed)
    R, V, K, T = case["rows"], case["vocab"], case["k"], case["temperature"]
    loss, lse = torch.zeros((2, R), dtype=torch.float64, device="cuda")
    dlogits = torch.zeros((R, V), dtype=torch.float64, device="cuda") if case["way"] != "forward" else None
    step = max(1, 2 ** 27 // V)
    for at in range(0, R, step):
        rows = slice(at, at + step)
        ids, w = s["ids"][rows].long(), s["weights"][rows].double()
        there = ids >= 0
        t = s["values"][rows].double() / T
        t[~there] = -math.inf
        lt = torch.logsumexp(t, 1) if s["teacher_lse"] is None else s["teacher_lse"][rows].double()
        counts = (w != 0) & there.any(1)
        logp = t - lt[:, None]
        p = torch.exp(logp).masked_fill(~there | ~counts[:, None], 0)
        z = s["logits"][rows].double() / T
        mine = torch.logsumexp(z, 1) if case["way"] != "backward" else s["lse"][rows].double()
        logq = z - mine[:, None]
        at_ids = logq.gather(1, ids.clamp(min=0))
        terms = torch.where(p > 0, p * (logp - at_ids), torch.zeros_like(p))
        loss[rows] = T ** 2 * w * terms.sum(1)
        lse[rows] = torch.where(counts, mine, torch.zeros_like(mine))
        if dlogits is not None:
            q = torch.exp(logq) * p.sum(1, keepdim=True)
            q -= torch.zeros_like(q).scatter_add_(1, ids.clamp(min=0), p)
            dlogits[rows] = (q * (s["scale"] * T * w)[:, None]).masked_fill(~counts[:, None], 0)
    out = {"loss": loss, "lse": lse} if case["way"] != "backward" else {}
    return out | ({"dlogits": dlogits} if dlogits is not None else {})
