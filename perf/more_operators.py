"""The rest of a token model's worker gradient, and how long each part takes: the layers' matrix products with
bias, activation and residual, the cross entropy of the output layer without its logits, and the clipping of the
workers' gradients on their way into the rows that the compressed step reads.

All of them are batched over the workers of Algorithm 2, each with its own parameters (or shared ones) and its own
gradient row.  `run` computes an operator from elementary torch operations in 32 bits, rounded once at the end, or
(where `own` is true) through the package's operators.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6


def _linear(name, way, workers, rows, inputs, outputs, **kw):
    """way: forward or backward.  weight: the weights' type.  pad: unused values between rows.  shared: one weight
    and bias for all workers.  residual: added after the activation (forward)."""
    case = dict(name=name, op="linear", way=way, workers=workers, rows=rows, inputs=inputs, outputs=outputs, dtype="bf16",
                weight="bf16", activation="none", residual=False, pad=0, shared=False)
    case.update(kw)
    return case


def _loss(name, way, workers, rows, vocab, width, **kw):
    """way: forward, backward or step (both at once).  masked: share of the rows without a target."""
    case = dict(name=name, op="loss", way=way, workers=workers, rows=rows, vocab=vocab, width=width, dtype="bf16",
                weight="bf16", token_bits=32, masked=0.0, pad=0, shared=False)
    case.update(kw)
    return case


def _clip(name, way, workers, layers, width, vocab, **kw):
    """way: clip, or norm alone.  The gradients of a model of `layers` layers of `width`: an embedding of `vocab` rows,
    two norms, two products with their biases each.  pad: unused values between workers."""
    case = dict(name=name, op="clip", way=way, workers=workers, layers=layers, width=width, vocab=vocab, dtype="f32",
                pad=0, max_norm=1.0)
    case.update(kw)
    return case


def listed():
    return [
        # Four workers with a handful of rows each: launches and latency.
        _linear("linear_few", "forward", 4, 4, 512, 512, activation="gelu"),
        # One token through a wide layer: its weights are read once.
        _linear("linear_token", "forward", 1, 1, 4096, 4096, residual=True),
        # The widening product of a layer, eight workers, weights as the lookahead point holds them.
        _linear("linear_forward", "forward", 8, 2048, 1024, 4096, weight="f32", activation="gelu"),
        # Its gradient.
        _linear("linear_backward", "backward", 8, 2048, 1024, 4096, activation="gelu"),
        # A wide layer's gradient without an activation, one worker with long sequences.
        _linear("linear_backward_wide", "backward", 1, 16384, 4096, 4096),
        # Ragged: odd widths in 32 bits, rows that are not aligned, an odd number of workers.
        _linear("linear_backward_odd", "backward", 3, 777, 515, 1031, dtype="f32", weight="f32", activation="relu", pad=3),
        # A worker's batch, and a small vocabulary in 32 bits with odd sizes.
        _loss("loss_step", "step", 4, 1024, 32000, 1024, masked=0.05),
        _loss("loss_forward_odd", "forward", 2, 333, 5003, 129, dtype="f32", weight="f32", token_bits=64, pad=1),
        # A large vocabulary and long sequences.
        _loss("loss_step_large", "step", 1, 4096, 128000, 2048),
        # A small model's tensors: launches and latency.
        _clip("clip_few", "clip", 2, 2, 64, 500, max_norm=0.01),
        # Eight workers' gradients of a model of 33.6 million parameters.
        _clip("clip_model", "clip", 8, 4, 640, 32000, max_norm=0.1),
        # One worker's bf16 gradients of 720 million parameters in 303 tensors, from odd places.
        _clip("clip_many", "clip", 1, 50, 1280, 50000, dtype="bf16", pad=1),
    ]


def _log_uniform(rng, low, high):
    return int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))


def draw(rng):
    """Sizes over their whole range by their logarithm, odd ones among them, every direction and type."""
    dtype = rng.choice(("bf16", "bf16", "f32", "f16"))
    weight = rng.choice((dtype, "f32"))
    pad = rng.choice((0, 0, 0, 8, 3))
    op = rng.choice(("linear", "loss", "clip"))
    workers = rng.choice((1, 1, 2, 3, 4, 8, 16))
    even = rng.choice((1, 8, 64))  # widths as models have them, or any
    shared = rng.random() < 0.3

    def width(low, high):
        return -(-_log_uniform(rng, low, high) // even) * even

    if op == "linear":
        inputs, outputs = width(16, 8192), width(16, 8192)
        most = min(32768, 400_000_000_000 // (workers * inputs * outputs))
        case = _linear("", rng.choice(("forward", "backward")), workers, _log_uniform(rng, 1, max(1, most)), inputs, outputs,
                       dtype=dtype, weight=weight, activation=rng.choice(("none", "relu", "gelu", "silu")),
                       residual=rng.random() < 0.5, pad=pad, shared=shared)
        case["residual"] = case["residual"] and case["way"] == "forward"
    elif op == "loss":
        columns = width(16, 4096)
        vocab = _log_uniform(rng, 64, min(200_000, 600_000_000 // (workers * columns)))
        most = min(8192, 300_000_000_000 // (workers * columns * vocab))
        case = _loss("", rng.choice(("forward", "backward", "step", "step")), workers, _log_uniform(rng, 1, max(1, most)),
                     vocab, columns, dtype=dtype, weight=weight, token_bits=rng.choice((32, 64)),
                     masked=rng.choice((0.0, 0.05, 0.3)), pad=pad, shared=shared)
    else:
        columns = width(16, 2048)
        layers = _log_uniform(rng, 1, 60)
        layers = min(layers, max(1, 500_000_000 // (8 * workers * columns * columns)))
        vocab = _log_uniform(rng, 100, max(100, min(200_000, 200_000_000 // (workers * columns))))
        case = _clip("", rng.choice(("clip", "clip", "norm")), workers, layers, columns, vocab, dtype=dtype, pad=pad,
                     max_norm=rng.choice((0.01, 0.1, 1.0)))
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


def _linear_inputs(case, seed):
    """Activations with a few large channels; the workers' weights and biases side by side in their parameter vectors,
    the weights in a copy of their type where that is not the parameters'; output gradients."""
    W, R, K, N = case["workers"], case["rows"], case["inputs"], case["outputs"]
    gen = _generator(seed, "linear")
    x = _normal((W * R, K), gen) * torch.exp(0.5 * _normal((K,), gen))
    held = 1 if case["shared"] else W
    params = torch.zeros((held, (N * K + N + 3) // 4 * 4), device="cuda")
    params[:, :N * K] = _normal((held, N * K), gen) / math.sqrt(K)
    params[:, N * K:N * K + N] = 0.1 * _normal((held, N), gen)
    weight = params if case["weight"] == "f32" else _rows(params[:, :N * K], 0, case["weight"])
    state = dict(x=_rows(x, case["pad"], case["dtype"]), params=params, weight=weight, pre=None, residual=None)
    if case["residual"]:
        state["residual"] = _rows(_normal((W * R, N), gen), case["pad"], case["dtype"])
    if case["way"] == "backward":
        state["dy"] = _rows(1e-3 * _normal((W * R, N), gen), case["pad"], case["dtype"])
        if case["activation"] != "none":
            state["pre"] = _rows(_normal((W * R, N), gen), case["pad"], case["dtype"])
    return state


def _loss_inputs(case, seed):
    """Rows that lean towards their target's row of the output layer, as those of a model in training."""
    W, R, V, C = case["workers"], case["rows"], case["vocab"], case["width"]
    gen = _generator(seed, "loss")
    held = 1 if case["shared"] else W
    weight = torch.empty((held, (V * C + 3) // 4 * 4), dtype=DTYPES[case["weight"]], device="cuda")
    for row in weight:
        row.copy_(1.5 / math.sqrt(C) * _normal((weight.shape[1],), gen))
    targets = torch.randint(0, V, (W, R), generator=gen, device="cuda")
    at = targets + (0 if case["shared"] else V * torch.arange(W, device="cuda")[:, None])
    table = weight[:, :V * C].reshape(-1, C)
    x = _normal((W * R, C), gen) + 2 * table[at.view(-1)].float()
    targets[torch.rand((W, R), generator=gen, device="cuda") < case["masked"]] = -1
    weights = torch.ones(W * R, device="cuda")
    if case["masked"]:
        weights = 0.5 + torch.rand(W * R, generator=gen, device="cuda")
    scale = (1024.0 if case["dtype"] == "f16" else 1.0) / R  # f16 gradients are scaled up, or they would vanish
    state = dict(x=_rows(x, case["pad"], case["dtype"]), weight=weight, weights=weights, scale=scale,
                 targets=targets.to(torch.int32 if case["token_bits"] == 32 else torch.int64))
    if case["way"] == "backward":
        lse = torch.empty((W, R), device="cuda")
        step = max(1, 2 ** 28 // V)
        for m in range(W):
            table = weight[0 if case["shared"] else m, :V * C].view(V, C).float()
            for at in range(0, R, step):
                rows = state["x"][m * R + at:m * R + min(R, at + step)].float()
                lse[m, at:at + step] = torch.logsumexp((rows @ table.t()).double(), 1).float()
        state["lse"] = torch.where(targets >= 0, lse, 0).view(-1)
    return state


def _sizes(case):
    """The sizes of the model's tensors in the order of its parameters."""
    C = case["width"]
    layer = [C, C, 4 * C * C, 4 * C, 4 * C * C, C]
    return [case["vocab"] * C] + case["layers"] * layer + [C, C]


def _clip_inputs(case, seed):
    """Each tensor's gradients of all workers, `pad` unused values after each worker's, the layers' of different size."""
    gen = _generator(seed, "clip")
    tensors = []
    for n in _sizes(case):
        size = 1e-4 * math.exp(random.Random(n + seed).uniform(-1, 1))
        buffer = torch.zeros((case["workers"], n + case["pad"]), dtype=DTYPES[case["dtype"]], device="cuda")
        for row in buffer:
            row[:n] = size * _normal((n,), gen)
        tensors.append(buffer[:, :n])
    return dict(tensors=tensors)


INPUTS = {"linear": _linear_inputs, "loss": _loss_inputs, "clip": _clip_inputs}


def _operator(case):
    """The package's operator, as a training program makes it once."""
    import paper_2010_13359_gb300 as P

    types = {"f32": P.F32, "bf16": P.BF16, "f16": P.F16}
    stream = torch.cuda.current_stream().cuda_stream
    dtype = types[case["dtype"]]
    if case["op"] == "linear":
        activations = {"none": P.NONE, "relu": P.RELU, "gelu": P.GELU, "silu": P.SILU}
        return P.Linear(inputs=case["inputs"], outputs=case["outputs"], max_rows=case["rows"], workers=case["workers"],
                        dtype=dtype, weight_dtype=types[case["weight"]], activation=activations[case["activation"]],
                        cuda_stream=stream)
    if case["op"] == "loss":
        return P.TokenLoss(vocab=case["vocab"], width=case["width"], max_rows=case["rows"], workers=case["workers"],
                           dtype=dtype, weight_dtype=types[case["weight"]], token_bits=case["token_bits"],
                           cuda_stream=stream)
    return P.GradientClip(workers=case["workers"], dtype=dtype, out_dtype=P.F32, eps=EPS, cuda_stream=stream)


def prepare(case, seed):
    """The inputs, the buffers of the outputs and the operator."""
    state = INPUTS[case["op"]](case, seed) | dict(case=case)
    if case["op"] == "linear":
        W, R, K, N = case["workers"], case["rows"], case["inputs"], case["outputs"]
        if case["way"] == "forward":
            state["out"] = _empty_rows(W * R, N, case["pad"], case["dtype"])
            if case["activation"] != "none":
                state["pre"] = _empty_rows(W * R, N, case["pad"], case["dtype"])
        else:
            state["out"] = _empty_rows(W * R, K, case["pad"], case["dtype"])
            state["g"] = torch.zeros((W, (N * K + N + 3) // 4 * 4), device="cuda")
    elif case["op"] == "loss":
        W, R, V, C = case["workers"], case["rows"], case["vocab"], case["width"]
        if case["way"] != "forward":
            state["out"] = _empty_rows(W * R, C, case["pad"], case["dtype"])
            state["g"] = torch.zeros((W, (V * C + 3) // 4 * 4), device="cuda")
        if case["way"] != "backward":
            state["loss"], state["lse"] = torch.zeros((2, W * R), device="cuda")
    else:
        state["norms"] = torch.zeros(case["workers"], device="cuda")
        if case["way"] == "clip":
            state["g"] = torch.zeros((case["workers"], (sum(_sizes(case)) + 3) // 4 * 4), device="cuda")
    if own:
        state["operator"] = _operator(case)
        if case["op"] == "clip":
            state |= _lists(case, state)
    return state


def _lists(case, state):
    """The tensors as the operator takes them: address, size and the workers' distance of each; and their places in the
    workers' gradient rows."""
    import paper_2010_13359_gb300 as P

    lists = {"from": P.TensorList([(t, t.shape[1], t.stride(0)) for t in state["tensors"]])}
    if case["way"] == "clip":
        g, at, places = state["g"], 0, []
        for t in state["tensors"]:
            places.append((g[:, at:], t.shape[1], g.stride(0)))
            at += t.shape[1]
        lists["to"] = P.TensorList(places)
    return lists


def _act(u, activation):
    if activation == "none":
        return u
    if activation == "relu":
        return torch.where(u > 0, u, 0)
    if activation == "gelu":
        return 0.5 * u * (1 + torch.erf(u * math.sqrt(0.5)))
    return u / (1 + torch.exp(-u))


def _act_slope(u, activation):
    if activation == "relu":
        return (u > 0).to(u.dtype)
    if activation == "gelu":
        return 0.5 * (1 + torch.erf(u * math.sqrt(0.5))) + u * torch.exp(-0.5 * u * u) / math.sqrt(2 * math.pi)
    s = 1 / (1 + torch.exp(-u))
    return s * (1 + u * (1 - s))


def _plain_linear(state):
    case = state["case"]
    W, R, K, N = case["workers"], case["rows"], case["inputs"], case["outputs"]
    weight = state["weight"][:, :N * K].float().view(-1, N, K)
    bias = state["params"][:, None, N * K:N * K + N]
    x = state["x"].float().view(W, R, K)
    dtype = DTYPES[case["dtype"]]
    if case["way"] == "forward":
        u = torch.matmul(x, weight.transpose(1, 2)) + bias
        y = _act(u, case["activation"]).view(W * R, N)
        if state["residual"] is not None:
            y = y + state["residual"].float()
        out = {"y": y.to(dtype)}
        return out | ({"pre": u.view(W * R, N).to(dtype)} if state["pre"] is not None else {})
    du = state["dy"].float()
    if state["pre"] is not None:
        du = du * _act_slope(state["pre"].float(), case["activation"])
    du = du.view(W, R, N)
    dx = torch.matmul(du, weight).view(W * R, K).to(dtype)
    return {"dx": dx, "dweight": torch.matmul(du.transpose(1, 2), x).view(W, N * K), "dbias": du.sum(1)}


def _own_linear(state):
    case, op, x, out, pre = state["case"], state["operator"], state["x"], state["out"], state["pre"]
    R, K, N = case["rows"], case["inputs"], case["outputs"]
    weight, params, residual = state["weight"], state["params"], state["residual"]
    p_stride, b_stride = (0, 0) if case["shared"] else (weight.stride(0), params.stride(0))
    pre_stride = 0 if pre is None else pre.stride(0)
    if case["way"] == "forward":
        op.forward(R, x, x.stride(0), weight, p_stride, params[:, N * K:], b_stride, residual,
                   0 if residual is None else residual.stride(0), out, out.stride(0), pre, pre_stride)
        return {"y": out} | ({"pre": pre} if pre is not None else {})
    g, dy = state["g"], state["dy"]
    op.backward(R, dy, dy.stride(0), x, x.stride(0), weight, p_stride, pre, pre_stride, out, out.stride(0), g, g[:, N * K:],
                g.stride(0))
    return {"dx": out, "dweight": g[:, :N * K], "dbias": g[:, N * K:N * K + N]}


def _plain_loss(state):
    case = state["case"]
    W, R, V, C = case["workers"], case["rows"], case["vocab"], case["width"]
    weight = state["weight"][:, :V * C].float().view(-1, V, C)
    x = state["x"].float().view(W, R, C)
    targets = state["targets"].long().view(W, R, 1)
    counts = (targets >= 0) & (targets < V)
    c = torch.where(counts, state["weights"].view(W, R, 1), 0)
    z = torch.matmul(x, weight.transpose(1, 2))
    out = {}
    if case["way"] == "backward":
        lse = state["lse"].view(W, R, 1)
    else:
        most = z.amax(2, keepdim=True)
        lse = most + (z - most).exp().sum(2, keepdim=True).log()
        loss = c * (lse - z.gather(2, targets.clamp(0, V - 1)))
        out = {"loss": loss.view(-1), "lse": torch.where(counts, lse, 0).view(-1)}
    if case["way"] != "forward":
        dz = z.sub_(lse).exp_()
        dz.scatter_add_(2, targets.clamp(0, V - 1), -torch.ones_like(lse))
        dz = torch.where(counts, dz * (state["scale"] * c), 0)
        out["dx"] = torch.matmul(dz, weight).view(W * R, C).to(DTYPES[case["dtype"]])
        out["dweight"] = torch.matmul(dz.transpose(1, 2), x).view(W, V * C)
    return out


def _own_loss(state):
    case, op, x, weight = state["case"], state["operator"], state["x"], state["weight"]
    R, V, C = case["rows"], case["vocab"], case["width"]
    data = (R, x, x.stride(0), weight, 0 if case["shared"] else weight.stride(0), state["targets"], state["weights"])
    if case["way"] == "forward":
        op.forward(*data, state["loss"], state["lse"])
        return {"loss": state["loss"], "lse": state["lse"]}
    out, g = state["out"], state["g"]
    grads = {"dx": out, "dweight": g[:, :V * C]}
    if case["way"] == "backward":
        op.backward(*data, state["lse"], state["scale"], out, out.stride(0), g, g.stride(0))
        return grads
    op.step(*data, state["scale"], state["loss"], state["lse"], out, out.stride(0), g, g.stride(0))
    return {"loss": state["loss"], "lse": state["lse"]} | grads


def _plain_clip(state):
    case = state["case"]
    g = torch.cat(state["tensors"], 1).float()
    norms = g.square().sum(1, dtype=torch.float64).sqrt()
    if case["way"] == "norm":
        return {"norms": norms.float()}
    factor = (case["max_norm"] / (norms + EPS)).clamp(max=1).float()
    return {"norms": norms.float(), "g": g * factor[:, None]}


def _own_clip(state):
    case, op, norms = state["case"], state["operator"], state["norms"]
    if case["way"] == "norm":
        op.norm(state["from"], norms)
        return {"norms": norms}
    op.clip(state["from"], state["to"], case["max_norm"], norms)
    return {"norms": norms, "g": state["g"][:, :sum(t.shape[1] for t in state["tensors"])]}


PLAIN = {"linear": _plain_linear, "loss": _plain_loss, "clip": _plain_clip}
OWN = {"linear": _own_linear, "loss": _own_loss, "clip": _own_clip}


def run(state):
    return (OWN if own else PLAIN)[state["case"]["op"]](state)


def work(case):
    """Each input read once, each output written once, each product computed once (of the loss's gradient: the logits',
    the rows' gradient and the weights')."""
    size, W = SIZES[case["dtype"]], case["workers"]
    if case["op"] == "clip":
        n = W * sum(_sizes(case))
        return {"bytes": n * size + 4 * W + (4 * n if case["way"] == "clip" else 0),
                "flops": 2 * n + (n if case["way"] == "clip" else 0)}
    held = 1 if case["shared"] else W
    R = case["rows"]
    if case["op"] == "linear":
        K, N = case["inputs"], case["outputs"]
        total = W * R * K * size + held * N * K * SIZES[case["weight"]]
        acts = (case["activation"] != "none")
        if case["way"] == "forward":
            total += held * N * 4 + W * R * N * size * (1 + acts + case["residual"])
            return {"bytes": total, "flops": 2 * W * R * K * N}
        total += W * R * N * size * (1 + acts) + W * R * K * size + 4 * W * (N * K + N)
        return {"bytes": total, "flops": 4 * W * R * K * N}
    V, C = case["vocab"], case["width"]
    live = int(W * R * (1 - case["masked"]))
    total = live * C * size + held * V * C * SIZES[case["weight"]] + W * R * (4 + case["token_bits"] // 8)
    if case["way"] != "backward":
        total += 8 * W * R
    else:
        total += 4 * W * R
    if case["way"] != "forward":
        total += W * R * C * size + 4 * W * V * C
    return {"bytes": total, "flops": (2 if case["way"] == "forward" else 6) * live * V * C}


def exact(case, seed):
    """The definitions in 64 bits."""
    return {"linear": _exact_linear, "loss": _exact_loss, "clip": _exact_clip}[case["op"]](case, seed)


def _exact_act(u, activation):
    F = torch.nn.functional
    return {"none": lambda v: v, "relu": F.relu, "gelu": F.gelu, "silu": F.silu}[activation](u)


def _exact_linear(case, seed):
    s = _linear_inputs(case, seed)
    W, R, K, N = case["workers"], case["rows"], case["inputs"], case["outputs"]
    found = {}
    for m in range(W):
        held, rows = 0 if case["shared"] else m, slice(m * R, (m + 1) * R)
        weight = s["weight"][held, :N * K].double().view(N, K)
        x = s["x"][rows].double()
        if case["way"] == "forward":
            u = torch.addmm(s["params"][held, N * K:N * K + N].double(), x, weight.t())
            y = _exact_act(u, case["activation"])
            part = {"y": y if s["residual"] is None else y + s["residual"][rows].double()}
            if case["activation"] != "none":
                part["pre"] = u
        else:
            du = s["dy"][rows].double()
            if s["pre"] is not None:  # the derivative by automatic differentiation
                u = s["pre"][rows].double().requires_grad_()
                du, = torch.autograd.grad(_exact_act(u, case["activation"]), u, du)
            part = {"dx": du @ weight, "dweight": (du.t() @ x).view(1, N * K), "dbias": du.sum(0, keepdim=True)}
        for key, value in part.items():
            found.setdefault(key, []).append(value)
    return {key: torch.cat(values) for key, values in found.items()}


def _exact_loss(case, seed):
    s = _loss_inputs(case, seed)
    W, R, V, C = case["workers"], case["rows"], case["vocab"], case["width"]
    loss, lse = torch.zeros((2, W * R), dtype=torch.float64, device="cuda")
    if case["way"] != "forward":
        dx = torch.zeros((W * R, C), dtype=torch.float64, device="cuda")
        dweight = torch.zeros((W, V, C), dtype=torch.float64, device="cuda")
    step = max(1, 2 ** 27 // V)
    for m in range(W):
        weight = s["weight"][0 if case["shared"] else m, :V * C].double().view(V, C)
        for at in range(0, R, step):
            rows = slice(m * R + at, m * R + min(R, at + step))
            x, t = s["x"][rows].double(), s["targets"][m, at:at + step].long()
            live = t >= 0
            c = s["weights"][rows].double() * live
            logp = torch.mm(x, weight.t())
            mine = torch.logsumexp(logp, 1) if case["way"] != "backward" else s["lse"][rows].double()
            logp -= mine[:, None]
            loss[rows] = -c * logp.gather(1, t.clamp(min=0)[:, None])[:, 0]
            lse[rows] = mine * live
            if case["way"] != "forward":
                d = logp.exp_()
                d[torch.arange(len(t), device="cuda"), t.clamp(min=0)] -= 1
                d *= (s["scale"] * c)[:, None]
                dx[rows] = d @ weight
                dweight[m].addmm_(d.t(), x)
    out = {"loss": loss, "lse": lse} if case["way"] != "backward" else {}
    return out | ({"dx": dx, "dweight": dweight.view(W, V * C)} if case["way"] != "forward" else {})


def _exact_clip(case, seed):
    tensors = _clip_inputs(case, seed)["tensors"]
    total = torch.zeros(case["workers"], dtype=torch.float64, device="cuda")
    for t in tensors:
        total += torch.linalg.vector_norm(t.double(), dim=1) ** 2
    norms = torch.sqrt(total)
    if case["way"] == "norm":
        return {"norms": norms}
    factor = torch.minimum(torch.ones_like(norms), case["max_norm"] / (norms + EPS))
    return {"norms": norms, "g": torch.cat([t.double() * factor[:, None] for t in tensors], 1)}
