"""A small token model trained through the full Algorithm 2 loop on the device.

Every worker holds a batch of tokens and a teacher's top logits at each of
them.  The student is an embedding, a layer norm and an output layer that
shares the embedding's table: z = norm(sqrt(width) E[token]) E^T.  Its loss is
the distillation from the teacher's entries, and F(w) the gradient of the
workers' mean loss per token with respect to the flat vector

    w = [E (vocab x width) | norm weight (width) | norm bias (width)].

All M workers run at once: `operators` reads each worker's parameters at its
lookahead point and writes its gradient into its row of the buffer that the
worker step compresses; the output layer's products are library products (the
rest of a user's model would stand there).
"""
from __future__ import annotations

import math

from . import dqgan, operators


class TokenModel:
    def __init__(self, vocab: int, width: int, tokens: int, workers: int, k: int, temperature: float = 1.0,
                 cuda_stream: int | None = None):
        """`tokens` per worker; `k` teacher entries a token; `cuda_stream`: the current stream of the torch
        calls around it."""
        self.vocab, self.width, self.tokens, self.workers, self.k = vocab, width, tokens, workers, k
        self.embedding = operators.Embedding(vocab=vocab, width=width, max_tokens=tokens, workers=workers,
                                             scale=math.sqrt(width), cuda_stream=cuda_stream)
        self.norm = operators.LayerNorm(width=width, workers=workers, cuda_stream=cuda_stream)
        self.distillation = operators.Distillation(vocab=vocab, k=k, temperature=temperature, cuda_stream=cuda_stream)

    @property
    def d(self) -> int:
        return self.vocab * self.width + 2 * self.width

    def buffers(self, device) -> dict:
        """The activations of one step."""
        import torch
        rows = (self.workers * self.tokens, self.width)
        b = {name: torch.empty(rows, device=device) for name in ("x", "y", "dy")}
        b["logits"] = torch.empty((self.workers * self.tokens, self.vocab), device=device)
        b |= {name: torch.empty(rows[0], device=device) for name in ("mean", "rstd", "loss")}
        return b

    def _check_batch(self, params, ids, teacher_ids, teacher_values, weights, g) -> None:
        """The kernels take addresses, and one row stride for both teacher tensors."""
        M, rows, k = self.workers, self.workers * self.tokens, self.k
        for name, t in (("params", params), ("g", g)):
            if t.dim() != 2 or t.shape[0] != M or t.shape[1] < self.d or t.stride(1) != 1:
                raise ValueError(f"{name}: {M} rows of at least {self.d} values are needed")
        for name, t in (("ids", ids), ("weights", weights)):
            if t is not None and not (t.is_contiguous() and (t.numel() == rows or t.dim() == 1 and t.numel() > rows)):
                raise ValueError(f"{name}: {rows} values without gaps are needed")
        for name, t in (("teacher_ids", teacher_ids), ("teacher_values", teacher_values)):
            if t.dim() != 2 or t.shape[0] < rows or t.shape[1] < k or k > 1 and t.stride(1) != 1:
                raise ValueError(f"{name}: {rows} rows of at least {k} values are needed")
        if rows > 1 and teacher_ids.stride(0) != teacher_values.stride(0):
            raise ValueError("teacher_ids and teacher_values: rows of one stride are needed")

    def operator(self, params, ids, teacher_ids, teacher_values, weights, g, b) -> None:
        """g[m] = F(params[m]) for every worker m, and b["loss"] each token's loss.  params: (workers, d) fp32,
        its rows p_stride floats apart; ids: (workers, tokens) int32, -1 for no token; teacher_ids (int32) and
        teacher_values: (workers * tokens, k), rows of one stride; weights: a token's weight, 0 where it does
        not count, or None; g: rows of at least d floats."""
        import torch
        self._check_batch(params, ids, teacher_ids, teacher_values, weights, g)
        M, n, V, C = self.workers, self.tokens, self.vocab, self.width
        p_stride, g_stride = params.stride(0), g.stride(0)
        table = params[:, :V * C].view(M, V, C)
        weight, bias = params[:, V * C:], params[:, V * C + C:]
        logits = b["logits"].view(M, n, V)
        self.embedding.forward(n, ids, params, p_stride, b["x"], C)
        self.norm.forward(n, b["x"], C, weight, bias, p_stride, b["y"], C, b["mean"], b["rstd"])
        torch.bmm(b["y"].view(M, n, C), table.transpose(1, 2), out=logits)
        # the logits' gradient in the logits' place
        self.distillation.step(M * n, b["logits"], V, teacher_ids, teacher_values, teacher_ids.stride(0), None, weights,
                               1.0 / n, b["loss"], None, b["logits"], V)
        torch.bmm(logits, table, out=b["dy"].view(M, n, C))
        g[:, :V * C].view(M, V, C).copy_(torch.bmm(logits.transpose(1, 2), b["y"].view(M, n, C)))
        self.norm.backward(n, b["dy"], C, b["x"], C, weight, p_stride, b["mean"], b["rstd"], b["dy"], C,
                           g[:, V * C:], g[:, V * C + C:], g_stride)
        self.embedding.backward(n, ids, b["dy"], C, g, g_stride, accumulate=True)


def train(handle, model: TokenModel, w, batch, steps: int, on_step=None):
    """Runs `steps` iterations of Algorithm 2 on the device parameters `w`.  `batch(t)` gives step t's ids,
    teacher_ids, teacher_values and weights; the handle (d = model.d, M = model.workers) keeps the lookahead
    offsets.  `on_step(t, loss)` sees each step's mean loss per worker (a device tensor)."""
    import torch
    if handle.cfg.d != model.d or handle.cfg.M != model.workers:
        raise ValueError("handle and model disagree on d or M")
    if not (handle.cfg.flags & dqgan.KEEP_LOOKAHEAD):
        raise ValueError("train needs a handle created with KEEP_LOOKAHEAD")
    M, d = model.workers, model.d
    ld = (d + 3) // 4 * 4
    g = torch.zeros((M, ld), device=w.device)
    w_half = torch.empty((M, ld), device=w.device)
    msgs = torch.zeros((M, handle.message_bytes()), dtype=torch.uint8, device=w.device)
    b = model.buffers(w.device)
    for t in range(steps):
        for i in range(M):
            handle.worker_lookahead(i, w, w_half[i])
        model.operator(w_half[:, :d], *batch(t), g, b)
        handle.workers_compress_all(g, ld, msgs)
        handle.server_aggregate_update(msgs, w)
        if on_step is not None:
            on_step(t, b["loss"].view(M, -1).mean(1))
    return w
