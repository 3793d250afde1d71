"""Binding of the token-model operators of the C-ABI (include/dqgan.h).

A worker's gradient F(w; xi) comes from the caller's model; these are the ends
of that gradient that a matrix product does not cover, batched over the
workers.  As in ``dqgan``, the classes only marshal arguments: pointers are
``torch.Tensor``s, integer addresses or None where the header allows NULL, and
strides are in elements.
"""
from __future__ import annotations

import ctypes

from .dqgan import F32, OK, DqganError, _ptr, load_library


class LayerNormConfig(ctypes.Structure):
    """Mirror of ``dqgan_layer_norm_config`` (32 bytes, no padding)."""
    _fields_ = [
        ("width", ctypes.c_int64),
        ("workers", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("eps", ctypes.c_float),
        ("reserved", ctypes.c_uint32),
        ("cuda_stream", ctypes.c_void_p),
    ]


class EmbeddingConfig(ctypes.Structure):
    """Mirror of ``dqgan_embedding_config`` (56 bytes, no padding)."""
    _fields_ = [
        ("vocab", ctypes.c_int64),
        ("width", ctypes.c_int64),
        ("max_tokens", ctypes.c_int64),
        ("workers", ctypes.c_int32),
        ("table_dtype", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("token_bits", ctypes.c_int32),
        ("scale", ctypes.c_float),
        ("reserved", ctypes.c_uint32),
        ("cuda_stream", ctypes.c_void_p),
    ]


class DistillationConfig(ctypes.Structure):
    """Mirror of ``dqgan_distillation_config`` (40 bytes, no padding)."""
    _fields_ = [
        ("vocab", ctypes.c_int64),
        ("k", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("teacher_dtype", ctypes.c_int32),
        ("temperature", ctypes.c_float),
        ("reserved", ctypes.c_uint32 * 2),
        ("cuda_stream", ctypes.c_void_p),
    ]


assert (ctypes.sizeof(LayerNormConfig), ctypes.sizeof(EmbeddingConfig), ctypes.sizeof(DistillationConfig)) == (32, 56, 40)


def _check(status: int, op=None):
    if status != OK:
        raise DqganError(status, load_library().dqgan_operator_last_error(op).decode())


class Operator:
    """Owner of one ``dqgan_operator``."""

    def __init__(self, create: str, cfg):
        self.cfg = cfg
        self._h = None
        L = load_library()
        h = ctypes.c_void_p()
        _check(getattr(L, create)(ctypes.byref(cfg), ctypes.byref(h)))
        self._h = h

    def destroy(self) -> None:
        h, self._h = self._h, None  # freed even where an error of earlier work is returned
        if h is not None and h.value:
            _check(load_library().dqgan_operator_destroy(h))

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.destroy()

    def synchronize(self) -> None:
        _check(load_library().dqgan_operator_synchronize(self._h), self._h)

    def launch_count(self) -> int:
        return int(load_library().dqgan_operator_launch_count(self._h))

    def last_error(self) -> str:
        return load_library().dqgan_operator_last_error(self._h).decode()


class LayerNorm(Operator):
    """Layer norm over the last `width` values of every worker's rows, and its gradient."""

    def __init__(self, width: int, workers: int = 1, dtype: int = F32, eps: float = 1e-5,
                 cuda_stream: int | None = None):
        super().__init__("dqgan_layer_norm_create",
                         LayerNormConfig(width=width, workers=workers, dtype=dtype, eps=eps, cuda_stream=cuda_stream))
        L = load_library()
        self._forward = L.dqgan_layer_norm_forward
        self._backward = L.dqgan_layer_norm_backward

    def forward(self, rows: int, x, x_stride: int, weight, bias, p_stride: int, y, y_stride: int, mean=None,
                rstd=None) -> None:
        """`rows` rows per worker; worker m's weight and bias p_stride * m floats after worker 0's."""
        status = self._forward(self._h, rows, _ptr(x), x_stride, _ptr(weight), _ptr(bias), p_stride, _ptr(y), y_stride,
                               _ptr(mean), _ptr(rstd))
        if status:
            _check(status, self._h)

    def backward(self, rows: int, dy, dy_stride: int, x, x_stride: int, weight, p_stride: int, mean, rstd, dx,
                 dx_stride: int, dweight, dbias, g_stride: int, accumulate: bool = False) -> None:
        """dx, and each worker's dweight and dbias, g_stride floats apart."""
        status = self._backward(self._h, rows, _ptr(dy), dy_stride, _ptr(x), x_stride, _ptr(weight), p_stride,
                                _ptr(mean), _ptr(rstd), _ptr(dx), dx_stride, _ptr(dweight), _ptr(dbias), g_stride,
                                accumulate)
        if status:
            _check(status, self._h)


class Embedding(Operator):
    """Lookup in every worker's table, scaled, and the table's gradient."""

    def __init__(self, vocab: int, width: int, max_tokens: int, workers: int = 1, table_dtype: int = F32,
                 dtype: int = F32, token_bits: int = 32, scale: float = 1.0, cuda_stream: int | None = None):
        super().__init__("dqgan_embedding_create",
                         EmbeddingConfig(vocab=vocab, width=width, max_tokens=max_tokens, workers=workers,
                                         table_dtype=table_dtype, dtype=dtype, token_bits=token_bits, scale=scale,
                                         cuda_stream=cuda_stream))
        L = load_library()
        self._forward = L.dqgan_embedding_forward
        self._backward = L.dqgan_embedding_backward

    def forward(self, tokens: int, ids, table, p_stride: int, y, y_stride: int) -> None:
        """`tokens` tokens per worker; worker m's table p_stride * m elements after worker 0's."""
        status = self._forward(self._h, tokens, _ptr(ids), _ptr(table), p_stride, _ptr(y), y_stride)
        if status:
            _check(status, self._h)

    def backward(self, tokens: int, ids, dy, dy_stride: int, dtable, g_stride: int, accumulate: bool = False) -> None:
        """Each worker's gradient of its table, g_stride floats apart."""
        status = self._backward(self._h, tokens, _ptr(ids), _ptr(dy), dy_stride, _ptr(dtable), g_stride, accumulate)
        if status:
            _check(status, self._h)


class Distillation(Operator):
    """Loss of student logits against a teacher's top entries, and its gradient."""

    def __init__(self, vocab: int, k: int, dtype: int = F32, teacher_dtype: int = F32, temperature: float = 1.0,
                 cuda_stream: int | None = None):
        super().__init__("dqgan_distillation_create",
                         DistillationConfig(vocab=vocab, k=k, dtype=dtype, teacher_dtype=teacher_dtype,
                                            temperature=temperature, cuda_stream=cuda_stream))
        L = load_library()
        self._forward = L.dqgan_distillation_forward
        self._backward = L.dqgan_distillation_backward
        self._step = L.dqgan_distillation_step

    def forward(self, rows: int, logits, logits_stride: int, ids, values, teacher_stride: int, teacher_lse, weights,
                loss, lse=None) -> None:
        status = self._forward(self._h, rows, _ptr(logits), logits_stride, _ptr(ids), _ptr(values), teacher_stride,
                               _ptr(teacher_lse), _ptr(weights), _ptr(loss), _ptr(lse))
        if status:
            _check(status, self._h)

    def backward(self, rows: int, logits, logits_stride: int, lse, ids, values, teacher_stride: int, teacher_lse,
                 weights, scale: float, dlogits, dlogits_stride: int) -> None:
        status = self._backward(self._h, rows, _ptr(logits), logits_stride, _ptr(lse), _ptr(ids), _ptr(values),
                                teacher_stride, _ptr(teacher_lse), _ptr(weights), scale, _ptr(dlogits), dlogits_stride)
        if status:
            _check(status, self._h)

    def step(self, rows: int, logits, logits_stride: int, ids, values, teacher_stride: int, teacher_lse, weights,
             scale: float, loss, lse, dlogits, dlogits_stride: int) -> None:
        """The forward and the backward pass in one call."""
        status = self._step(self._h, rows, _ptr(logits), logits_stride, _ptr(ids), _ptr(values), teacher_stride,
                            _ptr(teacher_lse), _ptr(weights), scale, _ptr(loss), _ptr(lse), _ptr(dlogits),
                            dlogits_stride)
        if status:
            _check(status, self._h)
