"""Binding of the token-model operators of the C-ABI (include/dqgan.h).

A worker's gradient F(w; xi) comes from the caller's model; these are the ends
of that gradient that a matrix product does not cover, batched over the
workers.  As in ``dqgan``, the classes only marshal arguments: pointers are
``torch.Tensor``s, integer addresses or None where the header allows NULL, and
strides are in elements.  A tensor has to be of the type that the operator was
made for (ids as torch.topk gives them are int64, the distillation's int32);
memory that a tensor of another type holds is given by its address, or as bytes.
"""
from __future__ import annotations

import ctypes

from .dqgan import BF16, ERR_INVALID_ARG, F16, F32, OK, DqganError, _ptr, load_library


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


def _types(*names: str):
    """torch's types of these names; None where torch is not there to make tensors."""
    try:
        import torch
    except ImportError:
        return (None,) * len(names)
    return tuple(getattr(torch, name) for name in names)


_NAMES = {F32: "float32", BF16: "bfloat16", F16: "float16"}


def _at(x, dtype) -> int | None:
    """Address of x, whose elements are read or written as `dtype`."""
    if x is None:
        return None
    try:
        if x.dtype is dtype:
            return x.data_ptr()
    except AttributeError:
        return _ptr(x)
    if dtype is not None and hasattr(x, "data_ptr"):
        got = str(x.dtype)
        if got != "torch.uint8" and got.replace("torch.u", "torch.") != str(dtype):
            raise DqganError(ERR_INVALID_ARG, f"a tensor of {got} where the operator has {dtype}")
    return _ptr(x)


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
        self._f32, self._rows = _types("float32", _NAMES[dtype])
        L = load_library()
        self._forward = L.dqgan_layer_norm_forward
        self._backward = L.dqgan_layer_norm_backward

    def forward(self, rows: int, x, x_stride: int, weight, bias, p_stride: int, y, y_stride: int, mean=None,
                rstd=None) -> None:
        """`rows` rows per worker; worker m's weight and bias p_stride * m floats after worker 0's."""
        T, f32 = self._rows, self._f32
        status = self._forward(self._h, rows, _at(x, T), x_stride, _at(weight, f32), _at(bias, f32), p_stride,
                               _at(y, T), y_stride, _at(mean, f32), _at(rstd, f32))
        if status:
            _check(status, self._h)

    def backward(self, rows: int, dy, dy_stride: int, x, x_stride: int, weight, p_stride: int, mean, rstd, dx,
                 dx_stride: int, dweight, dbias, g_stride: int, accumulate: bool = False) -> None:
        """dx, and each worker's dweight and dbias, g_stride floats apart."""
        T, f32 = self._rows, self._f32
        status = self._backward(self._h, rows, _at(dy, T), dy_stride, _at(x, T), x_stride, _at(weight, f32), p_stride,
                                _at(mean, f32), _at(rstd, f32), _at(dx, T), dx_stride, _at(dweight, f32),
                                _at(dbias, f32), g_stride, accumulate)
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
        self._f32, self._rows, self._table, self._ids = _types("float32", _NAMES[dtype], _NAMES[table_dtype],
                                                               f"int{token_bits}")
        L = load_library()
        self._forward = L.dqgan_embedding_forward
        self._backward = L.dqgan_embedding_backward

    def forward(self, tokens: int, ids, table, p_stride: int, y, y_stride: int) -> None:
        """`tokens` tokens per worker; worker m's table p_stride * m elements after worker 0's."""
        T, E, I = self._rows, self._table, self._ids
        status = self._forward(self._h, tokens, _at(ids, I), _at(table, E), p_stride, _at(y, T), y_stride)
        if status:
            _check(status, self._h)

    def backward(self, tokens: int, ids, dy, dy_stride: int, dtable, g_stride: int, accumulate: bool = False) -> None:
        """Each worker's gradient of its table, g_stride floats apart."""
        T, I, f32 = self._rows, self._ids, self._f32
        status = self._backward(self._h, tokens, _at(ids, I), _at(dy, T), dy_stride, _at(dtable, f32), g_stride,
                                accumulate)
        if status:
            _check(status, self._h)


class Distillation(Operator):
    """Loss of student logits against a teacher's top entries, and its gradient."""

    def __init__(self, vocab: int, k: int, dtype: int = F32, teacher_dtype: int = F32, temperature: float = 1.0,
                 cuda_stream: int | None = None):
        super().__init__("dqgan_distillation_create",
                         DistillationConfig(vocab=vocab, k=k, dtype=dtype, teacher_dtype=teacher_dtype,
                                            temperature=temperature, cuda_stream=cuda_stream))
        self._f32, self._i32, self._rows, self._values = _types("float32", "int32", _NAMES[dtype], _NAMES[teacher_dtype])
        L = load_library()
        self._forward = L.dqgan_distillation_forward
        self._backward = L.dqgan_distillation_backward
        self._step = L.dqgan_distillation_step

    def forward(self, rows: int, logits, logits_stride: int, ids, values, teacher_stride: int, teacher_lse, weights,
                loss, lse=None) -> None:
        T, I, V, f32 = self._rows, self._i32, self._values, self._f32
        status = self._forward(self._h, rows, _at(logits, T), logits_stride, _at(ids, I), _at(values, V),
                               teacher_stride, _at(teacher_lse, f32), _at(weights, f32), _at(loss, f32), _at(lse, f32))
        if status:
            _check(status, self._h)

    def backward(self, rows: int, logits, logits_stride: int, lse, ids, values, teacher_stride: int, teacher_lse,
                 weights, scale: float, dlogits, dlogits_stride: int) -> None:
        T, I, V, f32 = self._rows, self._i32, self._values, self._f32
        status = self._backward(self._h, rows, _at(logits, T), logits_stride, _at(lse, f32), _at(ids, I),
                                _at(values, V), teacher_stride, _at(teacher_lse, f32), _at(weights, f32), scale,
                                _at(dlogits, T), dlogits_stride)
        if status:
            _check(status, self._h)

    def step(self, rows: int, logits, logits_stride: int, ids, values, teacher_stride: int, teacher_lse, weights,
             scale: float, loss, lse, dlogits, dlogits_stride: int) -> None:
        """The forward and the backward pass in one call."""
        T, I, V, f32 = self._rows, self._i32, self._values, self._f32
        status = self._step(self._h, rows, _at(logits, T), logits_stride, _at(ids, I), _at(values, V), teacher_stride,
                            _at(teacher_lse, f32), _at(weights, f32), scale, _at(loss, f32), _at(lse, f32),
                            _at(dlogits, T), dlogits_stride)
        if status:
            _check(status, self._h)
