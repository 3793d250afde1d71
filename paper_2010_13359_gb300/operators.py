"""Binding of the token-model operators of the C-ABI (include/dqgan.h).

A worker's gradient F(w; xi) comes from the caller's model; these are the parts
that models over tokens are made of, batched over the workers.  As in ``dqgan``, the classes only marshal arguments: pointers are
``torch.Tensor``s, integer addresses or None where the header allows NULL, and
strides are in elements.  A tensor has to be of the type that the operator was
made for (ids as torch.topk gives them are int64, the distillation's int32);
memory that a tensor of another type holds is given by its address, or as bytes.
"""
from __future__ import annotations

import ctypes

from .dqgan import BF16, ERR_INVALID_ARG, F16, F32, NONE, OK, DqganError, _ptr, load_library


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


class LinearConfig(ctypes.Structure):
    """Mirror of ``dqgan_linear_config`` (56 bytes, no padding)."""
    _fields_ = [
        ("inputs", ctypes.c_int64),
        ("outputs", ctypes.c_int64),
        ("max_rows", ctypes.c_int64),
        ("workers", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("weight_dtype", ctypes.c_int32),
        ("activation", ctypes.c_int32),
        ("reserved", ctypes.c_uint32 * 2),
        ("cuda_stream", ctypes.c_void_p),
    ]


class TokenLossConfig(ctypes.Structure):
    """Mirror of ``dqgan_token_loss_config`` (56 bytes, no padding)."""
    _fields_ = [
        ("vocab", ctypes.c_int64),
        ("width", ctypes.c_int64),
        ("max_rows", ctypes.c_int64),
        ("workers", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("weight_dtype", ctypes.c_int32),
        ("token_bits", ctypes.c_int32),
        ("reserved", ctypes.c_uint32 * 2),
        ("cuda_stream", ctypes.c_void_p),
    ]


class GradientClipConfig(ctypes.Structure):
    """Mirror of ``dqgan_gradient_clip_config`` (32 bytes, no padding)."""
    _fields_ = [
        ("workers", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("out_dtype", ctypes.c_int32),
        ("eps", ctypes.c_float),
        ("reserved", ctypes.c_uint32 * 2),
        ("cuda_stream", ctypes.c_void_p),
    ]


class Tensor(ctypes.Structure):
    """Mirror of ``dqgan_tensor`` (24 bytes, no padding)."""
    _fields_ = [
        ("data", ctypes.c_void_p),
        ("size", ctypes.c_int64),
        ("stride", ctypes.c_int64),
    ]


assert (ctypes.sizeof(LayerNormConfig), ctypes.sizeof(EmbeddingConfig), ctypes.sizeof(DistillationConfig)) == (32, 56, 40)
assert (ctypes.sizeof(LinearConfig), ctypes.sizeof(TokenLossConfig), ctypes.sizeof(GradientClipConfig),
        ctypes.sizeof(Tensor)) == (56, 56, 32, 24)


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

    def selftest_wait_timeout(self, polls: int = 0) -> None:
        """Enqueue the bounded-wait self-test; the next synchronize() raises DqganError with status ERR_TIMEOUT."""
        _check(load_library().dqgan_operator_selftest_wait_timeout(self._h, polls), self._h)

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


class Linear(Operator):
    """Linear layers of the workers, y = act(x W^T + b) + r, and their gradients."""

    def __init__(self, inputs: int, outputs: int, max_rows: int, workers: int = 1, dtype: int = F32,
                 weight_dtype: int = F32, activation: int = NONE, cuda_stream: int | None = None):
        super().__init__("dqgan_linear_create",
                         LinearConfig(inputs=inputs, outputs=outputs, max_rows=max_rows, workers=workers, dtype=dtype,
                                      weight_dtype=weight_dtype, activation=activation, cuda_stream=cuda_stream))
        self._f32, self._rows, self._weight = _types("float32", _NAMES[dtype], _NAMES[weight_dtype])
        L = load_library()
        self._forward = L.dqgan_linear_forward
        self._backward = L.dqgan_linear_backward

    def forward(self, rows: int, x, x_stride: int, weight, p_stride: int, bias, b_stride: int, residual,
                residual_stride: int, y, y_stride: int, pre=None, pre_stride: int = 0) -> None:
        """`rows` rows per worker; worker m's weight p_stride * m elements, its bias b_stride * m floats after worker
        0's; `pre` receives x W^T + b for the backward pass of an activation."""
        T, E, f32 = self._rows, self._weight, self._f32
        status = self._forward(self._h, rows, _at(x, T), x_stride, _at(weight, E), p_stride, _at(bias, f32), b_stride,
                               _at(residual, T), residual_stride, _at(y, T), y_stride, _at(pre, T), pre_stride)
        if status:
            _check(status, self._h)

    def backward(self, rows: int, dy, dy_stride: int, x, x_stride: int, weight, p_stride: int, pre, pre_stride: int, dx,
                 dx_stride: int, dweight, dbias, g_stride: int, accumulate: bool = False) -> None:
        """dx, and each worker's dweight and dbias, g_stride floats apart."""
        T, E, f32 = self._rows, self._weight, self._f32
        status = self._backward(self._h, rows, _at(dy, T), dy_stride, _at(x, T), x_stride, _at(weight, E), p_stride,
                                _at(pre, T), pre_stride, _at(dx, T), dx_stride, _at(dweight, f32), _at(dbias, f32),
                                g_stride, accumulate)
        if status:
            _check(status, self._h)


class TokenLoss(Operator):
    """Cross entropy of the workers' output layers over a vocabulary, without its logits, and its gradient."""

    def __init__(self, vocab: int, width: int, max_rows: int, workers: int = 1, dtype: int = F32, weight_dtype: int = F32,
                 token_bits: int = 32, cuda_stream: int | None = None):
        super().__init__("dqgan_token_loss_create",
                         TokenLossConfig(vocab=vocab, width=width, max_rows=max_rows, workers=workers, dtype=dtype,
                                         weight_dtype=weight_dtype, token_bits=token_bits, cuda_stream=cuda_stream))
        self._f32, self._rows, self._weight, self._ids = _types("float32", _NAMES[dtype], _NAMES[weight_dtype],
                                                                f"int{token_bits}")
        L = load_library()
        self._forward = L.dqgan_token_loss_forward
        self._backward = L.dqgan_token_loss_backward
        self._step = L.dqgan_token_loss_step

    def forward(self, rows: int, x, x_stride: int, weight, p_stride: int, targets, weights, loss, lse=None) -> None:
        """`rows` rows per worker; worker m's weight p_stride * m elements after worker 0's."""
        T, E, I, f32 = self._rows, self._weight, self._ids, self._f32
        status = self._forward(self._h, rows, _at(x, T), x_stride, _at(weight, E), p_stride, _at(targets, I),
                               _at(weights, f32), _at(loss, f32), _at(lse, f32))
        if status:
            _check(status, self._h)

    def backward(self, rows: int, x, x_stride: int, weight, p_stride: int, targets, weights, lse, scale: float, dx,
                 dx_stride: int, dweight, g_stride: int, accumulate: bool = False) -> None:
        """dx, and each worker's dweight, g_stride floats apart."""
        T, E, I, f32 = self._rows, self._weight, self._ids, self._f32
        status = self._backward(self._h, rows, _at(x, T), x_stride, _at(weight, E), p_stride, _at(targets, I),
                                _at(weights, f32), _at(lse, f32), scale, _at(dx, T), dx_stride, _at(dweight, f32),
                                g_stride, accumulate)
        if status:
            _check(status, self._h)

    def step(self, rows: int, x, x_stride: int, weight, p_stride: int, targets, weights, scale: float, loss, lse, dx,
             dx_stride: int, dweight, g_stride: int, accumulate: bool = False) -> None:
        """The forward and the backward pass in one call."""
        T, E, I, f32 = self._rows, self._weight, self._ids, self._f32
        status = self._step(self._h, rows, _at(x, T), x_stride, _at(weight, E), p_stride, _at(targets, I),
                            _at(weights, f32), scale, _at(loss, f32), _at(lse, f32), _at(dx, T), dx_stride,
                            _at(dweight, f32), g_stride, accumulate)
        if status:
            _check(status, self._h)


class TensorList:
    """Tensors of all workers, as the clipping takes them: (tensor or address, values of one worker, distance between
    workers) of each.  Keeps the tensors; made once, it serves every call as long as they stay where they are."""

    def __init__(self, tensors):
        tensors = list(tensors)
        self._keep = [t for t, _, _ in tensors]
        self._list = (Tensor * len(tensors))(*[Tensor(_ptr(t), size, stride) for t, size, stride in tensors])
        self._types = {str(t.dtype) for t in self._keep if hasattr(t, "dtype")}

    def __len__(self) -> int:
        return len(self._list)

    def _check(self, dtype) -> None:
        for t in self._types:
            if dtype is not None and t != str(dtype) and t != "torch.uint8":
                raise DqganError(ERR_INVALID_ARG, f"a tensor of {t} where the operator has {dtype}")


class GradientClip(Operator):
    """The norm of every worker's gradient over many tensors, and its clipping into the rows a worker step reads."""

    def __init__(self, workers: int = 1, dtype: int = F32, out_dtype: int = F32, eps: float = 1e-6,
                 cuda_stream: int | None = None):
        super().__init__("dqgan_gradient_clip_create",
                         GradientClipConfig(workers=workers, dtype=dtype, out_dtype=out_dtype, eps=eps,
                                            cuda_stream=cuda_stream))
        self._f32, self._from, self._to = _types("float32", _NAMES[dtype], _NAMES[out_dtype])
        L = load_library()
        self._norm = L.dqgan_gradient_norm
        self._clip = L.dqgan_gradient_clip

    def norm(self, tensors: TensorList, norms) -> None:
        tensors._check(self._from)
        status = self._norm(self._h, len(tensors), tensors._list, _at(norms, self._f32))
        if status:
            _check(status, self._h)

    def clip(self, tensors: TensorList, places: TensorList, max_norm: float, norms=None) -> None:
        """Each tensor, scaled where its worker's norm is above max_norm, into its place."""
        tensors._check(self._from)
        places._check(self._to)
        if len(tensors) != len(places):
            raise DqganError(ERR_INVALID_ARG, f"{len(tensors)} tensors and {len(places)} places")
        status = self._clip(self._h, len(tensors), tensors._list, places._list, max_norm, _at(norms, self._f32))
        if status:
            _check(status, self._h)
