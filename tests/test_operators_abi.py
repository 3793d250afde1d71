"""The token-model operators on the host: struct layouts, refused configs, NULL handles.  No call here
launches a kernel."""
from __future__ import annotations

import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def P():
    from paper_2010_13359_gb300 import build
    build.build()
    import paper_2010_13359_gb300 as P
    P.dqgan.load_library()
    return P


def test_struct_layouts_match_the_header(tmp_path, P):
    from paper_2010_13359_gb300 import operators as O
    lines = ['#include <stddef.h>', '#include "dqgan.h"']
    for c_name, cls in (("dqgan_layer_norm_config", O.LayerNormConfig), ("dqgan_embedding_config", O.EmbeddingConfig),
                        ("dqgan_distillation_config", O.DistillationConfig)):
        lines.append(f'_Static_assert(sizeof({c_name}) == {ctypes.sizeof(cls)}, "size");')
        for name, _ in cls._fields_:
            lines.append(f'_Static_assert(offsetof({c_name}, {name}) == {getattr(cls, name).offset}, "{name}");')
    for name in ("F32", "BF16", "F16"):
        lines.append(f'_Static_assert(DQGAN_{name} == {getattr(P, name)}, "{name}");')
    c = tmp_path / "layout.c"
    c.write_text("\n".join(lines))
    subprocess.run(["gcc", "-std=c11", "-fsyntax-only", "-I", os.path.join(ROOT, "include"), str(c)], check=True)


NORM = dict(width=64)
EMBED = dict(vocab=100, width=8, max_tokens=10)
DISTILL = dict(vocab=100, k=4)


@pytest.mark.parametrize("kind,kw,needle", [
    ("LayerNorm", NORM | dict(width=0), "width"),
    ("LayerNorm", NORM | dict(width=65537), "width"),
    ("LayerNorm", NORM | dict(workers=0), "workers"),
    ("LayerNorm", NORM | dict(dtype=3), "dtype"),
    ("LayerNorm", NORM | dict(eps=-1.0), "eps"),
    ("LayerNorm", NORM | dict(eps=float("nan")), "eps"),
    ("Embedding", EMBED | dict(vocab=0), "vocab"),
    ("Embedding", EMBED | dict(vocab=(1 << 24) + 1), "vocab"),
    ("Embedding", EMBED | dict(width=0), "width"),
    ("Embedding", EMBED | dict(max_tokens=0), "max_tokens"),
    ("Embedding", EMBED | dict(workers=4097), "workers"),
    ("Embedding", EMBED | dict(workers=4096, vocab=1 << 20), "2^28"),
    ("Embedding", EMBED | dict(table_dtype=-1), "dtype"),
    ("Embedding", EMBED | dict(token_bits=16), "token_bits"),
    ("Embedding", EMBED | dict(scale=float("inf")), "scale"),
    ("Distillation", DISTILL | dict(vocab=0), "vocab"),
    ("Distillation", DISTILL | dict(k=0), "k "),
    ("Distillation", DISTILL | dict(k=1025), "k "),
    ("Distillation", DISTILL | dict(teacher_dtype=9), "dtype"),
    ("Distillation", DISTILL | dict(temperature=0.0), "temperature"),
    ("Distillation", DISTILL | dict(temperature=float("nan")), "temperature"),
])
def test_invalid_configs_are_refused(P, kind, kw, needle):
    with pytest.raises(P.DqganError) as ei:
        getattr(P, kind)(**kw)
    assert ei.value.status == P.dqgan.ERR_INVALID_ARG
    assert needle in str(ei.value)


def test_null_handles(P):
    L = P.dqgan.load_library()
    assert L.dqgan_operator_destroy(None) == P.dqgan.OK
    assert L.dqgan_operator_synchronize(None) == P.dqgan.ERR_INVALID_ARG
    assert L.dqgan_operator_launch_count(None) == 0
    assert L.dqgan_layer_norm_create(None, None) == P.dqgan.ERR_INVALID_ARG
    h = ctypes.c_void_p()
    for name in ("layer_norm", "embedding", "distillation"):
        assert getattr(L, f"dqgan_{name}_create")(None, ctypes.byref(h)) == P.dqgan.ERR_INVALID_ARG and not h.value
    assert L.dqgan_layer_norm_forward(None, 1, None, 1, None, None, 0, None, 1, None, None) == P.dqgan.ERR_INVALID_ARG
    assert L.dqgan_embedding_backward(None, 1, None, None, 1, None, 1, 0) == P.dqgan.ERR_INVALID_ARG
    assert L.dqgan_distillation_forward(None, 1, None, 1, None, None, 1, None, None, None, None) == P.dqgan.ERR_INVALID_ARG
    assert b"NULL" in L.dqgan_operator_last_error(None)


@pytest.mark.parametrize("owner,call", [("Operator", "dqgan_operator_destroy"), ("Handle", "dqgan_destroy")])
def test_a_destroy_that_fails_is_not_repeated(P, monkeypatch, owner, call):
    """The library frees the object whatever it returns: an error of earlier work that shows there is raised once, and
    the owner lets go of the object."""
    from paper_2010_13359_gb300 import dqgan, operators
    destroyed = []

    class Library:
        def dqgan_operator_last_error(self, op):
            return b"destroy: an earlier error"

        dqgan_last_error = dqgan_operator_last_error

    def destroy(self, h):
        destroyed.append(h.value)
        return P.dqgan.ERR_CUDA

    setattr(Library, call, destroy)
    module, cls = (operators, operators.Operator) if owner == "Operator" else (dqgan, dqgan.Handle)
    monkeypatch.setattr(module, "load_library", lambda: Library())
    o = object.__new__(cls)
    o._h = ctypes.c_void_p(1234)
    with pytest.raises(P.DqganError, match="earlier error"):
        o.destroy()
    o.destroy()
    del o
    assert destroyed == [1234]


def fake_operators(P, monkeypatch):
    """The three operators over a library that only records its calls."""
    from paper_2010_13359_gb300 import operators
    calls = []

    class Library:
        def __getattr__(self, name):
            if name.endswith(("create", "destroy")):
                return lambda *args: 0
            return lambda *args: calls.append(name) or 0

    monkeypatch.setattr(operators, "load_library", lambda: Library())
    return (P.LayerNorm(width=8, dtype=P.BF16), P.Embedding(vocab=4, width=8, max_tokens=2, table_dtype=P.F16, token_bits=64),
            P.Distillation(vocab=8, k=2, teacher_dtype=P.BF16)), calls


def operator_calls(torch, ops):
    """Every call with tensors of the right types: (call, arguments, which of them are tensors)."""
    norm, embed, distill = ops
    half, f16, f32 = (torch.zeros(16, dtype=t) for t in (torch.bfloat16, torch.float16, torch.float32))
    ids32, ids64 = torch.zeros(4, dtype=torch.int32), torch.zeros(4, dtype=torch.int64)
    return [
        (norm.forward, [1, half, 8, f32, f32, 8, half, 8, f32, f32]),
        (norm.backward, [1, half, 8, half, 8, f32, 8, f32, f32, half, 8, f32, f32, 8]),
        (embed.forward, [1, ids64, f16, 32, f32, 8]),
        (embed.backward, [1, ids64, f32, 8, f32, 32]),
        (distill.forward, [1, f32, 8, ids32, half, 2, f32, f32, f32, f32]),
        (distill.backward, [1, f32, 8, f32, ids32, half, 2, f32, f32, 1.0, f32, 8]),
        (distill.step, [1, f32, 8, ids32, half, 2, f32, f32, 1.0, f32, f32, f32, 8]),
    ]


def test_tensors_of_another_type_are_refused(P, monkeypatch):
    """torch.topk and torch's default integers give int64 ids: read as 32-bit ones every second is the upper half."""
    torch = pytest.importorskip("torch")
    ops, calls = fake_operators(P, monkeypatch)
    types = (torch.float32, torch.bfloat16, torch.float16, torch.float64, torch.int32, torch.int64, torch.int8)
    for call, args in operator_calls(torch, ops):
        for i, right in enumerate(args):
            if not isinstance(right, torch.Tensor):
                continue
            for t in types:
                if t is right.dtype:
                    continue
                with pytest.raises(P.DqganError) as ei:
                    call(*args[:i], right.to(t), *args[i + 1:])
                assert ei.value.status == P.dqgan.ERR_INVALID_ARG
                assert str(t) in str(ei.value) and str(right.dtype) in str(ei.value)
    assert calls == []


def test_what_the_types_let_through(P, monkeypatch):
    """The config's types, addresses, None, raw bytes and unsigned ids of the same size."""
    torch = pytest.importorskip("torch")
    ops, calls = fake_operators(P, monkeypatch)
    for call, args in operator_calls(torch, ops):
        call(*args)
        tensors = [i for i, a in enumerate(args) if isinstance(a, torch.Tensor)]
        for other in (lambda x: None, lambda x: x.data_ptr(), lambda x: x.view(torch.uint8),
                      lambda x: x.view({torch.int32: torch.uint32, torch.int64: torch.uint64}.get(x.dtype, x.dtype))):
            call(*[other(a) if i in tensors else a for i, a in enumerate(args)])
    assert len(calls) == 5 * 7


def test_temperatures_whose_reciprocal_overflows_are_refused(P):
    """The kernels multiply by 1 / T: infinite for a subnormal T, and every result NaN."""
    least = 2.0 ** -126
    P.Distillation(vocab=8, k=1, temperature=least)._h = None  # kept from a destroy, which needs a GPU
    for t in (least / 2, least / 8, 2.0 ** -149):
        with pytest.raises(P.DqganError, match="temperature") as ei:
            P.Distillation(vocab=8, k=1, temperature=t)
        assert ei.value.status == P.dqgan.ERR_INVALID_ARG
