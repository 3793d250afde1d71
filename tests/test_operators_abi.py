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
