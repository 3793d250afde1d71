"""Linear layers, token loss and gradient clipping on the host: struct layouts, refused configs, NULL handles, tensors of
another type, what the models take for a batch, and the clipping's arithmetic of units and blocks.  No call here launches a
kernel."""
from __future__ import annotations

import ctypes
import os
import subprocess

import pytest

from test_operators_abi import P  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_struct_layouts_match_the_header(tmp_path, P):  # noqa: F811
    from paper_2010_13359_gb300 import operators as O
    lines = ['#include <stddef.h>', '#include "dqgan.h"']
    for c_name, cls in (("dqgan_linear_config", O.LinearConfig), ("dqgan_token_loss_config", O.TokenLossConfig),
                        ("dqgan_gradient_clip_config", O.GradientClipConfig), ("dqgan_tensor", O.Tensor)):
        lines.append(f'_Static_assert(sizeof({c_name}) == {ctypes.sizeof(cls)}, "size");')
        for name, _ in cls._fields_:
            lines.append(f'_Static_assert(offsetof({c_name}, {name}) == {getattr(cls, name).offset}, "{name}");')
    for name in ("NONE", "RELU", "GELU", "SILU"):
        lines.append(f'_Static_assert(DQGAN_{name} == {getattr(P, name)}, "{name}");')
    c = tmp_path / "layout.c"
    c.write_text("\n".join(lines))
    subprocess.run(["gcc", "-std=c11", "-fsyntax-only", "-I", os.path.join(ROOT, "include"), str(c)], check=True)


LINEAR = dict(inputs=64, outputs=32, max_rows=10)
LOSS = dict(vocab=100, width=8, max_rows=10)


@pytest.mark.parametrize("kind,kw,needle", [
    ("Linear", LINEAR | dict(inputs=0), "inputs"),
    ("Linear", LINEAR | dict(inputs=65537), "inputs"),
    ("Linear", LINEAR | dict(outputs=0), "outputs"),
    ("Linear", LINEAR | dict(outputs=1 << 40), "outputs"),
    ("Linear", LINEAR | dict(max_rows=0), "max_rows"),
    ("Linear", LINEAR | dict(max_rows=(1 << 24) + 1), "max_rows"),
    ("Linear", LINEAR | dict(workers=0), "workers"),
    ("Linear", LINEAR | dict(workers=4097), "workers"),
    ("Linear", LINEAR | dict(workers=4096, max_rows=1 << 17), "2^28"),
    ("Linear", LINEAR | dict(dtype=3), "dtype"),
    ("Linear", LINEAR | dict(dtype=0, weight_dtype=1), "weight_dtype"),
    ("Linear", LINEAR | dict(dtype=1, weight_dtype=2), "weight_dtype"),
    ("Linear", LINEAR | dict(activation=4), "activation"),
    ("Linear", LINEAR | dict(activation=-1), "activation"),
    ("TokenLoss", LOSS | dict(vocab=0), "vocab"),
    ("TokenLoss", LOSS | dict(vocab=(1 << 24) + 1), "vocab"),
    ("TokenLoss", LOSS | dict(width=0), "width"),
    ("TokenLoss", LOSS | dict(width=65537), "width"),
    ("TokenLoss", LOSS | dict(max_rows=-1), "max_rows"),
    ("TokenLoss", LOSS | dict(workers=5000), "workers"),
    ("TokenLoss", LOSS | dict(dtype=2, weight_dtype=1), "weight_dtype"),
    ("TokenLoss", LOSS | dict(token_bits=16), "token_bits"),
    ("GradientClip", dict(workers=0), "workers"),
    ("GradientClip", dict(dtype=7), "dtype"),
    ("GradientClip", dict(dtype=0, out_dtype=1), "out_dtype"),
    ("GradientClip", dict(dtype=1, out_dtype=2), "out_dtype"),
    ("GradientClip", dict(eps=-1.0), "eps"),
    ("GradientClip", dict(eps=float("nan")), "eps"),
])
def test_invalid_configs_are_refused(P, kind, kw, needle):  # noqa: F811
    with pytest.raises((P.DqganError, KeyError)) as ei:
        getattr(P, kind)(**kw)
    assert ei.value.status == P.dqgan.ERR_INVALID_ARG
    assert needle in str(ei.value)


def test_reserved_fields_and_null(P):  # noqa: F811
    from paper_2010_13359_gb300 import operators as O
    L = P.dqgan.load_library()
    h = ctypes.c_void_p()
    for name, cls, kw in (("linear", O.LinearConfig, LINEAR | dict(workers=1)),
                          ("token_loss", O.TokenLossConfig, LOSS | dict(workers=1, token_bits=32)),
                          ("gradient_clip", O.GradientClipConfig, dict(workers=1))):
        create = getattr(L, f"dqgan_{name}_create")
        assert create(None, ctypes.byref(h)) == P.dqgan.ERR_INVALID_ARG and not h.value
        cfg = cls(**kw)
        assert create(ctypes.byref(cfg), None) == P.dqgan.ERR_INVALID_ARG
        cfg.reserved[1] = 1
        assert create(ctypes.byref(cfg), ctypes.byref(h)) == P.dqgan.ERR_INVALID_ARG and not h.value
        assert b"reserved" in L.dqgan_operator_last_error(None)
    assert L.dqgan_linear_forward(None, 1, None, 1, None, 0, None, 0, None, 0, None, 1, None, 0) == P.dqgan.ERR_INVALID_ARG
    assert L.dqgan_token_loss_forward(None, 1, None, 1, None, 0, None, None, None, None) == P.dqgan.ERR_INVALID_ARG
    assert L.dqgan_gradient_norm(None, 0, None, None) == P.dqgan.ERR_INVALID_ARG
    assert L.dqgan_gradient_clip(None, 0, None, None, 1.0, None) == P.dqgan.ERR_INVALID_ARG


class CountingLibrary:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        if name.endswith(("create", "destroy")):
            return lambda *args: 0
        return lambda *args: self.calls.append(name) or 0


@pytest.fixture
def library(P, monkeypatch):  # noqa: F811
    from paper_2010_13359_gb300 import operators
    L = CountingLibrary()
    monkeypatch.setattr(operators, "load_library", lambda: L)
    return L


def test_tensors_of_another_type_are_refused(P, library):  # noqa: F811
    torch = pytest.importorskip("torch")
    half, f32 = torch.zeros(64, dtype=torch.bfloat16), torch.zeros(64)
    ids = torch.zeros(4, dtype=torch.int64)
    linear = P.Linear(inputs=8, outputs=8, max_rows=2, dtype=P.BF16)
    loss = P.TokenLoss(vocab=8, width=8, max_rows=2, dtype=P.F16, weight_dtype=P.F16, token_bits=64)
    f16 = half.half()
    clip = P.GradientClip(dtype=P.BF16, out_dtype=P.F32)
    calls = [
        (linear.forward, [1, half, 8, f32, 64, f32, 8, half, 8, half, 8, half, 8]),
        (linear.backward, [1, half, 8, half, 8, f32, 64, half, 8, half, 8, f32, f32, 72]),
        (loss.forward, [1, f16, 8, f16, 64, ids, f32, f32, f32]),
        (loss.backward, [1, f16, 8, f16, 64, ids, f32, f32, 1.0, f16, 8, f32, 64]),
        (loss.step, [1, f16, 8, f16, 64, ids, f32, 1.0, f32, f32, f16, 8, f32, 64]),
    ]
    for call, args in calls:
        call(*args)
        for i, right in enumerate(args):
            if not isinstance(right, torch.Tensor):
                continue
            for t in (torch.float32, torch.bfloat16, torch.float16, torch.float64, torch.int32, torch.int64):
                if t is right.dtype:
                    continue
                with pytest.raises(P.DqganError) as ei:
                    call(*args[:i], right.to(t), *args[i + 1:])
                assert ei.value.status == P.dqgan.ERR_INVALID_ARG
    assert len(library.calls) == len(calls)
    right, wrong = P.TensorList([(half, 8, 8)]), P.TensorList([(half, 8, 8), (f32, 8, 8)])
    places = P.TensorList([(f32, 8, 8)])
    clip.norm(right, f32)
    clip.clip(right, places, 1.0, f32)
    for call in (lambda: clip.norm(wrong, f32), lambda: clip.norm(right, half), lambda: clip.clip(right, right, 1.0),
                 lambda: clip.clip(wrong, places, 1.0), lambda: clip.clip(right, P.TensorList([]), 1.0)):
        with pytest.raises(P.DqganError) as ei:
            call()
        assert ei.value.status == P.dqgan.ERR_INVALID_ARG
    assert len(library.calls) == len(calls) + 2


def test_batches_of_the_next_token_model(P, library):  # noqa: F811
    torch = pytest.importorskip("torch")
    from paper_2010_13359_gb300.token_model import NextTokenModel
    M, n, V, C, H, L = 2, 3, 11, 4, 6, 2
    model = NextTokenModel(V, C, H, L, n, M)
    assert model.d == V * C + L * (2 * C + H * C + H + C * H + C) + 2 * C
    places = model.places()
    assert places[0][0] == V * C and places[L][1] + C == model.d and len(places[0]) == 6
    i32 = torch.int32

    def batch():
        return dict(params=torch.zeros((M, model.d + 1)), ids=torch.zeros((M, n), dtype=i32),
                    targets=torch.zeros((M, n), dtype=i32), weights=torch.ones(M * n), g=torch.zeros((M, model.d + 3)),
                    b=model.buffers("cpu"))

    model.operator(**batch())
    # embedding 2, final norm 2, loss 1; per layer: norm 2, two linear layers 4
    assert len(library.calls) == 5 + 6 * L
    model.operator(**batch() | dict(weights=None))
    library.calls.clear()
    for change in (dict(params=torch.zeros((M, model.d - 1))), dict(g=torch.zeros((M + 1, model.d))),
                   dict(params=torch.zeros((model.d, M)).t()), dict(ids=torch.zeros((M, n + 1), dtype=i32)),
                   dict(targets=torch.zeros((M, 2 * n), dtype=i32)[:, ::2]), dict(weights=torch.ones(M * n - 1))):
        with pytest.raises(ValueError):
            model.operator(**batch() | change)
    assert library.calls == []


PROGRAM = r"""
#include <cstdio>
#include "operators.cuh"

// Every unit belongs to the block that clip_block_of names, blocks follow one another without gaps, and the places
// b + m of the blocks' sums for workers are met once each and stay inside the scratch space.
int main() {
  long bad = 0, met = 0;
  for (long units = 1; units <= 40; ++units)
    for (int workers = 1; workers <= 9; ++workers)
      for (int most = 1; most <= 50; ++most) {
        const long all = units * workers;
        const int blocks = (int)(all < most ? all : most);
        static int places[128];
        for (int& p : places) p = 0;
        if (dq::clip_first_unit(units, workers, 0, blocks) != 0 || dq::clip_first_unit(units, workers, blocks, blocks) != all) ++bad;
        for (long b = 0; b < blocks; ++b) {
          const long begin = dq::clip_first_unit(units, workers, b, blocks), end = dq::clip_first_unit(units, workers, b + 1, blocks);
          if (end <= begin) ++bad;
          long known = -1;
          for (long u = begin; u < end; ++u) {
            if (dq::clip_block_of(units, workers, u, blocks) != b) ++bad;
            if (u / units != known) {
              known = u / units;
              if (b + known >= blocks + workers || places[b + known]++) ++bad;
              ++met;
            }
          }
        }
      }
  // no product of these leaves its type: 2^40 values a tensor, 4096 of them, 4096 workers
  const long units = (1L << 40) / 2048 * 4096;
  if (dq::clip_first_unit(units, 4096, 607, 608) <= 0 || dq::clip_block_of(units, 4096, units * 4096 - 1, 608) != 607) ++bad;
  std::printf("%ld bad, %ld met\n", bad, met);
  return bad || met == 0;
}
"""


def test_units_and_blocks_of_the_clipping(tmp_path):
    from paper_2010_13359_gb300 import build
    source = tmp_path / "units.cu"
    source.write_text(PROGRAM)
    exe = tmp_path / "units"
    subprocess.run([build.nvcc(), *build.ARCH, "-O1", "-std=c++17", "--expt-relaxed-constexpr", "-I", build.INCLUDE, "-I",
                    build.CSRC, str(source), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0, out.stdout
