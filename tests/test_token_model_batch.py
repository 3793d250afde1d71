"""What TokenModel.operator takes for a batch, on the host: the kernels get addresses and one stride, so a batch that is
laid out otherwise must be refused and not read wrongly."""
from __future__ import annotations

import pytest

from test_operators_abi import P  # noqa: F401

torch = pytest.importorskip("torch")

M, N, V, C, K = 2, 3, 11, 4, 5


@pytest.fixture
def model(P, monkeypatch):  # noqa: F811
    """A model over a library that only counts its calls."""
    from paper_2010_13359_gb300 import operators, token_model
    calls = []

    class Library:
        def __getattr__(self, name):
            if name.endswith(("create", "destroy")):
                return lambda *args: 0
            return lambda *args: calls.append(name) or 0

    monkeypatch.setattr(operators, "load_library", lambda: Library())
    m = token_model.TokenModel(V, C, N, M, K)
    m.calls = calls
    return m


def batch(model):
    d = model.d
    return dict(params=torch.zeros((M, d + 1)), ids=torch.zeros((M, N), dtype=torch.int32),
                teacher_ids=torch.zeros((M * N, K), dtype=torch.int32), teacher_values=torch.zeros((M * N, K)),
                weights=torch.ones(M * N), g=torch.zeros((M, d + 3)), b=model.buffers("cpu"))


def test_batches_that_are_taken(model):
    i32 = torch.int32
    for change in ({}, dict(weights=None), dict(ids=torch.zeros(M * N, dtype=i32)),
                   dict(teacher_ids=torch.zeros((M * N, K + 2), dtype=i32), teacher_values=torch.zeros((M * N, K + 2))),
                   dict(teacher_ids=torch.zeros((M * N, K + 2), dtype=i32)[:, :K],
                        teacher_values=torch.zeros((M * N, K + 2))[:, 1:K + 1]),
                   dict(params=torch.zeros((1, model.d)).expand(M, model.d))):
        model.calls.clear()
        model.operator(**batch(model) | change)
        assert len(model.calls) == 5


@pytest.mark.parametrize("what,change", [
    ("ids", lambda d: torch.zeros((M, N + 1), dtype=torch.int32)[:, :N]),  # a batch without its last token
    ("ids", lambda d: torch.zeros((N, M), dtype=torch.int32).t()),
    ("ids", lambda d: torch.zeros((M, N - 1), dtype=torch.int32)),
    ("teacher_values", lambda d: torch.zeros((M * N, K + 3))[:, :K]),  # another stride than the ids'
    ("teacher_values", lambda d: torch.zeros((K, M * N)).t()),
    ("teacher_values", lambda d: torch.zeros((M * N - 1, K))),
    ("teacher_ids", lambda d: torch.zeros((M * N, K + 3), dtype=torch.int32)[:, :K]),
    ("teacher_ids", lambda d: torch.zeros((M, N, K), dtype=torch.int32)),
    ("teacher_ids", lambda d: torch.zeros((M * N, K - 1), dtype=torch.int32)),
    ("weights", lambda d: torch.ones(2 * M * N)[::2]),
    ("weights", lambda d: torch.ones(M * N - 1)),
    ("params", lambda d: torch.zeros((M, d - 1))),  # no room for the last bias
    ("params", lambda d: torch.zeros((M + 1, d))),
    ("g", lambda d: torch.zeros((M, d - 1))),
    ("g", lambda d: torch.zeros((M - 1, d))),
])
def test_batches_that_are_refused(model, what, change):
    with pytest.raises(ValueError, match=what.split("_")[0]):
        model.operator(**batch(model) | {what: change(model.d)})
    assert model.calls == []
