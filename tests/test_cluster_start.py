"""A block may touch the shared memory of another block of its cluster only once that block is known to run,
which a cluster barrier passed before the first access guarantees.  A run shows nothing as long as the blocks
start close together, so the rule is held to the source: in a function that loads from or stores to
shared::cluster, the wait of a cluster barrier stands before the first such access.
"""
from __future__ import annotations

import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2010_13359_gb300", "csrc")
REMOTE = re.compile(r'"(?:ld|st|red|atom)\.[\w.]*shared::cluster')
WAIT = re.compile(r"barrier\.cluster\.wait|\bcluster_wait\(\)|\.sync\(\);")


def functions(text):
    """The file's function definitions that stand at the start of a line, each up to its closing brace."""
    return re.findall(r"^(?!namespace|struct|\}|#)\S[^\n]*[^;}\n](?:\n(?!\})[^\n]*)*\n\}", text, re.M)


def early_accesses(text):
    text = re.sub(r"[ \t]*(?://[^\n]*)?$", "", text, flags=re.M)
    found = []
    for body in functions(text):
        first = REMOTE.search(body)
        wait = WAIT.search(body)
        if first and not (wait and wait.start() < first.start()):
            found.append(body[:body.index("{")])
    return found


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "*.cu*"))), ids=os.path.basename)
def test_remote_shared_memory_is_touched_after_a_cluster_barrier(path):
    assert early_accesses(open(path).read()) == []


def test_the_rule_sees_an_early_access():
    early = '__global__ void k() {\n  asm volatile("st.shared::cluster.u32 [%0], %1;");\n  cluster_wait();\n}\n'
    late = '__global__ void k() {\n  cluster_wait();\n  asm volatile("st.shared::cluster.u32 [%0], %1;");\n}\n'
    assert len(early_accesses(early)) == 1 and early_accesses(late) == []
