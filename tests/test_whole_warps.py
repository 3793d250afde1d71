"""Tensor memory is read, allocated and freed by instructions that a warp executes as one (.sync.aligned).  Lanes that
decide for themselves whether a wait ended, or leave an epilogue at different times, may reach such an instruction
apart, which a run shows only where the compiler happens not to join them again.  So the rule is held to the source of
the products' kernel: a wait before such an instruction is decided by all lanes together, and every branch that single
lanes take or leave is followed by a warp barrier.
"""
from __future__ import annotations

import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2010_13359_gb300", "csrc")
WAIT = re.compile(r"mbar_wait_bounded\(")
TOGETHER = re.compile(r"__all_sync\(kFullMask,\s*mbar_wait_bounded\(")


def body(text, name):
    """The definition of `name`, comments left out, up to the brace that closes it at the start of a line."""
    text = re.sub(r"//[^\n]*", "", text)
    at = re.search(r"\b" + name + r"\([^;{]*\)\s*\{", text).start()
    return text[at:text.index("\n}", at)]


def lone_decisions(kernel):
    """Waits of the summing warps that a lane decides for itself, and whole-warp steps without a barrier before them."""
    found = []
    summing = kernel[kernel.index("setmaxnreg.inc"):]
    if len(WAIT.findall(summing)) != len(TOGETHER.findall(summing)):
        found.append("wait")
    load = summing.index("tensor_load32(")
    wait = summing.index("mbar_wait_bounded(")
    if not wait < summing.rfind("__syncwarp();", 0, load):
        found.append("load")
    run = summing.index("Epilogue::template run")
    if not re.match(r"[^;]*;\s*\}\s*__syncwarp\(\);", summing[run:]):
        found.append("epilogue")
    end = re.search(r"\}\s*__syncwarp\(\);\s*tensor_fence_before\(\);\s*__syncthreads\(\);", summing)
    if not (end and run < end.start() < summing.index("tensor_memory_free")):
        found.append("end")
    start = kernel[:kernel.index("tensor_memory_allocate")]
    if not start.rstrip().endswith("__syncwarp();\n  if (warp == 2)"):
        found.append("start")
    return found


def test_the_products_kernel_reads_tensor_memory_by_whole_warps():
    assert lone_decisions(body(open(os.path.join(CSRC, "product_kernel.cuh")).read(), "product_kernel")) == []


def test_the_rule_sees_a_lane_that_decides_alone():
    text = body(open(os.path.join(CSRC, "product_kernel.cuh")).read(), "product_kernel")
    alone = re.sub(r"__all_sync\(kFullMask,\s*(mbar_wait_bounded\([^;]*?\))\)\)\) break;", r"\1)) break;", text)
    assert alone != text and lone_decisions(alone) == ["wait"]
    assert lone_decisions(text.replace("__syncwarp();", "")) == ["load", "epilogue", "end", "start"]
