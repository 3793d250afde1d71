"""Calls of an operator run on the device that was current when it was made, where its scratch is.  A machine with one
GPU cannot show a call on another, so the rule is held to the source: the check that every computing call begins with
compares the devices, and creation keeps the device before it allocates.
"""
from __future__ import annotations

import os
import re

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2010_13359_gb300", "csrc",
                      "operators.cu")


def function(text, head):
    at = text.index(head)
    return text[at:text.index("\n}", at)]


def test_every_call_that_computes_checks_the_device():
    text = re.sub(r"//[^\n]*", "", open(SOURCE).read())
    check = function(text, "int check(dqgan_operator* op, Kind kind")
    assert "cudaGetDevice(&device)" in check and "device != op->device" in check
    create = function(text, "int create(Kind kind")
    assert create.index("cudaGetDevice(&op->device)") < create.index("device_allocate")
    for call in ("dqgan_layer_norm_forward", "dqgan_layer_norm_backward", "dqgan_embedding_forward", "dqgan_embedding_backward",
                 "dqgan_linear_forward", "dqgan_linear_backward", "distillation", "token_loss", "check_clip"):
        body = function(text, f"int {call}(dqgan_operator* op")
        assert re.search(r"\{\s*(?:using \S+ = \S+;\s*)?if \(int r = check\(op, Kind::", body), call
