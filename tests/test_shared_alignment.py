"""A shared array of single values that is read or written 16 bytes at a time has to say that it starts on a 16-byte
boundary: the compiler may put it on any boundary of its element, and where it does a run shows a misaligned
address.  The rule is held to the source."""
from __future__ import annotations

import glob
import os
import re

import pytest

from test_cluster_start import CSRC, functions

ARRAY = re.compile(r"__shared__\s+(?:float|int32_t|uint32_t|int|uint16_t|unsigned char)\s+(.*?);")
WIDE = r"reinterpret_cast<(?:const )?(?:float4|uint4|int4)\s?\*>\(([^()]*)"


def unaligned(text):
    text = re.sub(r"[ \t]*(?://[^\n]*)?$", "", text, flags=re.M)
    found = []
    for body in functions(text):
        for declared in ARRAY.findall(body):
            for name in re.findall(r"(\w+)\s*(?:\[[^\]]*\])+", declared):
                # the array, and pointers that are set from it
                names = {name} | set(re.findall(rf"\*\s*(?:const\s+)?(\w+)\s*=\s*[^;]*\b{name}\b", body))
                if any(re.search(rf"\b{n}\b", at) for at in re.findall(WIDE, body) for n in names):
                    found.append(name)
    return found


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "*.cu*"))), ids=os.path.basename)
def test_shared_arrays_read_in_packs_are_aligned(path):
    assert unaligned(open(path).read()) == []


def test_the_rule_sees_an_unaligned_array():
    body = "__global__ void k() {{\n  __shared__ {} float a[64], b[2];\n  float* p = a + 4;\n  *reinterpret_cast<float4*>(p) = v;\n}}\n"
    assert unaligned(body.format("")) == ["a"]
    assert unaligned(body.format("__align__(16)")) == []
