"""Arrays in LDS that are read or written sixteen bytes at a time say so: a float array alone is aligned to four, and what lies before it decides the rest."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2602_01410_amd", "csrc")
# by store8 / load8, or through a pointer to four floats or words
WIDE = r"(?:(?:store8|load8)\(&?|(?:float4|uint4|v4f|v4u) ?\*>?\(?\)?\(?&?)%s\b"


def unaligned(text):
    found = set()
    for kernel in text.split("__global__"):                      # (a name is one array in a kernel, and may be another in the next)
        arrays = re.findall(r"__shared__\s+((?:__attribute__\(\(aligned\(\d+\)\)\)\s+)?)(?:float|int|unsigned|uint8_t|uint16_t|uint32_t)\s+(\w+)\[", kernel)
        found |= {name for attribute, name in arrays if not attribute and re.search(WIDE % name, kernel)}
    return sorted(found)


def test_scan():
    assert unaligned("__shared__ float a[8];\n store8(&a[0], f);") == ["a"]
    assert unaligned("__shared__ float a[8];\n x = a[3];") == []
    assert unaligned("__shared__ int b[4];\n *reinterpret_cast<uint4*>(&b[0]) = v;") == ["b"]
    assert unaligned("__shared__ __attribute__((aligned(16))) float a[8];\n store8(&a[0], f);") == []


@pytest.mark.parametrize("name", sorted(n for n in os.listdir(CSRC) if n.endswith((".hip", ".h"))))
def test_source(name):
    with open(os.path.join(CSRC, name)) as f:
        assert unaligned(f.read()) == []
