"""The byte counters that bench.py quotes are keyed by a hash of the kernels' sources: every
file that holds a counted kernel, or that such a file includes, has to be among them."""

import os
import re

import pytest

from bench import KERNEL_SOURCES
from profile_bench import ENTRY_KERNELS

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2505_07680_amd", "csrc")
TEXT = {n: open(os.path.join(CSRC, n)).read() for n in os.listdir(CSRC)}


def _with_includes(names):
    found, todo = set(), list(names)
    while todo:
        n = todo.pop()
        if n in TEXT and n not in found:
            found.add(n)
            todo += re.findall(r'#include "([^"]+)"', TEXT[n])
    return found


@pytest.mark.parametrize("entry", sorted(ENTRY_KERNELS))
def test_every_source_of_a_counted_kernel_is_hashed(entry):
    listed = set(KERNEL_SOURCES[entry])
    assert listed <= set(TEXT)
    for kernel in ENTRY_KERNELS[entry]:
        holders = {n for n, t in TEXT.items() if re.search(rf"\b{kernel}\s*\([^)]*\)\s*{{", re.sub(r"//.*", "", t))}
        assert holders, f"{kernel} is defined nowhere"
        assert holders <= listed, f"{kernel} is in {sorted(holders)}"
    assert _with_includes(listed) <= listed
