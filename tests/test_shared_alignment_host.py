"""Arrays in shared memory that the kernels read or write 16 bytes at a time are declared with that alignment (CPU: the sources are read).

Without it their place depends on what else a kernel declares, and a misaligned access faults."""
import glob
import os
import re

import pytest

from paper_2405_06219_b200 import build

WIDE = r"reinterpret_cast<\s*(?:const\s+)?(?:uint4|int4|float4|double2|longlong2|ulonglong2)\s*\*>\(([^;]*)"
SOURCES = sorted(glob.glob(os.path.join(build.CSRC, "*.cu")) + glob.glob(os.path.join(build.CSRC, "*.cuh")))


def narrow_arrays_read_wide(text):
    text = re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)
    names = set()
    for m in re.finditer(r"(?<!extern )__shared__\s+((?:__align__\((\d+)\)|alignas\((\d+)\))\s+)?(?:static\s+)?[\w:]+\s+([^;(]*);", text):
        if int(m[2] or m[3] or 0) < 16:
            names |= set(re.findall(r"(\w+)\s*(?:\[[^\]]*\]\s*)+", m[4]))
    # pointers into them
    for _ in range(2):
        for m in re.finditer(r"\*\s*(?:const\s+)?(\w+)\s*=\s*&?(\w+)\b", text):
            if m[2] in names:
                names.add(m[1])
    return sorted(n for n in names for m in re.finditer(WIDE, text) if re.search(rf"\b{n}\b", m[1]))


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_wide_accesses_of_shared_arrays_are_aligned(path):
    assert narrow_arrays_read_wide(open(path).read()) == []


def test_the_reader_sees_what_it_looks_for():
    declared = "__shared__ %s int a[2][8], b;\nint *p = a[1];\nconst int4 v = *reinterpret_cast<const int4 *>(f(p, 3) + 4);\n"
    assert narrow_arrays_read_wide(declared % "") == ["p"]
    assert narrow_arrays_read_wide(declared % "__align__(8)") == ["p"]
    assert narrow_arrays_read_wide(declared % "__align__(16)") == []
