"""Arrays in shared memory that kernels read or write 16 bytes at a time are declared
on 16-byte boundaries: an array of floats alone is only promised its element's."""
import glob
import os
import re

import pytest

import paper_2609_09020_gb300 as package

CSRC = os.path.join(os.path.dirname(os.path.abspath(package.__file__)), "csrc")
WIDE = {"float4": 16, "uint4": 16, "float2": 8, "uint2": 8}
ELEMENT = {"double": 8, "uint4": 16, "float4": 16, "int4": 16, "float2": 8, "uint2": 8, "unsigned long long": 8}


def faults(text):
    """Names of __shared__ arrays that are cast to a wider type than their declaration's alignment."""
    found = []
    for m in re.finditer(r"__shared__\s+(__align__\((\d+)\)\s+)?((?:unsigned |long )*\w+)\s+(\w+)\[", text):
        align = int(m.group(2) or ELEMENT.get(m.group(3), 4))
        name = m.group(4)
        for wide, bytes_ in WIDE.items():
            cast = rf"reinterpret_cast<(?:const )?{wide}\s*\*>\(&?{name}\b"
            if bytes_ > align and re.search(cast, text):
                found.append((name, wide))
    return found


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(CSRC, "*.cu*"))), ids=os.path.basename)
def test_declarations(path):
    assert faults(open(path).read()) == []


def test_a_fault_is_seen():
    bad = "__shared__ float a[4];\n f = *reinterpret_cast<const float4*>(&a[0]);"
    assert faults(bad) == [("a", "float4")]
    assert faults(bad.replace("float a", "__align__(16) float a")) == []
