"""A shared array that is read or written by 8 or 16 bytes says so in its declaration: without it the compiler places the array
on its element's boundary, and an access that is not on its own is a fault (read from the sources, no GPU)."""
import glob
import os
import re

import pytest

from paper_2509_26092_gb300 import build_lib

WIDTH = {"float4": 16, "uint4": 16, "int4": 16, "float2": 8, "uint2": 8, "int2": 8, "uint64_t": 8, "double": 8}
ELEMENT = {**WIDTH, "float": 4, "int": 4, "uint32_t": 4, "uint16_t": 2, "uint8_t": 1, "char": 1}
SOURCES = sorted(glob.glob(os.path.join(build_lib.CSRC, "*.cu*")))


def arrays(text):
    """(name, the boundary that its declaration promises) of every shared array."""
    for m in re.finditer(r"__shared__\s+(?:__align__\((\d+)\)\s+)?(?:volatile\s+)?(\w+)\s+([^;(]+);", text):
        for name in re.findall(r"(\w+)\s*\[", re.sub(r"\[[^\]]*\]", "[", m.group(3))):
            yield name, max(int(m.group(1) or 1), ELEMENT.get(m.group(2), 1))


def accesses(text, name):
    """Bytes of the accesses by cast to `name`."""
    for m in re.finditer(r"reinterpret_cast<(?:const\s+)?(?:volatile\s+)?(\w+)\s*\*>\(\s*&?\s*" + name + r"\b", text):
        yield WIDTH.get(m.group(1), 1)


def functions(path):
    text = re.sub(r"//[^\n]*", "", open(path).read())
    starts = [m.start() for m in re.finditer(r"__global__|__device__ __forceinline__", text)]
    for a, b in zip(starts, starts[1:] + [len(text)]):
        yield text[a:b]


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_shared_arrays_are_aligned_as_they_are_accessed(path):
    for body in functions(path):
        for name, boundary in arrays(body):
            for width in accesses(body, name):
                assert boundary >= width, f"{os.path.basename(path)}: {name} on {boundary} bytes, accessed by {width}"


def test_the_accesses_are_seen():
    """The router's bias, and an array of which the declaration says too little."""
    route = next(p for p in SOURCES if p.endswith("route.cu"))
    assert any(16 in accesses(body, name) for body in functions(route) for name, _ in arrays(body) if name == "bias")
    text = "__shared__ float a[4], b[2][8]; __shared__ __align__(16) float c[4]; x = *reinterpret_cast<const float4*>(b + 4);"
    assert list(arrays(text)) == [("a", 4), ("b", 4), ("c", 16)]
    assert list(accesses(text, "b")) == [16] and not list(accesses(text, "a"))
