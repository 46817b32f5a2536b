"""Arrays in shared memory that the kernels read or write in pieces wider than their elements say so in their declaration: without that
their place, and with it whether such an access faults, is up to the compiler."""
import re
from pathlib import Path

import pytest

CSRC = Path(__file__).parent.parent / "paper_2510_07535_b200" / "csrc"
SIZE = {"float4": 16, "uint4": 16, "int4": 16, "ulonglong2": 16, "longlong2": 16, "float2": 8, "uint2": 8, "int2": 8, "uint64_t": 8}
OF = {**SIZE, "float": 4, "int": 4, "unsigned": 4, "uint32_t": 4, "int32_t": 4, "unsigned long long": 8, "long long": 8, "double": 8, "char": 1,
      "unsigned char": 1, "short": 2}
FILES = sorted(f.name for f in CSRC.glob("*.cu*"))


def shared_arrays(text):
    """(name, size of an element, stated alignment) of every array that a `__shared__` declaration names."""
    for align, kind, names in re.findall(r"(?<!extern )__shared__ (?:__align__\((\d+)\) )?((?:unsigned long long|long long|unsigned char|\w+)) ([^;]*);", text):
        for name in re.findall(r"(\w+)\[", names):
            yield name, OF.get(kind, 1), int(align or 0)


@pytest.mark.parametrize("file", FILES)
def test_wide_accesses_are_to_aligned_arrays(file):
    text = re.sub(r"//[^\n]*|/\*.*?\*/", "", (CSRC / file).read_text(), flags=re.S)
    arrays = {name: (size, align) for name, size, align in shared_arrays(text)}
    for kind, name in re.findall(r"reinterpret_cast<(?:const )?(?:volatile )?(\w+)\*>\(&?(\w+)", text):
        if name in arrays and kind in SIZE:
            size, align = arrays[name]
            assert max(size, align) >= SIZE[kind], (name, kind)


def test_what_the_search_finds():
    names = {name for f in FILES for name, _, _ in shared_arrays((CSRC / f).read_text())}
    assert {"s_max", "s_groups", "s_keys", "s_rows", "s_path", "s_most"} <= names
