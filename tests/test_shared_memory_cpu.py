"""Dynamic shared memory that a kernel reads in vectors is declared with their alignment: otherwise the static arrays in front of it
and the compiler decide where it begins."""
import pathlib
import re

import pytest

CSRC = pathlib.Path(__file__).resolve().parents[1] / "paper_2412_05896_b200" / "csrc"
WIDTH = {"2": 8, "4": 16}


@pytest.mark.parametrize("path", sorted(CSRC.glob("*.cu")), ids=lambda p: p.name)
def test_dynamic_shared_memory_read_in_vectors_is_aligned(path):
    text = path.read_text()
    for m in re.finditer(r"extern __shared__ ([^;\[]*?)(\w+)\[\];", text):
        words = re.findall(r"reinterpret_cast<(?:const )?(?:u?int|float)([24])\s*\*>\(\s*" + m.group(2) + r"\b", text)
        align = re.search(r"__align__\((\d+)\)", m.group(1))
        assert not words or (align and int(align.group(1)) >= max(WIDTH[w] for w in words)), m.group(0)
