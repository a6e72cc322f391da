"""What can be seen from the kernels' sources."""
import pathlib
import re

import pytest

CSRC = pathlib.Path(__file__).resolve().parents[1] / "paper_2412_05896_b200" / "csrc"
WIDTH = {"2": 8, "4": 16}


@pytest.mark.parametrize("path", sorted(CSRC.glob("*.cu")), ids=lambda p: p.name)
def test_dynamic_shared_memory_read_in_vectors_is_aligned(path):
    """Otherwise the static arrays in front of it and the compiler decide where it begins."""
    text = path.read_text()
    for m in re.finditer(r"extern __shared__ ([^;\[]*?)(\w+)\[\];", text):
        words = re.findall(r"reinterpret_cast<(?:const )?(?:u?int|float)([24])\s*\*>\(\s*" + m.group(2) + r"\b", text)
        align = re.search(r"__align__\((\d+)\)", m.group(1))
        assert not words or (align and int(align.group(1)) >= max(WIDTH[w] for w in words)), m.group(0)


def test_page_plans_read_what_the_launch_before_writes_by_ordinary_loads():
    """Their launches are in place before the launch ahead of them ends, so what that one writes (lengths, say) is not read-only for
    them; copies by a caller's page ids are launched after it."""
    text = (CSRC / "xkv_pages.cu").read_text()
    text = re.sub(r"//.*", "", text)
    copies = re.search(r"copy_pages_kernel\(.*?\n}\n", text, re.S).group(0)
    assert "__ldg" in copies and "__ldg" not in text.replace(copies, "") and "ld.global.nc" not in text
