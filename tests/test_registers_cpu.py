"""The differential prompt kernel hands registers from some warps to others: the split counts on what the launch has."""
import pathlib
import re
import shutil
import subprocess

import pytest

CSRC = pathlib.Path(__file__).resolve().parents[1] / "paper_2412_05896_b200" / "csrc"
NVCC = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"


@pytest.mark.skipif(not pathlib.Path(NVCC).exists(), reason="no compiler")
def test_the_compiler_gives_the_launch_what_the_split_counts_on(tmp_path):
    """Otherwise every call would be refused."""
    src = CSRC / "xkv_diff_prefill.cu"
    want = int(re.search(r"kLaunchRegs = (\d+)", src.read_text()).group(1))
    res = subprocess.run([NVCC, "-O3", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-Xcompiler", "-fPIC",
                          "-Xptxas", "-v", "-c", str(src), "-o", str(tmp_path / "x.o")], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    used = re.findall(r"Compiling entry function '(\w*diff_prefill_kernel\w*)'.*?Used (\d+) registers", res.stderr, re.S)
    assert len(used) == 2 and all(int(n) == want for _, n in used), used
