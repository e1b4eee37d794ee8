"""Registers of the kernel for few rows, as the assembler reports them: its instances share a template, and are at the limit."""
import os
import re
import subprocess

import pytest

from paper_2605_14513_b200 import build


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """(rows / 8, e4m3, to be done again, cross attention) -> bytes of stack, of spills stored and loaded"""
    out = str(tmp_path_factory.mktemp("rows") / "cache_rows.o")
    text = subprocess.run([build.nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17", "-Xcompiler", "-fPIC", "-Xptxas=-v",
                           "-I", os.path.join(build.ROOT, "include"), "-c", os.path.join(build.HERE, "csrc", "cache_rows.cu"), "-o", out],
                          check=True, capture_output=True, text=True).stderr
    found = re.findall(r"cache_rows_kernelILi(\d)ELb(\d)ELb(\d)ELb(\d)E.*?(\d+) bytes stack frame, (\d+) bytes spill stores, (\d+) bytes spill loads", text, re.S)
    return {tuple(int(x) for x in f[:4]): tuple(int(x) for x in f[4:]) for f in found}


def test_kernels_of_few_rows_do_not_spill(kernels):
    assert len(kernels) == 7
    for (rows, e4m3, redo, cross), bytes_of in kernels.items():
        # (what is done again, as a rule nothing, may: 40 bytes)
        assert sum(bytes_of) == 0 or (redo and sum(bytes_of[1:]) <= 40), (rows, e4m3, redo, cross, bytes_of)
