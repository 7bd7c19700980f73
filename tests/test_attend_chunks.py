"""The chunks that sifar_paged_attention's kernels take (csrc/attend_plan.h). No GPU."""
from __future__ import annotations

import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_08973_amd", "csrc")


def test_chunks_fit_their_places(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("g++ not available")
    exe = tmp_path / "attend_chunk_check"
    subprocess.run([cxx, "-std=c++17", "-O2", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"),
                    "-I", CSRC, os.path.join(ROOT, "tests", "attend_chunk_check.cpp"), "-o", str(exe)],
                   check=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True)
    assert res.returncode == 0, res.stdout
    assert res.stdout.startswith("checked 300000 ")


def test_the_kernel_takes_its_chunks_from_there():
    source = open(os.path.join(CSRC, "attention.hip")).read()
    assert re.findall(r"\.chunk = (\w+)\(", source) == ["chunk_of"]
    assert len(re.findall(r"\.chunk\s*=[^=]", source)) == 1
