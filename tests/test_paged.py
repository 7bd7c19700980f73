"""The paged cache's stride rules (csrc/paged.h), exhaustively on small layouts. No GPU."""
from __future__ import annotations

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_extents_and_shared_elements(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("g++ not available")
    exe = tmp_path / "paged_check"
    subprocess.run([cxx, "-std=c++17", "-O2", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2607_08973_amd", "csrc"),
                    os.path.join(ROOT, "tests", "paged_check.cpp"), "-o", str(exe)], check=True)
    res = subprocess.run([str(exe)], capture_output=True, text=True)
    assert res.returncode == 0, res.stdout
    layouts, offsets = int(res.stdout.split()[1]), int(res.stdout.split()[3])
    assert layouts > 500 and offsets > 100000, res.stdout
