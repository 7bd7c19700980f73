"""csrc/exp2.h, the 64-bit 2^t of the row operators, against 80-bit arithmetic on
the host: the bound that its comment states."""
from __future__ import annotations

import os
import shutil
import subprocess

import pytest

from paper_2607_08973_amd import build as B

HERE = os.path.dirname(os.path.abspath(__file__))


def test_error_of_exp2(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    exe = tmp_path / "exp2_check"
    subprocess.run([cxx, "-O2", "-std=c++17", "-ffp-contract=off", "-Wall", "-Wextra", "-Werror",
                    "-I", B.CSRC, os.path.join(HERE, "exp2_check.cpp"), "-o", str(exe)],
                   check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stdout
