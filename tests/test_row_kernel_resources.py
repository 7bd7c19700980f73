"""Registers of the row operators' kernels, checked at compile time: nothing in scratch
memory, and workgroups of 1024 threads within the 128 registers that they get. No GPU
is used."""
from __future__ import annotations

import os
import re
import shutil
import subprocess

import pytest

from paper_2607_08973_amd import build as B


def resources(source, tmp):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    out = tmp / "kernels.s"
    flags = [f for f in B.FLAGS if f not in ("-fPIC", "-shared")]
    res = subprocess.run([hipcc, *flags, "--cuda-device-only", "-S", "-I", B.INCLUDE, "-I", B.CSRC,
                          os.path.join(B.CSRC, source), "-o", str(out)], capture_output=True,
                         text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    found = {}
    for m in re.finditer(r"\.name:\s+(\S+)\n(.*?)(?=\n\s+- \.|\n\s+-\s|\Z)", out.read_text(), re.S):
        n = lambda key: int((re.search(rf"\.{key}:\s+(\d+)", m.group(2)) or [0, -1])[1])
        if n("vgpr_count") >= 0:
            found[m.group(1)] = (n("vgpr_count"), n("vgpr_spill_count"),
                                 n("private_segment_fixed_size"))
    return found


@pytest.mark.parametrize("source,kernels,vgprs", [
    ("block_norm.hip", 20, 128), ("route.hip", 33, 256), ("sample.hip", 12, 128),
])
def test_registers(source, kernels, vgprs, tmp_path):
    found = resources(source, tmp_path)
    assert len(found) == kernels, sorted(found)
    for name, (vgpr, spill, scratch) in found.items():
        assert vgpr <= vgprs and spill == 0 and scratch == 0, (name, vgpr, spill, scratch)
