"""Registers of the layer blocks' kernels, checked at compile time: nothing in scratch
memory, and no more registers than the waves that hide their loads leave. No GPU is used."""
from __future__ import annotations

import pytest

from test_row_kernel_resources import resources


@pytest.mark.parametrize("source,kernels,vgprs", [
    ("cache_append.hip", 12, 64), ("attention.hip", 30, 512), ("experts.hip", 6, 184),
])
def test_registers(source, kernels, vgprs, tmp_path):
    found = resources(source, tmp_path)
    assert len(found) == kernels, sorted(found)
    for name, (vgpr, spill, scratch) in found.items():
        assert vgpr <= vgprs and spill == 0 and scratch == 0, (name, vgpr, spill, scratch)
        # two waves a SIMD of the attention's kernels, but of fp32 heads above 128
        if "attend_kernel" in name and "ILi2ELi256E" not in name:
            assert vgpr <= 256, (name, vgpr)
