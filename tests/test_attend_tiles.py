"""The shapes of tests/test_gpu_layer_loops.py turn the attention's loop many times: ten tiles
and more a wave for every type and head width, past the caches and through them. No GPU."""
from __future__ import annotations

import os
import shutil
import subprocess

import pytest

import paper_2607_08973_amd as S
import test_gpu_layer_loops as loops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_many_tiles_a_wave(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("g++ not available")
    exe = tmp_path / "attend_tiles"
    subprocess.run([cxx, "-std=c++17", "-O2", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2607_08973_amd", "csrc"),
                    os.path.join(ROOT, "tests", "attend_tiles.cpp"), "-o", str(exe)], check=True)
    shapes = [(t, *g, d, r) for t in (S.SIFAR_BF16, S.SIFAR_FP16, S.SIFAR_FP32)
              for g in loops.GROUPS for d in loops.DIMS for r in loops.REACH]
    res = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, s)) for s in shapes),
                         capture_output=True, text=True, check=True)
    for shape, line in zip(shapes, res.stdout.split("\n")):
        tiles, once = map(int, line.split())
        assert tiles >= 10, (shape, tiles)
        assert once == (shape[2] == 4 and shape[4] in (64, 128, 256)), shape
    assert len(res.stdout.split()) == 2 * len(shapes)
