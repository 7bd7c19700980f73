"""sifar_route refuses, on the host and before any device call, what its contract
leaves out. No GPU is used."""
from __future__ import annotations

import ctypes
import os
import re
import shutil
import subprocess

import pytest
import torch

import paper_2607_08973_amd as S

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include",
                      "sifar.h")
T, E, K = 4, 64, 8
BASE = 1 << 20  # addresses that a refused call never touches


def args(**kw):
    a = S.sifar_route_args(
        dtype=S.SIFAR_BF16, tokens=T, experts=E, topk=K, score=S.SIFAR_ROUTE_SIGMOID, groups=8,
        top_groups=4, group_top=2, renorm=1, scale=1.0, logits=BASE, logits_stride=E,
        bias=2 * BASE, ids=3 * BASE, weights=4 * BASE)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


BAD = [
    dict(dtype=3), dict(dtype=-1), dict(tokens=-1), dict(tokens=S.SIFAR_ROWS_MAX_TOKENS + 1),
    dict(experts=0), dict(experts=1032), dict(experts=63), dict(topk=0), dict(topk=33),
    dict(experts=4, groups=1, top_groups=1, topk=5), dict(score=2), dict(score=-1),
    dict(groups=0), dict(groups=64), dict(groups=7), dict(top_groups=0), dict(top_groups=9),
    dict(group_top=0), dict(group_top=3), dict(renorm=2),
    dict(logits=None), dict(ids=None), dict(weights=None),
    dict(logits=BASE + 1), dict(bias=2 * BASE + 2), dict(ids=3 * BASE + 2),
    dict(weights=4 * BASE + 1), dict(logits_stride=E - 1), dict(logits_stride=-E),
    dict(ids=4 * BASE + 4), dict(ids=BASE), dict(weights=2 * BASE + 4), dict(weights=BASE + 128),
]


@pytest.mark.parametrize("kw", BAD, ids=lambda kw: ",".join(f"{k}={v}" for k, v in kw.items()))
def test_refused_by_the_library(kw):
    assert S.load().sifar_route(ctypes.byref(args(**kw)), None) == S.SIFAR_EINVAL


def test_null_and_empty_calls():
    L = S.load()
    assert L.sifar_route(None, None) == S.SIFAR_EINVAL
    a = args(tokens=0, logits=None, ids=None, weights=None)
    assert L.sifar_route(ctypes.byref(a), None) == S.SIFAR_OK


def test_layout_matches_a_c_compiler(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    cls = S.sifar_route_args
    body = re.search(r"typedef struct \{([^{}]*)\} sifar_route_args;",
                     open(HEADER).read()).group(1)
    assert re.findall(r"\b(\w+);", body) == [f for f, _ in cls._fields_]
    assert S._ROUTE.size == ctypes.sizeof(cls)
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "sifar.h"', "int main(void) {",
             '    printf("size %zu\\n", sizeof(sifar_route_args));']
    lines += [f'    printf("{f} %zu\\n", offsetof(sifar_route_args, {f}));' for f, _ in cls._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["    return 0;", "}"]) + "\n")
    subprocess.run([cc, "-std=c11", "-I", os.path.dirname(HEADER), str(src), "-o", str(exe)],
                   check=True)
    for line in subprocess.run([str(exe)], check=True, capture_output=True,
                               text=True).stdout.split("\n")[:-1]:
        what, value = line.split()
        assert int(value) == (ctypes.sizeof(cls) if what == "size" else getattr(cls, what).offset)


class Recorder:
    """Stands in for the library where host tensors play device tensors."""

    def __init__(self):
        self.calls = []

    def sifar_route(self, packed, stream):
        self.calls.append(S.sifar_route_args.from_buffer_copy(packed))
        return 0

    def sifar_strerror(self, code):
        return b""


@pytest.fixture
def recorder(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(S, "_lib", r)
    monkeypatch.setattr(S, "_gpu", lambda fn, name, t: -1)   # a host tensor's device
    monkeypatch.setattr(S, "_row_stream", lambda stream, dev: 0)
    return r


def tensors(**kw):
    a = dict(logits=torch.zeros(T, 2 * E)[:, :E], ids=torch.zeros(T, K, dtype=torch.int32),
             weights=torch.zeros(T, K), bias=torch.zeros(E))
    a.update(kw)
    return a


def test_marshalling(recorder):
    t = tensors()
    S.sifar_route(**t, score="sigmoid", groups=8, top_groups=4, group_top=2, renorm=False,
                  scale=2.5)
    c = recorder.calls[0]
    assert (c.dtype, c.tokens, c.experts, c.topk, c.score, c.groups, c.top_groups, c.group_top,
            c.renorm, c.scale, c.logits_stride) == (
        S.SIFAR_FP32, T, E, K, S.SIFAR_ROUTE_SIGMOID, 8, 4, 2, 0, 2.5, 2 * E)
    for name in ("logits", "ids", "weights", "bias"):
        assert getattr(c, name) == t[name].data_ptr(), name


@pytest.mark.parametrize("kw", [
    dict(logits=torch.zeros(T, E, dtype=torch.float64)), dict(logits=torch.zeros(E)),
    dict(logits=torch.zeros(E, T).t()), dict(logits=torch.zeros(T, 1032)),
    dict(ids=torch.zeros(T, K, dtype=torch.int64)), dict(ids=torch.zeros(T + 1, K, dtype=torch.int32)),
    dict(ids=torch.zeros(T, 2 * K, dtype=torch.int32)[:, :K]),
    dict(weights=torch.zeros(T, K + 1)), dict(weights=torch.zeros(T, K, dtype=torch.bfloat16)),
    dict(bias=torch.zeros(E, dtype=torch.bfloat16)), dict(bias=torch.zeros(E + 1)),
    dict(score="relu"), dict(score=None),
], ids=range(13))
def test_refused_by_the_binding(recorder, kw):
    with pytest.raises(S.SifarError) as e:
        S.sifar_route(**tensors(**kw))
    assert e.value.code == S.SIFAR_EINVAL and not recorder.calls


def test_host_tensors_are_refused():
    with pytest.raises(S.SifarError) as e:
        S.sifar_route(**tensors())
    assert e.value.code == S.SIFAR_EINVAL
