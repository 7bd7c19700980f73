"""sifar_sample refuses, on the host and before any device call, what its contract
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
T, V = 4, 1500
BASE = 1 << 20  # addresses that a refused call never touches
NEED = S.sifar_sample_workspace(T, V)


def args(**kw):
    a = S.sifar_sample_args(
        dtype=S.SIFAR_BF16, tokens=T, vocab=V, logits=BASE, logits_stride=V, uniform=2 * BASE,
        temperature=3 * BASE, top_k=4 * BASE, top_p=5 * BASE, min_p=6 * BASE, out=7 * BASE,
        probs=8 * BASE, workspace=9 * BASE, workspace_bytes=NEED)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


BAD = [
    dict(dtype=3), dict(dtype=-1), dict(tokens=-1), dict(tokens=S.SIFAR_ROWS_MAX_TOKENS + 1),
    dict(vocab=0), dict(vocab=S.SIFAR_SAMPLE_MAX_VOCAB + 1),
    dict(logits=None), dict(uniform=None), dict(out=None), dict(workspace=None),
    dict(logits=BASE + 1), dict(uniform=2 * BASE + 2), dict(temperature=3 * BASE + 1),
    dict(top_k=4 * BASE + 2), dict(top_p=5 * BASE + 2), dict(min_p=6 * BASE + 2),
    dict(out=7 * BASE + 2), dict(probs=8 * BASE + 2), dict(workspace=9 * BASE + 8),
    dict(workspace_bytes=NEED - 1), dict(workspace_bytes=-1), dict(logits_stride=V - 1),
    dict(logits_stride=-V),
    dict(out=8 * BASE + 4), dict(out=2 * BASE), dict(probs=BASE + 1000), dict(out=9 * BASE + 16),
    dict(probs=3 * BASE + 12), dict(workspace=BASE), dict(workspace=4 * BASE - 16),
]


@pytest.mark.parametrize("kw", BAD, ids=lambda kw: ",".join(f"{k}={v}" for k, v in kw.items()))
def test_refused_by_the_library(kw):
    assert S.load().sifar_sample(ctypes.byref(args(**kw)), None) == S.SIFAR_EINVAL


def test_null_and_empty_calls():
    L = S.load()
    assert L.sifar_sample(None, None) == S.SIFAR_EINVAL
    a = args(tokens=0, logits=None, uniform=None, out=None, workspace=None)
    assert L.sifar_sample(ctypes.byref(a), None) == S.SIFAR_OK


def test_workspace_sizes():
    assert S.sifar_sample_workspace(0, 1) == 0
    assert 0 < S.sifar_sample_workspace(1, 1) <= S.sifar_sample_workspace(1, 1024)
    assert S.sifar_sample_workspace(1, 1024) < S.sifar_sample_workspace(1, 1025)
    for v in (1, 65535, 65536, 128256, 1 << 20):     # more tokens or logits never need less
        need = [S.sifar_sample_workspace(t, v) for t in (0, 1, 2, 63, 64, 65, 256, 4096)]
        assert need == sorted(need)
        assert need[3] <= S.sifar_sample_workspace(63, min(v + 1, 1 << 20))
    big = S.sifar_sample_workspace(S.SIFAR_ROWS_MAX_TOKENS, S.SIFAR_SAMPLE_MAX_VOCAB)
    assert big >= 1 << 30    # past 32 bits of bytes, not wrapped
    for t, v in ((-1, 5), (5, 0), (5, -1), (1 << 21, 5), (5, 1 << 21), (1 << 40, 5)):
        with pytest.raises(S.SifarError) as e:
            S.sifar_sample_workspace(t, v)
        assert e.value.code == S.SIFAR_EINVAL


def test_layout_matches_a_c_compiler(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    cls = S.sifar_sample_args
    body = re.search(r"typedef struct \{([^{}]*)\} sifar_sample_args;",
                     open(HEADER).read()).group(1)
    assert re.findall(r"\b(\w+);", body) == [f for f, _ in cls._fields_]
    assert S._SAMPLE.size == ctypes.sizeof(cls)
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "sifar.h"', "int main(void) {",
             '    printf("size %zu\\n", sizeof(sifar_sample_args));']
    lines += [f'    printf("{f} %zu\\n", offsetof(sifar_sample_args, {f}));'
              for f, _ in cls._fields_]
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

    def sifar_sample(self, packed, stream):
        self.calls.append(S.sifar_sample_args.from_buffer_copy(packed))
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
    z = lambda dt=torch.float32: torch.zeros(T, dtype=dt)
    a = dict(logits=torch.zeros(T, V + 3, dtype=torch.float16)[:, :V], uniform=z(),
             out=z(torch.int32), workspace=torch.zeros(NEED, dtype=torch.uint8), probs=z(),
             temperature=z(), top_k=z(torch.int32), top_p=z(), min_p=z())
    a.update(kw)
    return a


def test_marshalling(recorder):
    t = tensors()
    S.sifar_sample(**t)
    c = recorder.calls[0]
    assert (c.dtype, c.tokens, c.vocab, c.logits_stride, c.workspace_bytes) == (
        S.SIFAR_FP16, T, V, V + 3, NEED)
    for name, tensor in t.items():
        assert getattr(c, name) == tensor.data_ptr(), name
    S.sifar_sample(t["logits"], t["uniform"], t["out"], t["workspace"])
    c = recorder.calls[1]
    assert not any((c.probs, c.temperature, c.top_k, c.top_p, c.min_p))


@pytest.mark.parametrize("kw", [
    dict(logits=torch.zeros(T, V, dtype=torch.float64)), dict(logits=torch.zeros(V)),
    dict(logits=torch.zeros(V, T).t()), dict(uniform=torch.zeros(T + 1)),
    dict(uniform=torch.zeros(T, dtype=torch.float64)), dict(uniform=torch.zeros(2 * T)[::2]),
    dict(out=torch.zeros(T, dtype=torch.int64)), dict(top_k=torch.zeros(T)),
    dict(top_p=torch.zeros(T, 1)), dict(min_p=torch.zeros(1)), dict(probs=torch.zeros(T - 1)),
    dict(temperature=torch.zeros(T, dtype=torch.float16)),
    dict(workspace=torch.zeros(NEED)), dict(workspace=torch.zeros(2, NEED, dtype=torch.uint8)),
    dict(workspace=torch.zeros((), dtype=torch.uint8)),
], ids=range(15))
def test_refused_by_the_binding(recorder, kw):
    with pytest.raises(S.SifarError) as e:
        S.sifar_sample(**tensors(**kw))
    assert e.value.code == S.SIFAR_EINVAL and not recorder.calls


def test_host_tensors_are_refused():
    with pytest.raises(S.SifarError) as e:
        S.sifar_sample(**tensors())
    assert e.value.code == S.SIFAR_EINVAL
