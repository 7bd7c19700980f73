"""The row operators' binding, beside what test_*_refusals.py cover: its first calls from
several threads. No GPU is used."""
from __future__ import annotations

import threading

import pytest
import torch

import paper_2607_08973_amd as S

T, H, E, K, V = 3, 64, 16, 2, 100


class Library:
    """Stands in for the library where host tensors play device tensors."""

    calls = 0

    def __getattr__(self, name):
        if name == "sifar_strerror":
            return lambda code: b""
        return self.call

    def call(self, *a):
        self.calls += 1
        return 0


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(S, "_lib", lib)
    monkeypatch.setattr(S, "_gpu", lambda fn, name, t: -1)   # a host tensor's device
    monkeypatch.setattr(S, "_row_stream", lambda stream, dev: 0)
    return lib


def norm(**kw):
    a = dict(x=torch.zeros(T, H), residual=torch.zeros(T, H), residual_out=torch.zeros(T, H))
    S.sifar_block_norm(**{**a, **kw})


def route(**kw):
    a = dict(logits=torch.zeros(T, E), ids=torch.zeros(T, K, dtype=torch.int32),
             weights=torch.zeros(T, K))
    S.sifar_route(**{**a, **kw})


def sample(**kw):
    a = dict(logits=torch.zeros(T, V), uniform=torch.zeros(T),
             out=torch.zeros(T, dtype=torch.int32), workspace=torch.zeros(64, dtype=torch.uint8))
    S.sifar_sample(**{**a, **kw})


def test_plain_calls(library):
    norm()
    route()
    sample()
    assert library.calls == 3


class Torch:
    """torch, as two threads see it that call at once: the second one calls while the
    first looks up its types."""

    def __init__(self):
        self.seen = []

    def __getattr__(self, name):
        self.seen.append(S._C)
        return getattr(torch, name)


def test_first_calls_of_two_threads(monkeypatch):
    """Callers look at _C only, so what else they use has to be there before it is."""
    stub = Torch()
    monkeypatch.setitem(__import__("sys").modules, "torch", stub)
    for name in ("_C", "_DTYPES", "_F32", "_I32", "_U8"):
        monkeypatch.setattr(S, name, None)
    S._torch()
    assert stub.seen and all(c is None for c in stub.seen)
    assert S._C is torch._C and S._DTYPES[torch.float16] == S.SIFAR_FP16
    assert (S._F32, S._I32, S._U8) == (torch.float32, torch.int32, torch.uint8)


def test_calls_of_many_threads_at_the_start(library, monkeypatch):
    for name in ("_C", "_DTYPES", "_F32", "_I32", "_U8"):
        monkeypatch.setattr(S, name, None)
    failed, start = [], threading.Barrier(8)

    def call():
        start.wait()
        try:
            route()
            sample()
        except Exception as e:   # noqa: BLE001 (reported below)
            failed.append(e)

    threads = [threading.Thread(target=call) for _ in range(8)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed
