"""The row operators' binding, beside what test_*_refusals.py cover: values that
no struct of the library holds and first calls from several threads. No GPU is used."""
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


@pytest.mark.parametrize("call,kw", [
    (norm, dict(eps=1e39)), (norm, dict(branch_scale=-1e39)), (norm, dict(residual_scale=1e300)),
    (norm, dict(weight_offset=1e39)), (norm, dict(eps=None)), (norm, dict(branch_scale="1")),
    (route, dict(scale=1e39)), (route, dict(scale=None)), (route, dict(groups=1 << 31)),
    (route, dict(groups=-(1 << 40))), (route, dict(top_groups=1 << 64)),
    (route, dict(group_top=1.5)), (route, dict(groups=None)),
])
def test_values_that_no_struct_holds(library, call, kw):
    with pytest.raises(S.SifarError) as e:
        call(**kw)
    assert e.value.code == S.SIFAR_EINVAL and not library.calls
    assert str(e.value).startswith("sifar_" + ("block_norm" if call is norm else "route"))


@pytest.mark.parametrize("eps", [0.0, 3.4e38, 1e-45])
def test_values_at_the_ends_of_their_range(library, eps):
    norm(eps=eps)
    route(scale=-eps)
    assert library.calls == 2


@pytest.mark.parametrize("call,name", [
    (norm, "x"), (norm, "residual_out"), (route, "logits"), (route, "ids"), (route, "weights"),
    (sample, "logits"), (sample, "uniform"), (sample, "out"), (sample, "workspace"),
])
def test_operands_that_are_missing(library, call, name):
    with pytest.raises(S.SifarError) as e:
        call(**{name: None})
    assert e.value.code == S.SIFAR_EINVAL and f"no {name}" in str(e.value) and not library.calls


@pytest.mark.parametrize("tokens,vocab", [
    (-(1 << 32) + 5, 100), (5, -(1 << 32) + 100), (-(1 << 40), 5), (-(1 << 64), 5), (5, -(1 << 31)),
])
def test_workspace_of_sizes_below_32_bits(tokens, vocab):
    """Not taken for the sizes that their low 32 bits spell."""
    with pytest.raises(S.SifarError) as e:
        S.sifar_sample_workspace(tokens, vocab)
    assert e.value.code == S.SIFAR_EINVAL


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
