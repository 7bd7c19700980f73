"""Tests that call on a stream of their own after filling outputs and workspaces on the current
one: the call waits for the fills. No GPU is used."""
from __future__ import annotations

import pytest
import torch

import conftest
import paper_2607_08973_amd as S
import test_gpu_experts as experts_test
import test_gpu_paged_attention as attention_test


class Library:
    """Stands in for the library: notes when it is called, and on which stream."""

    def __init__(self, events):
        self.events = events

    def __getattr__(self, name):
        if name.endswith("_workspace"):
            return lambda *sizes: 64
        return lambda packed, stream: self.events.append((name, stream)) or 0


class Stream:
    cuda_stream = 5

    def __init__(self, events):
        self.events = events

    def wait_stream(self, other):
        self.events.append(("wait", other))


@pytest.mark.parametrize("module,fn", [(experts_test, "sifar_experts"),
                                       (attention_test, "sifar_paged_attention")])
def test_a_call_on_another_stream_waits(module, fn, monkeypatch):
    events = []
    monkeypatch.setattr(module, "DEV", "cpu")
    monkeypatch.setattr(S, "_lib", Library(events))
    monkeypatch.setattr(S, "load", lambda: S._lib)
    monkeypatch.setattr(S, "_gpu", lambda fn, name, t: -1)   # a host tensor's device
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: "current")
    monkeypatch.setattr(torch.cuda, "synchronize", lambda: events.append("synchronize"))
    assert module.__name__ in conftest.FILL_FIRST
    monkeypatch.setattr(S, "_row_stream", conftest.ordered(S._row_stream))
    i = (experts_test.inputs(1, 2, 2, 1, 8, 8) if module is experts_test
         else attention_test.inputs(1, [3, 2], 2, 1, 8, 8))
    module.run(i, stream=Stream(events))
    assert events == [("wait", "current"), (fn, 5), "synchronize"]
