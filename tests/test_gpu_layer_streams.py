"""GPU: the blocks of a decode layer on two streams at once, over outputs that were
overwritten before each call: one that does not run, or runs elsewhere or too early, shows."""
from __future__ import annotations

import pytest
import torch

import paper_2607_08973_amd as S
from test_gpu_decode_layer import E, HK, HQ, N, PAGE, T, Layer

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    S.load()
    yield
    torch.cuda.synchronize()


def spoil(s, r):
    """Nothing that rank r's calls write is left."""
    at = s.position.long()
    row, slot = s.pages[torch.arange(T, device=DEV), at // PAGE].long(), at % PAGE
    s.caches[r][:, row, slot] = float("nan")
    for t in (s.turned[r], s.seen[r], s.lse[r], s.experts[r]):
        t.fill_(float("nan"))
    s.ws.fill_(255)
    s.ews.fill_(255)


def calls(s, r, stream=None):
    x, (k, v) = s.rows[r], s.caches[r]
    here = slice(r * E // N, (r + 1) * E // N)
    S.sifar_cache_append(x[:, HQ:HQ + HK], x[:, HQ + HK:], s.position, s.pages, k, v,
                         q=x[:, :HQ], q_out=s.turned[r], inv_freq=s.freq, stream=stream)
    S.sifar_paged_attention(s.turned[r], k, v, s.pages, s.lengths, s.seen[r], s.ws, lse=s.lse[r],
                            stream=stream)
    S.sifar_experts(s.y, s.ids, s.weights, s.w_in[here], s.w_out[here], s.experts[r], s.ews,
                    first_expert=here.start, stream=stream)


@pytest.mark.parametrize("passed", [False, True])
def test_two_streams_at_once(passed):
    """The stream is the current one, or passed (and ordered behind what it needs)."""
    layers = [Layer(4), Layer(5)]
    want = []
    for s in layers:
        s.run()
        torch.cuda.synchronize()
        want.append(s.outputs())
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in layers:
        for r in range(N):
            spoil(s, r)
    torch.cuda.synchronize()
    for s, w in zip(layers, want):
        assert not any(torch.equal(a, b) for a, b in zip(
            (s.turned, s.seen, s.lse, s.experts, s.caches), (w[0], w[1], w[2], w[8], w[11])))
    for _ in range(15):
        for s, st in zip(layers, streams):
            for r in range(N):
                with torch.cuda.stream(st):
                    spoil(s, r)
                    if not passed:
                        calls(s, r)
                if passed:
                    calls(s, r, st)
    torch.cuda.synchronize()
    for s, w in zip(layers, want):
        for i, (a, b) in enumerate(zip(s.outputs(), w)):
            assert torch.equal(a, b), i
