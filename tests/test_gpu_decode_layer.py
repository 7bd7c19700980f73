"""GPU: a layer of a decode step as two tensor-parallel ranks run it. Each rank projects its
heads, appends to its cache, attends and projects back; the ranks' partials are
all-reduced and normed; the router's choice runs on each rank's experts, and their partials
are summed with the residual. Every stage is checked against its definition on the inputs
that it got, over steps of a growing cache; then a captured step replays them."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2607_08973_amd as S
import test_gpu_block_norm as norm_test
import test_gpu_cache_append as append_test
import test_gpu_experts as experts_test
import test_gpu_paged_attention as attention_test
import test_gpu_route as route_test

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF = torch.bfloat16
N, T, H, HQ, HK, D = 2, 3, 256, 4, 2, 64      # ranks; heads of one rank
PAGE, WIDTH, E, K, I = 16, 20, 12, 4, 136     # experts of all ranks
START = [0, 15, 290]


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    S.load()
    yield
    torch.cuda.synchronize()


class Layer:
    def __init__(self, seed):
        r = np.random.default_rng([2607, 95, seed])
        n = lambda *s: torch.from_numpy(r.standard_normal(s, dtype=np.float32)).to(DEV)
        w = lambda *s: (n(*s) / s[-2] ** 0.5).to(BF)
        self.qkv, self.back = w(N, H, (HQ + 2 * HK) * D), w(N, HQ * D, H)
        self.norms = [(1 + 0.1 * n(H)).to(BF) for _ in range(2)]
        self.router = n(H, E) / H ** 0.5
        self.w_in = (n(E, 2 * I, H) / H ** 0.5).to(BF)
        self.w_out = (n(E, H, I) / I ** 0.5).to(BF)
        pool = T * WIDTH + 2
        self.caches = n(N, 2, pool, PAGE, HK, D).to(BF)
        self.pages = torch.from_numpy(r.permutation(pool)[:T * WIDTH].astype(np.int32)).view(
            T, WIDTH).to(DEV)
        self.freq = append_test.freqs(D)
        self.position = torch.tensor(START, dtype=torch.int32, device=DEV)
        self.lengths = self.position + 1
        z = lambda *s, dt=BF: torch.zeros(*s, dtype=dt, device=DEV)
        self.x, self.residual = n(T, H).to(BF), n(T, H).to(BF)
        self.turned, self.seen = z(N, T, HQ, D), z(N, T, HQ, D)
        self.lse = z(N, T, HQ, dt=torch.float32)
        self.partials, self.summed, self.experts = z(N, T, H), z(T, H), z(N, T, H)
        self.stream, self.y, self.out, self.last = z(T, H), z(T, H), z(T, H), z(T, H)
        self.ids, self.weights = z(T, K, dt=torch.int32), z(T, K, dt=torch.float32)
        bytes_ = lambda n: torch.empty(n, dtype=torch.uint8, device=DEV)
        self.ws = bytes_(S.sifar_paged_attention_workspace(T, HQ, HK, D, WIDTH * PAGE))
        self.ews = bytes_(S.sifar_experts_workspace(T, K, I))

    def run(self):
        self.rows = []
        for r in range(N):
            x = (self.x @ self.qkv[r]).view(T, HQ + 2 * HK, D)
            self.rows.append(x)
            k, v = self.caches[r]
            S.sifar_cache_append(x[:, HQ:HQ + HK], x[:, HQ + HK:], self.position, self.pages, k, v,
                                 q=x[:, :HQ], q_out=self.turned[r], inv_freq=self.freq)
            S.sifar_paged_attention(self.turned[r], k, v, self.pages, self.lengths, self.seen[r],
                                    self.ws, lse=self.lse[r])
            self.partials[r] = self.seen[r].view(T, HQ * D) @ self.back[r]
        S.sifar_allreduce_noalloc(self.partials, T * H, N, T, H, self.summed)
        S.sifar_block_norm(self.summed, self.residual, self.stream, norm_weight=self.norms[0],
                           y=self.y)
        self.scores = self.y.float() @ self.router
        S.sifar_route(self.scores, self.ids, self.weights)
        for r in range(N):
            here = slice(r * E // N, (r + 1) * E // N)
            S.sifar_experts(self.y, self.ids, self.weights, self.w_in[here], self.w_out[here],
                            self.experts[r], self.ews, first_expert=here.start)
        S.sifar_block_norm(self.experts, self.stream, self.out, norm_weight=self.norms[1],
                           y=self.last)

    def next_inputs(self):
        """The next tokens: what the layer made of the last ones, one position on."""
        self.x.copy_(self.last)
        self.residual.copy_(self.out)
        self.position += 1
        self.lengths += 1

    def outputs(self):
        return [t.clone() for t in (self.turned, self.seen, self.lse, self.summed, self.stream,
                                    self.y, self.ids, self.weights, self.experts, self.out,
                                    self.last, self.caches)]


def check_stages(s):
    at = s.position.long()
    row, slot = s.pages[torch.arange(T, device=DEV), at // PAGE].long(), at % PAGE
    for r in range(N):
        x = s.rows[r]
        append_test.check(s.turned[r], *append_test.rotated(x[:, :HQ], s.position, s.freq, False, 1.0))
        append_test.check(s.caches[r, 0][row, slot],
                          *append_test.rotated(x[:, HQ:HQ + HK], s.position, s.freq, False, 1.0))
        assert torch.equal(s.caches[r, 1][row, slot], x[:, HQ + HK:])
        attention_test.check(dict(q=s.turned[r], k_cache=s.caches[r, 0], v_cache=s.caches[r, 1],
                                  pages=s.pages, lengths=s.lengths), s.seen[r], s.lse[r])
    norm_test.check(s.stream, *norm_test.formula(s.summed, s.residual, None, None, s.norms[0], 1.0,
                                                 1.0, 0.0, 1e-6)[:2])
    ids, w = route_test.definition(s.scores, K, "softmax", None, 1, 1, 1, True, 1.0)
    assert np.array_equal(s.ids.cpu().numpy(), ids)
    for r in range(N):
        here = slice(r * E // N, (r + 1) * E // N)
        experts_test.check(dict(x=s.y, w_in=s.w_in[here], w_out=s.w_out[here], ids=s.ids,
                                weights=s.weights), s.experts[r], first_expert=here.start)
    norm_test.check(s.out, *norm_test.formula(s.experts, s.stream, None, None, s.norms[1], 1.0, 1.0,
                                              0.0, 1e-6)[:2])


def test_every_stage_of_some_steps():
    s = Layer(1)
    for _ in range(4):
        s.run()
        torch.cuda.synchronize()
        check_stages(s)
        s.next_inputs()


def test_ranks_together_are_the_whole():
    """Both ranks' experts sum to what one rank with all of them computes."""
    s = Layer(2)
    s.run()
    whole = torch.empty_like(s.y)
    S.sifar_experts(s.y, s.ids, s.weights, s.w_in, s.w_out, whole, s.ews)
    both = s.experts.double().sum(0)
    # each is rounded once to bf16
    off = 2.0 ** -9 * (s.experts.double().abs().sum(0) + whole.double().abs()) * 2 + 1e-6
    assert ((both - whole.double()).abs() <= off).all()


def test_a_captured_step_replays():
    """Positions and lengths are read on the device, so one graph serves a growing cache."""
    s, eager = Layer(3), Layer(3)
    s.run()   # (library handles and workspaces come to be outside the capture)
    s.caches.copy_(eager.caches)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.run()
    for k in range(5):
        g.replay()
        eager.run()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(s.outputs(), eager.outputs())):
            assert torch.equal(a, b), (k, i)
        s.next_inputs()
        eager.next_inputs()


def test_two_streams_at_once():
    layers = [Layer(4), Layer(5)]
    want = []
    for s in layers:
        s.run()
        torch.cuda.synchronize()
        want.append(s.outputs())
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(15):
        for s, st in zip(layers, streams):
            with torch.cuda.stream(st):
                for r in range(N):
                    x, (k, v) = s.rows[r], s.caches[r]
                    S.sifar_cache_append(x[:, HQ:HQ + HK], x[:, HQ + HK:], s.position, s.pages, k,
                                         v, q=x[:, :HQ], q_out=s.turned[r], inv_freq=s.freq)
                    S.sifar_paged_attention(s.turned[r], k, v, s.pages, s.lengths, s.seen[r], s.ws,
                                            lse=s.lse[r])
                    here = slice(r * E // N, (r + 1) * E // N)
                    S.sifar_experts(s.y, s.ids, s.weights, s.w_in[here], s.w_out[here],
                                    s.experts[r], s.ews, first_expert=here.start)
    torch.cuda.synchronize()
    for s, w in zip(layers, want):
        for i, (a, b) in enumerate(zip(s.outputs(), w)):
            assert torch.equal(a, b), i
