"""GPU: the row operators as a decode step uses them, around an all-reduce: the ranks'
partials are summed, the block's output is normalised, gated and added to the
residual stream, the normed rows are routed to experts and, at the end, sampled.
Every stage is checked against its definition on the inputs that it got; then the
whole step is captured and replayed on new inputs, with eager steps in between."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2607_08973_amd as S
import test_gpu_block_norm as norm_test
import test_gpu_route as route_test
import test_gpu_sample as sample_test

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
N, T, H, E, K, V = 4, 6, 1024, 64, 4, 5003


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    S.load()
    yield
    torch.cuda.synchronize()


class Step:
    def __init__(self, seed):
        r = np.random.default_rng([2607, 77, seed])
        n = lambda *s: torch.from_numpy(r.standard_normal(s)).to(torch.bfloat16).to(DEV)
        self.post, self.norm, self.final, self.gate = n(H), n(H), n(H), n(H)
        self.router = (n(H, E).float() / 32).contiguous()
        self.head = (n(H, V) / 16).to(torch.bfloat16)
        self.bias = 0.1 * n(E).float()
        self.temperature = torch.full((T,), 0.8, device=DEV)
        self.top_k = torch.full((T,), 300, dtype=torch.int32, device=DEV)
        self.top_p = torch.full((T,), 0.9, device=DEV)
        self.x, self.res, self.u = n(N, T, H), n(T, H), torch.zeros(T, device=DEV)
        self.new_inputs(seed)
        z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt, device=DEV)
        self.a, self.stream, self.y = z(T, H), z(T, H), z(T, H)
        self.ids, self.weights = z(T, K, dt=torch.int32), z(T, K, dt=torch.float32)
        self.last, self.z = z(T, H, dt=torch.float32), z(T, H)
        self.tokens, self.probs = z(T, dt=torch.int32), z(T, dt=torch.float32)
        self.ws = torch.empty(S.sifar_sample_workspace(T, V), dtype=torch.uint8, device=DEV)

    def new_inputs(self, seed):
        r = np.random.default_rng([2607, 78, seed])
        n = lambda *s: torch.from_numpy(r.standard_normal(s)).to(torch.bfloat16)
        self.x.copy_(n(N, T, H))
        self.res.copy_(n(T, H))
        self.u.copy_(torch.from_numpy(r.random(T)))

    def run(self):
        S.sifar_allreduce_noalloc(self.x, T * H, N, T, H, self.a)
        S.sifar_block_norm(self.a, self.res, self.stream, self.post, self.gate, self.norm, self.y,
                           branch_scale=0.5)
        self.scores = self.y.float() @ self.router
        S.sifar_route(self.scores, self.ids, self.weights, "sigmoid", self.bias, 8, 4, 2)
        # the experts' output stands in for itself: the ranks' partials again, summed on the way
        S.sifar_block_norm(self.x, self.stream.float(), self.last, None, None, self.final, self.z)
        self.logits = (self.z @ self.head).contiguous()
        S.sifar_sample(self.logits, self.u, self.tokens, self.ws, self.probs, self.temperature,
                       self.top_k, self.top_p)

    def outputs(self):
        return [t.clone() for t in (self.a, self.stream, self.y, self.ids, self.weights, self.last,
                                    self.z, self.tokens, self.probs)]


def test_every_stage_of_a_step():
    s = Step(1)
    s.run()
    f = norm_test.formula
    r, e, y, ey = f(s.a, s.res, s.post, s.gate, s.norm, 0.5, 1.0, 0.0, 1e-6)
    norm_test.check(s.stream, r, e)
    norm_test.check(s.y, y, ey)
    ids, w = route_test.definition(s.scores, K, "sigmoid", s.bias, 8, 4, 2, True, 1.0)
    assert np.array_equal(s.ids.cpu().numpy(), ids)
    assert (np.abs(s.weights.double().cpu().numpy() - w) <= w * (2.0 ** -24 + 1e-13)).all()
    r, e, y, ey = f(s.x, s.stream.float(), None, None, s.final, 1.0, 1.0, 0.0, 1e-6)
    norm_test.check(s.last, r, e)
    norm_test.check(s.z, y, ey)
    x = s.logits.double().cpu().numpy()
    one = np.float64(np.float32(0.8)), 300, np.float64(np.float32(0.9)), 0.0
    want = [sample_test.one(x[t], float(s.u[t]), *one) for t in range(T)]
    assert s.tokens.tolist() == [w[0] for w in want]
    for p, w in zip(s.probs.tolist(), want):
        assert abs(p - w[1]) <= w[1] * (2.0 ** -24 + V * 2.0 ** -42)


def test_a_captured_step_replays():
    s, eager = Step(2), Step(2)
    s.run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.run()
    for k in range(4):
        s.new_inputs(10 + k)
        eager.new_inputs(10 + k)
        g.replay()
        eager.run()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(s.outputs(), eager.outputs())):
            assert torch.equal(a, b), (k, i)


def test_two_streams_at_once():
    """Steps of two requests on streams of their own, each with its own buffers and
    workspace: block norms, routes and samples run side by side."""
    steps = [Step(20), Step(21)]
    want = []
    for s in steps:
        s.run()
        torch.cuda.synchronize()
        want.append(s.outputs())
        for t in (s.stream, s.y, s.ids, s.weights, s.last, s.z, s.tokens, s.probs):
            t.zero_()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, st in zip(steps, streams):
            with torch.cuda.stream(st):
                S.sifar_block_norm(s.a, s.res, s.stream, s.post, s.gate, s.norm, s.y,
                                   branch_scale=0.5)
                S.sifar_route(s.scores, s.ids, s.weights, "sigmoid", s.bias, 8, 4, 2)
                S.sifar_block_norm(s.x, s.stream.float(), s.last, None, None, s.final, s.z)
                S.sifar_sample(s.logits, s.u, s.tokens, s.ws, s.probs, s.temperature, s.top_k,
                               s.top_p)
    torch.cuda.synchronize()
    for s, w in zip(steps, want):
        for a, b in zip(s.outputs(), w):
            assert torch.equal(a, b)
