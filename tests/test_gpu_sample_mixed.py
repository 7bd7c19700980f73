"""GPU: sifar_sample over batches of long rows whose requests differ in kind: some with
top-k, small or larger than any list of candidates, beside others whose nucleus is wide,
narrow, masked or greedy; and the nucleus of half-precision rows. Against the definition
in 64 bits, as in test_gpu_sample.py."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2607_08973_amd as S
import test_gpu_sample as base

pytestmark = pytest.mark.gpu

INF = math.inf


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    S.load()
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", list(base.DT))
@pytest.mark.parametrize("T,V", [(11, 70001), (11, 131072), (140, 66000)])
def test_top_k_for_some_rows(dtype, T, V):
    x = base.logits(70, T, V, dtype)
    x[1::4] = base.logits(71, len(range(1, T, 4)), V, dtype, "peaked")
    x[T - 1, : V // 3] = -INF
    r = base.rng(70, T, V)
    k = torch.tensor([[0, 5, -1, 9000, 0, 300, 1, 2 ** 31 - 1, 0, 60000, 0][t % 11] for t in range(T)])
    tau = 0.7 + 0.6 * r.random(T)
    tau[6::11] = 0.0
    u, p = r.random(T), 0.3 + 0.699 * r.random(T)
    base.check(x, u, temperature=tau, top_k=k, top_p=p)
    base.check(x, u, temperature=tau, top_k=k, top_p=p, min_p=0.003)
    base.check(x, u, temperature=tau, top_k=k)


@pytest.mark.parametrize("T,V", [(1, 65536), (3, 70001), (65, 66000), (2, 262144)])
def test_nucleus_of_large_half_precision_rows(T, V):
    x = base.logits(72, T, V, "fp16")
    x[T // 2] = base.logits(73, 1, V, "fp16", "peaked")[0]
    x[T - 1, : V // 3] = -INF
    r = base.rng(72, T, V)
    tau = 0.7 + 0.6 * r.random(T)
    u, p = r.random(T), 0.3 + 0.699 * r.random(T)
    base.check(x, u, temperature=tau, top_p=p)
    base.check(x, u, temperature=tau, top_p=p, min_p=0.02)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("V", [32000, 50257])
def test_top_k_around_the_number_of_chunks(dtype, V):
    """Rows of 63 and 99 chunks of 512 logits: from the largest of them on, top-k has no
    bound from the chunks' maxima."""
    n = (V + 511) // 512
    T = 8
    x, r = base.logits(74, T, V, dtype), base.rng(74, V)
    k = [n - 2, n - 1, n, n + 1, 1, 2 * n, 5000, 10]
    base.check(x, r.random(T), top_k=torch.tensor(k))
    base.check(x, r.random(T), top_k=torch.tensor(k), top_p=0.9, temperature=0.8)
