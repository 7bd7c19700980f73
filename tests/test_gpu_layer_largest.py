"""GPU: the blocks of a decode layer at the ends of their ranges: the most tokens, heads,
elements and positions that their contracts name."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2607_08973_amd as S
import test_gpu_cache_append as append_test
import test_gpu_experts as experts_test
import test_gpu_paged_attention as attention_test

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    S.load()
    yield
    torch.cuda.synchronize()


def test_append_of_the_most_tokens():
    T = S.SIFAR_ROWS_MAX_TOKENS
    x = torch.randn(T, 2, 8, device=DEV).to(torch.bfloat16)
    kc, vc = (torch.zeros(T // 16, 16, 1, 8, dtype=torch.bfloat16, device=DEV) for _ in "kv")
    pages = torch.randperm(T // 16, device=DEV).int().view(1, -1)
    at = torch.arange(T, dtype=torch.int32, device=DEV)
    f = append_test.freqs(8)
    S.sifar_cache_append(x[:, :1], x[:, 1:], at, pages, kc, vc, inv_freq=f,
                         sequence=torch.zeros_like(at))
    rows = pages[0].long()
    assert torch.equal(vc[rows].view(T, 1, 8), x[:, 1:])
    got = kc[rows].view(T, 1, 8)
    for part in (slice(0, 4096), slice(T - 4096, T)):
        append_test.check(got[part], *append_test.rotated(x[part, :1], at[part], f, False, 1.0))


def test_attention_of_the_most_tokens():
    T = S.SIFAR_ATTENTION_MAX_TOKENS
    r = np.random.default_rng(1)
    i = attention_test.inputs(2000, [int(n) for n in r.integers(0, 40, T)], 1, 1, 8, 8)
    out, lse = attention_test.run(i)
    rows = [0, 1, 2, 255, 256, T // 2, T - 2, T - 1] + [int(t) for t in r.integers(0, T, 60)]
    attention_test.check(i, out, lse, rows=rows)


@pytest.mark.parametrize("kv,group", [(1024, 1), (1, 1024), (64, 16)])
def test_attention_of_the_most_heads(kv, group):
    attention_test.run_and_check(attention_test.inputs(2001, [3, 300], kv * group, kv, 16, 16))


def test_attention_over_a_million_positions():
    """One sequence of 2^20 + 5 positions, bounds and all; and a window at its end."""
    n = 2 ** 20 + 5
    i = attention_test.inputs(2002, [n], 4, 1, 64, 256)
    attention_test.run_and_check(i)
    attention_test.run_and_check(i, window=1000)


@pytest.mark.parametrize("H,I", [(65536, 8), (8, 65536), (65528, 16)])
@pytest.mark.parametrize("T", [1, 9])
def test_experts_of_the_longest_rows(H, I, T):
    experts_test.run_and_check(experts_test.inputs(2003, T, 2, 1, H, I))


def test_experts_of_the_most_tokens_slots_and_experts():
    experts_test.run_and_check(experts_test.inputs(2004, 128, 8, 8, 32, 24))
    experts_test.run_and_check(experts_test.inputs(2005, 32, 1024, 32, 16, 8))
    i = experts_test.inputs(2006, 128, 1, 8, 16, 8, ids=np.zeros((128, 8)))
    experts_test.run_and_check(i)  # 1024 slots of one expert
