"""GPU: the blocks of a decode layer at seeded random shapes over their whole ranges, each
against its formula in 64 bits with the bounds of its own test."""
from __future__ import annotations

import random

import pytest
import torch

import paper_2607_08973_amd as S
import test_gpu_cache_append as append_test
import test_gpu_experts as experts_test
import test_gpu_paged_attention as attention_test

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    S.load()
    yield
    torch.cuda.synchronize()


def spread(r, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** r.random()))))


@pytest.mark.parametrize("seed", range(48))
def test_attention(seed):
    r = random.Random(f"attention {seed}")
    kv = r.choice([1, 2, 3, 8])
    group = r.choice([1, 2, 3, 5, 8, 12, 16, 17, 20])
    dim = 8 * r.randint(1, 32) if seed % 2 else r.choice([64, 128, 256])
    lengths = [r.choice([0, 1, spread(r, 1, 3000), spread(r, 1, 3000)])
               for _ in range(spread(r, 1, 12))]
    page = r.choice([1, 5, 16, 64, 200])
    i = attention_test.inputs(1000 + seed, lengths, kv * group, kv, dim, page,
                              ["bf16", "fp16", "fp32"][seed % 3],
                              layout=r.choice(["slots", "heads", "both"]),
                              spread=r.choice([0.5, 2.0, 4.0]), sinks=r.random() < 0.4)
    for _ in range(r.choice([0, 0, 3])):  # pages that are not there
        t = r.randrange(len(lengths))
        i["pages"][t, r.randrange(i["pages"].shape[1])] = r.choice([-1, 1 << 28])
    kw = dict(window=r.choice([0, 0, spread(r, 1, 2000)]), softcap=r.choice([0.0, 0.0, 25.0]))
    if r.random() < 0.3:
        kw["max_length"] = max(1, max(lengths) // r.choice([1, 2]))
    attention_test.run_and_check(i, **kw)


@pytest.mark.parametrize("seed", range(48))
def test_append(seed):
    r = random.Random(f"append {seed}")
    dim = 8 * r.randint(1, 32)
    i = append_test.inputs(1000 + seed, spread(r, 1, 200), r.randint(1, 24), r.choice([1, 2, 5, 8]),
                           dim, r.choice([1, 3, 16, 100]), ["bf16", "fp16", "fp32"][seed % 3],
                           width=r.choice([2, 5]), layout=r.choice(["slots", "heads", "both"]))
    append_test.run_and_check(i, 2 * r.randint(0, dim // 2), r.random() < 0.5,
                              r.choice([1.0, 0.7, -1.0]))


@pytest.mark.parametrize("seed", range(48))
def test_experts(seed):
    r = random.Random(f"experts {seed}")
    experts, ranks = spread(r, 1, 24), r.choice([1, 1, 3])
    topk = r.randint(1, min(8, experts * ranks))
    i = experts_test.inputs(1000 + seed, spread(r, 1, 128), experts, topk, 8 * spread(r, 1, 100),
                            8 * spread(r, 1, 60), ["bf16", "fp16", "fp32"][seed % 3],
                            total=experts * ranks)
    experts_test.run_and_check(i, activation=r.choice(["silu", "gelu"]),
                               first_expert=experts * (ranks // 2))
