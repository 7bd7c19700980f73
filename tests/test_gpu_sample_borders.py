"""GPU: sifar_sample where a row's light tokens decide: numbers at the ends of [0, 1) over
weights far below the likeliest, and chunks (the 1 KB of a row that a wave loads) whose
tokens differ in weight by orders of magnitude. Against the definition in 64 bits, as in
test_gpu_sample.py; the numbers lie more than a unit of 2^-42 of the largest weight from
any border that a token or a chunk moves."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2607_08973_amd as S
import test_gpu_sample as base

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
INF = math.inf


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    S.load()
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", list(base.DT))
@pytest.mark.parametrize("kw", [dict(top_k=1 << 20), dict(min_p=1e-38),
                                dict(top_k=1 << 20, min_p=1e-38)],
                         ids=lambda kw: "-".join(kw))
@pytest.mark.parametrize("light", [1, 20, 40])
def test_one_and_above_draw_the_last_token_kept(dtype, kw, light):
    """Behind 100000 tokens of equal weight a few of 2^-50: the whole weight, some 2^58
    units, is not a 64-bit number's to the unit, and the last token weighs one."""
    x = torch.zeros(3, 100000 + light, dtype=base.DT[dtype], device=DEV)
    x[:, 100000:] = -35.0
    base.check(x, [1.0, 7.0, INF], **kw)
