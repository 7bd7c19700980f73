"""GPU: sifar_sample inside a chunk (the 16 bytes of each of a wave's lanes: 256 logits
of 32 bits, 512 of 16) whose tokens differ in weight by orders of magnitude, in rows
without a filter. Against the definition in 64 bits, as in test_gpu_sample.py. A chunk's
sum is rounded to units of 2^-42 of the row's largest weight once, which moves the borders
of its tokens by half a unit's part of the chunk at most; the numbers lie further inside
the tokens that they have to draw."""
from __future__ import annotations

import math

import pytest
import torch

import paper_2607_08973_amd as S
import test_gpu_sample as base

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
INF = math.inf
LN2 = math.log(2.0)


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    S.load()
    yield
    torch.cuda.synchronize()


def row(dtype, V=1500):
    """The likeliest token at 1200, nothing else but what a test puts there."""
    x = torch.full((4, V), -INF, dtype=base.DT[dtype], device=DEV)
    x[:, 1200] = 0.0
    return x


@pytest.mark.parametrize("dtype", list(base.DT))
@pytest.mark.parametrize("bits", [38, 41])
def test_a_token_behind_many_light_ones(dtype, bits):
    """199 tokens of 2^-55 and one of 2^-bits: nearly all of the chunk's weight is its."""
    x = row(dtype)
    x[:, :199] = -55 * LN2
    x[:, 199] = -bits * LN2
    weight = 2.0 ** -bits
    u = [f * weight for f in (0.3, 0.5, 0.6, 0.7)]
    base.check(x, u)
    assert base.run(x, u)[0].tolist() == [199] * 4


@pytest.mark.parametrize("dtype", list(base.DT))
def test_light_tokens_behind_a_heavier_one(dtype):
    """Random numbers of 1 and above, and the last below 1, in rows that end with light
    tokens."""
    x = row(dtype)
    x[:, 1300] = -41 * LN2
    x[:, 1301:1450] = -55 * LN2
    base.check(x, [1.0, 3.0, INF, 1.0 - 2.0 ** -24])
    assert base.run(x, 1.0)[0].tolist() == [1449] * 4


@pytest.mark.parametrize("dtype", list(base.DT))
@pytest.mark.parametrize("tau", [0.3, 1.0, 5.0])
def test_tokens_of_a_light_chunk_are_drawn_by_weight(dtype, tau):
    """A first chunk of 2^-20 or so of the row, over the whole interval of its weight."""
    x = row(dtype, 2000).expand(4, 2000).contiguous()
    g = torch.Generator().manual_seed(5)
    part = torch.randn(256, generator=g, dtype=torch.float64) * 4 - 24
    x[:, :256] = (part * tau).to(x.dtype).to(DEV)
    w = torch.exp(x[0].double() / tau).cpu()
    first = (w[:256].sum() / w.sum()).item()
    for n in range(16):
        u = [first * (4 * n + i + 0.41) / 64 for i in range(4)]
        base.check(x, u, temperature=tau)


@pytest.mark.parametrize("dtype", list(base.DT))
def test_less_than_a_unit_into_a_chunk(dtype):
    """A chunk of one unit, 2^-42: half of it lies before its token of 2^-42."""
    x = row(dtype)
    x[:, :8] = -58 * LN2
    x[:, 8] = -42 * LN2
    base.check(x, [0.1 * 2.0 ** -42, 0.3 * 2.0 ** -42, 0.5 * 2.0 ** -42, 0.0])
