"""GPU: sifar_route where scores lie next to each other. c is compared without its ten
lowest bits, so two values on one side of such a step tie and two around its edge do
not; the groups' worths are compared as 64-bit numbers. A logit of -2000 scores 0 under
sigmoid, so that c is the bias, exactly."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2607_08973_amd as S
import test_gpu_route as base

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    S.load()
    yield
    torch.cuda.synchronize()


def picked(x, bias, k, **kw):
    t = lambda v: torch.tensor(v, dtype=torch.float32, device=DEV)
    return base.run(t([x]), k, "sigmoid", t(bias), **kw)[0][0].tolist()


def test_scores_around_the_edge_of_a_step():
    """c = bias + s: 0.75 + 2^-50 and 0.75 + 2^-44 share a step of 2^-43 with 0.75; 0.75 +
    2^-42.5 lies in another, and so does 1 - 2^-50 beside 1."""
    s = lambda b: -b * float(np.log(2.0))     # 1 / (1 + 2^b)
    off = -2000.0
    assert picked([s(-50), off], [0.0, 1.0], 2) == [1, 0]
    assert picked([off, s(50), s(44)], [0.75] * 3, 3) == [0, 1, 2]
    assert picked([off, s(42.5)], [0.75] * 2, 2) == [1, 0]
    # below an edge: -0.75 + 2^-50 is the smaller magnitude, the step nearer to zero
    assert picked([off, s(50)], [-0.75] * 2, 2) == [1, 0]
    assert picked([s(50), s(46)], [-0.75] * 2, 2) == [0, 1]


def test_groups_whose_sums_differ_in_the_last_bits():
    off = [-2000.0] * 6
    tiny = 2.0 ** -52
    kw = dict(groups=3, top_groups=1, group_top=2)
    assert picked(off, [0.75, 0.0, 0.75, tiny, 0.75, 0.0], 2, **kw) == [2, 3]
    assert picked(off, [0.75, 0.0, 0.75, 0.0, 0.75, 0.0], 2, **kw) == [0, 1]
    # 0.75 + 2^-60 rounds to 0.75: a tie
    assert picked(off, [0.75, 0.0, 0.75, 2.0 ** -60, 0.75, 0.0], 2, **kw) == [0, 1]


@pytest.mark.parametrize("dtype", list(base.DT))
def test_groups_by_their_best(dtype):
    x = torch.full((1, 8), -2000.0, device=DEV).to(base.DT[dtype])
    bias = torch.tensor([0.5, 0.25, 0.5, 0.3, 0.5, 0.2, 0.5 + 2.0 ** -24, 0.0], device=DEV)
    ids, _ = base.run(x, 3, "sigmoid", bias, 4, 2, 1)
    assert ids[0].tolist() == [6, 0, 1]
