"""GPU: infinities in what sifar_experts multiplies. An infinite weight or h makes what it
reaches infinite, of its sign; both signs, or a NaN, make NaN; everything else keeps its
bits. h is infinite where fp32 says so, not where 16 bits would round to it."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2607_08973_amd as S
import test_gpu_experts as experts_test

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
INF, NAN = float("inf"), float("nan")


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    S.load()
    yield
    torch.cuda.synchronize()


def check(got, want, i):
    """Where the formula in 64 bits is not finite, the same; elsewhere what was there without."""
    formula, _ = experts_test.formula(i)
    odd = ~torch.isfinite(formula)
    assert odd.any() and not odd.all()
    g = got.double().cpu()
    assert torch.equal(g[odd].nan_to_num(7.0, 8.0, 9.0), formula[odd].nan_to_num(7.0, 8.0, 9.0))
    assert torch.equal(got.cpu()[~odd], want.cpu()[~odd])


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("T,E,topk", [(1, 1, 1), (3, 9, 4), (13, 2, 1), (30, 1, 1), (64, 4, 2),
                                      (70, 1, 1)])
@pytest.mark.parametrize("H,I", [(24, 8), (72, 520), (40, 1096)])
def test_infinite_weights_of_the_second_product(dtype, T, E, topk, H, I):
    i = experts_test.inputs(5000, T, E, topk, H, I, dtype)
    want = experts_test.run(i)
    e = int(i["ids"][0, 0])
    i["w_out"][e, 1, 0] = INF
    i["w_out"][e, 5, I - 1] = -INF
    i["w_out"][e, H - 1, I // 2] = INF
    i["w_out"][e, 6, 1], i["w_out"][e, 6, 2] = INF, -INF  # NaN or infinite, as the signs of h are
    i["w_out"][e, 9, 3] = NAN
    check(experts_test.run(i), want, i)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("T", [1, 4, 9, 40])
@pytest.mark.parametrize("I", [8, 136, 1096])
def test_infinite_h(dtype, T, I):
    """An up weight that is infinite: h is, of the sign of its gate and of x, for every token of
    the expert; a second one of the other sign meets it in half of the rows."""
    i = experts_test.inputs(5001, T, 3, 2, 40, I, dtype, ids=[[t % 2, 2] for t in range(T)])
    want = experts_test.run(i)
    i["w_in"][0, I + I // 2, 3] = INF
    got = experts_test.run(i)
    if T > 1:
        check(got, want, i)
    i["w_in"][0, I + 1, 7] = -INF
    got = experts_test.run(i)
    formula, _ = experts_test.formula(i)
    assert not torch.isfinite(formula[::2]).any()
    assert torch.equal(got[::2].double().cpu().nan_to_num(7.0, 8.0, 9.0),
                       formula[::2].nan_to_num(7.0, 8.0, 9.0))
    assert torch.equal(got[1::2], want[1::2])


@pytest.mark.parametrize("T", [1, 6, 20])
def test_h_above_the_largest_of_16_bits(T):
    """h = 32 (2^123 - 2^112), in fp32 below 2^128, in bf16 rounded to infinity."""
    i = experts_test.inputs(5002, T, 2, 1, 16, 24, "bf16", ids=np.zeros((T, 1)))
    i["x"].zero_()
    i["x"][:, :3] = 1.0
    i["w_in"].zero_()
    i["w_in"][0, :24, 2] = 32.0
    i["w_in"][0, 24:, 0] = 2.0 ** 123 - 2.0 ** 115
    i["w_in"][0, 24:, 1] = 2.0 ** 115 - 2.0 ** 112
    i["w_in"][0, 24::2] *= -1
    i["w_out"].mul_(2.0 ** -100)
    got = experts_test.run(i)
    assert torch.isfinite(got).all()
    experts_test.check(i, got)


def test_a_token_that_is_nan_beside_others():
    """The other tokens of its tile keep their bits, those with infinite outputs too."""
    i = experts_test.inputs(5003, 20, 2, 1, 72, 264, ids=np.zeros((20, 1)))
    i["w_out"][0, 3, 9] = INF
    want = experts_test.run(i)
    i["x"][7] = NAN
    got = experts_test.run(i)
    assert got[7].isnan().all()
    keep = [t for t in range(20) if t != 7]
    assert torch.equal(got[keep], want[keep]) and torch.isinf(got[keep, 3]).all()
