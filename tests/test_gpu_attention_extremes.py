"""GPU: sifar_paged_attention at the ends of its numbers' ranges: sinks, scales
and bounds of scores that pass fp32 in base 2, and the sink as the lse of a row without
positions."""
from __future__ import annotations

import pytest
import torch

import paper_2607_08973_amd as S
import test_gpu_paged_attention as attention_test

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
INF = float("inf")
MOST = torch.finfo(torch.float32).max


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    S.load()
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("longest", [40, 3000])
def test_sinks_of_every_size(dtype, longest):
    """Where a sink is all there is, out is 0 and lse the sink; where it is nothing, as without."""
    sinks = [MOST, 3e38, 2.4e38, 2.3e38, 100.0, -100.0, -2.3e38, -2.4e38, -3e38, -MOST, -INF, 0.1]
    i = attention_test.inputs(6000, [longest, 0, 7, -2], 12, 3, 64, 16, dtype, width=longest // 16 + 1)
    none, none_lse = attention_test.run(i)
    i["sinks"] = torch.tensor(sinks, device=DEV)
    out, lse = attention_test.run_and_check(i)
    for t in (0, 2):
        assert (out[t, :4] == 0).all() and torch.equal(lse[t, :4], i["sinks"][:4])
        assert torch.equal(out[t, 6:11], none[t, 6:11])
        assert torch.equal(lse[t, 6:11], none_lse[t, 6:11])
    for t in (1, 3):
        assert (out[t] == 0).all() and torch.equal(lse[t], i["sinks"])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("scale", [2.0 ** 126, 1.8e38, 3e38, -MOST])
@pytest.mark.parametrize("softcap", [0.0, 20.0])
def test_scales_of_every_size(dtype, scale, softcap):
    """Keys so small that the scores are a few units all the same."""
    i = attention_test.inputs(6001, [50, 1500, 0], 4, 2, 64, 16, dtype, sinks=True)
    i["q"].mul_(2.0 ** -62)
    i["k_cache"].mul_(2.0 ** -66)
    out, lse = attention_test.run_and_check(i, scale=scale, softcap=softcap)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("softcap", [1e37, 2.4e38, MOST])
def test_softcaps_of_every_size(dtype, softcap):
    """Of scores of a few units it leaves them as they are. s / softcap is below fp32's normal
    numbers, so half a step of it is 2^-150, and 2^-22 of a score, which e^s passes on."""
    i = attention_test.inputs(6002, [50, 1500, 0], 4, 2, 64, 16, dtype, sinks=True)
    out, lse = attention_test.run(i, softcap=softcap)
    for t in range(3):
        want, err, wl, el = attention_test.formula(i, t)
        v = i["v_cache"].abs().max().double().cpu()
        more = 2.0 ** -20 * v   # two such roundings, on weights and on their sum
        assert ((out[t].double().cpu() - want).abs() <=
                err + more + attention_test.half_step(out.dtype, want.abs() + err + more)).all()
        assert ((lse[t].double().cpu() - wl).abs() <= el + 2.0 ** -21).all()
