"""GPU: infinities and NaN among the values that sifar_paged_attention reads. An infinite
value makes its element of the output infinite, of its own sign; two of both signs, or a NaN,
make it NaN; every other element keeps its bits."""
from __future__ import annotations

import pytest
import torch

import paper_2607_08973_amd as S
import test_gpu_paged_attention as attention_test

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
INF, NAN = float("inf"), float("nan")


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    S.load()
    yield
    torch.cuda.synchronize()


def plant(i, t, p, head, at, value):
    """`value` into element `at` of a head's values at position p of sequence t."""
    page = i["v_cache"].shape[1]
    i["v_cache"][int(i["pages"][t, p // page]), p % page, head, at] = value


def same(a, b):
    return torch.equal(torch.nan_to_num(a.float(), 7e30, 8e30, -8e30),
                       torch.nan_to_num(b.float(), 7e30, 8e30, -8e30))


# one tile and less, a chunk of many, several chunks that are joined
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("D", [24, 64, 80, 128, 136, 256])
@pytest.mark.parametrize("length", [1, 7, 40, 130, 1000, 3100])
def test_infinite_values(dtype, D, length):
    i = attention_test.inputs(4000 + length, [length, 33], 6, 2, D, 16, dtype, spread=0.5)
    want, want_lse = attention_test.run(i)
    last = length - 1
    plant(i, 0, last // 2, 0, 0, INF)
    plant(i, 0, last, 1, 3, -INF)
    plant(i, 0, 0, 1, D - 1, INF)
    plant(i, 0, last // 3, 0, D - 2, NAN)
    if length > 1:
        plant(i, 0, 0, 0, 5, INF)
        plant(i, 0, last, 0, 5, INF)    # of one sign: infinite
        plant(i, 0, 0, 1, 6, INF)
        plant(i, 0, last, 1, 6, -INF)   # of both: NaN
    out, lse = attention_test.run(i)
    for head in range(3):
        want[0, head, 0], want[0, head, D - 2] = INF, NAN
        want[0, 3 + head, 3], want[0, 3 + head, D - 1] = -INF, INF
        if length > 1:
            want[0, head, 5], want[0, 3 + head, 6] = INF, NAN
    assert same(out, want), (out - want).nonzero()[:8]
    assert torch.equal(lse, want_lse)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
def test_infinite_values_over_many_tiles(dtype, D):
    """Past the caches where the width allows, in the first, a middle and the last tile of a
    chunk as long as chunks get, beside pages that are not there and a window."""
    i = attention_test.inputs(4001, [1536, 1500, 1100] + [1] * 1097, 4, 2, D, 32, dtype, spread=0.5)
    i["pages"][0, 7] = -1
    want, _ = attention_test.run(i, window=1450)
    for k, p in enumerate((87, 700, 1535)):
        plant(i, 0, p, 1, 2 + k, -INF)
    plant(i, 0, 5, 1, 9, INF)  # before the window
    plant(i, 1, 1499, 0, 1, INF)
    out, _ = attention_test.run(i, window=1450)
    want[0, 2:, 2:5] = -INF
    want[1, :2, 1] = INF
    assert same(out, want), (out - want).nonzero()[:8]


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_small_weights_of_infinite_values(dtype):
    """Weights of 2^-30 and 2^-100 of the largest: infinite all the same, though 16 bits would
    round some of them away."""
    i = attention_test.inputs(4002, [200, 200], 1, 1, 64, 16, dtype, spread=0.0)
    i["k_cache"].zero_()
    i["q"][:, 0, 0] = 8.0
    for t, gap in enumerate((30.0, 100.0)):
        # the score is scale q k: 8 k / 8
        i["k_cache"][i["pages"][t].long(), :, 0, 0] = -gap * 0.6931
        i["k_cache"][int(i["pages"][t, 2]), 3, 0, 0] = 0.0
        plant(i, t, 150, 0, 4, INF)
        plant(i, t, 20, 0, 5, -INF)
    out, _ = attention_test.run(i)
    assert (out[:, 0, 4] == INF).all() and (out[:, 0, 5] == -INF).all()
    out[:, 0, 4:6] = 0
    assert torch.isfinite(out).all()
