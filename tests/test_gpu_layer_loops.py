"""GPU: the main loops of the layer's blocks, turned many times: chunks of a dozen tiles and
more a wave for every type and head width, padded, through the caches and past them; rows of
weights of many batches a wave for every number of columns. Each against its formula in 64
bits with the bounds of its own test. (tests/test_attend_tiles.py checks on the host that the
shapes below reach those loops.)"""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2607_08973_amd as S
import test_gpu_experts as experts_test
import test_gpu_paged_attention as attention_test

pytestmark = pytest.mark.gpu

DEV = "cuda:0"

# So many sequences that a chunk gets as long as it may; heads of 4 on 2 are read past the
# caches where they are not padded, 34 on 2 (two workgroups each) through them.
GROUPS = [(1100, 4, 2), (550, 34, 2)]
DIMS = [40, 64, 96, 128, 200, 256]
REACH = [1536, 4000]
LENGTHS = [1536, 1535, 1409, 1025, 897, 640, 385, 257]  # one chunk: 12 to 3 tiles of 32 a wave
LONGER = [4000, 3999, 2817, 1537]


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    S.load()
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("D", DIMS)
@pytest.mark.parametrize("T,Hq,Hk", GROUPS)
@pytest.mark.parametrize("reach", REACH)
def test_many_tiles_a_wave(dtype, D, T, Hq, Hk, reach):
    long = LENGTHS if reach == 1536 else LONGER
    if Hq > 4:
        long = long[::2]  # (the formula repeats the keys for each query head)
    lengths = long + [1 + t % 3 for t in range(T - len(long))]
    i = attention_test.inputs(3000, lengths, Hq, Hk, D, 32, dtype, width=reach // 32, spread=1.5,
                              sinks=D == 96)
    i["pages"][1, 5:40:3] = -1  # in the middle of tiles that others follow
    out, lse = attention_test.run(i)
    attention_test.check(i, out, lse, rows=list(range(len(long))) + [T - 2, T - 1])


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
def test_windows_and_caps_over_many_tiles(dtype, D):
    lengths = [1900, 1500, 1111, 600] + [1 + t % 3 for t in range(1096)]
    i = attention_test.inputs(3001, lengths, 4, 2, D, 32, dtype, width=60)
    out, lse = attention_test.run(i, window=1400, softcap=15.0)
    attention_test.check(i, out, lse, rows=[0, 1, 2, 3, 1099], window=1400, softcap=15.0)


# Slots of an expert: up to 4 columns, one, two and four tiles of them, and more than fit at
# once; rows of 129 and 65 steps of 64 bytes in 16 bits, the last of which rows end in.
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("columns", [1, 4, 5, 16, 17, 32, 33, 64, 70])
@pytest.mark.parametrize("H,I", [(4104, 72), (72, 4104)])
def test_many_batches_a_wave(dtype, columns, H, I):
    i = experts_test.inputs(3002, columns, 2, 1, H, I, dtype, ids=np.zeros((columns, 1)))
    experts_test.run_and_check(i)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("T,E,topk", [(2, 12, 8), (12, 9, 8), (40, 10, 8), (64, 12, 9)])
def test_many_batches_of_many_experts(dtype, T, E, topk):
    """More experts than waves: none shares `inter`, and a wave takes all of its steps."""
    experts_test.run_and_check(experts_test.inputs(3003, T, E, topk, 1032, 1032, dtype),
                               activation="gelu")
