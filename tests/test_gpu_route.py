"""GPU: sifar_route against its definition in 64 bits.

ids have to be equal. A weight is a 64-bit quotient (relative error below 1e-13)
rounded once to fp32: half a step, 2^-24 of its value."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2607_08973_amd as S

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
INF = float("inf")


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    S.load()
    yield
    torch.cuda.synchronize()


def definition(x, k, score, bias, groups, top_groups, group_top, renorm, scale):
    """One token at a time, with Python's sort."""
    x = x.double().cpu().numpy()
    b = np.zeros(x.shape[1]) if bias is None else bias.double().cpu().numpy()
    ids = np.full((x.shape[0], k), -1, np.int64)
    w = np.zeros((x.shape[0], k))
    per = x.shape[1] // groups
    for t, row in enumerate(x):
        there = [e for e in range(row.size) if row[e] > -INF]
        s = np.zeros(row.size)
        if score == "softmax" and there:
            m = max(row[e] for e in there)
            for e in there:
                s[e] = 1.0 if row[e] == m else np.exp(row[e] - m)
            s /= s.sum()
        elif there:
            with np.errstate(over="ignore"):
                s[there] = 1.0 / (1.0 + np.exp(-row[there]))
        s[s < 2.0 ** -1000] = 0.0
        c = s + b
        there = [e for e in there if c[e] > -INF]
        if groups > 1:
            worth = []
            for g in range(groups):
                best = sorted((c[e] for e in there if e // per == g), reverse=True)
                worth.append(sum(best[:group_top]) if best else -INF)
            stay = sorted(range(groups), key=lambda g: (-worth[g], g))[:top_groups]
            there = [e for e in there if e // per in stay]
        rank = row if bias is None else c
        chosen = sorted(there, key=lambda e: (-rank[e], e))[:k]
        ids[t, :len(chosen)] = chosen
        w[t, :len(chosen)] = s[chosen]
        if renorm:
            w[t] = w[t] / w[t].sum() if w[t].sum() > 0 else 0.0
    return ids, w * scale


def run(x, k, score="softmax", bias=None, groups=1, top_groups=1, group_top=1, renorm=True,
        scale=1.0):
    ids = torch.full((x.shape[0], k), -7, dtype=torch.int32, device=DEV)
    w = torch.full((x.shape[0], k), -7.0, device=DEV)
    S.sifar_route(x, ids, w, score, bias, groups, top_groups, group_top, renorm, scale)
    return ids, w


def check(x, k, score="softmax", bias=None, groups=1, top_groups=1, group_top=1, renorm=True,
          scale=1.0):
    ids, w = run(x, k, score, bias, groups, top_groups, group_top, renorm, scale)
    want, ww = definition(x, k, score, bias, groups, top_groups, group_top, renorm, scale)
    got, gw = ids.cpu().numpy(), w.double().cpu().numpy()
    assert np.array_equal(got, want), np.argwhere(got != want)[:4]
    assert (np.abs(gw - ww) <= ww * (2.0 ** -24 + 1e-13) + 2.0 ** -150).all()


def logits(seed, T, E, dtype="fp32", spread=1.5):
    r = np.random.default_rng([2607, seed, T, E])
    return torch.from_numpy(r.standard_normal((T, E)) * spread).to(DT[dtype]).to(DEV)


def balance(seed, E, size=0.1):
    r = np.random.default_rng([2608, seed, E])
    return torch.from_numpy(r.standard_normal(E) * size).float().to(DEV)


@pytest.mark.parametrize("E", [1, 2, 7, 60, 64, 65, 128, 200, 256, 333, 512, 1000, 1024])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("biased", [False, True])
def test_experts(E, score, biased):
    k = min(E, 8)
    bias = balance(1, E, 0.1 if score == "sigmoid" else 0.1 / E) if biased else None
    check(logits(1, 9, E), k, score, bias, renorm=E % 2 == 0, scale=2.5)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("T", [1, 3, 4, 5, 257])
def test_types_and_batches(dtype, T):
    """Rows of 16-bit logits repeat values: ties go to the lower index."""
    check(logits(2, T, 256, dtype), 8)
    check(logits(3, T, 256, dtype), 8, "sigmoid", balance(3, 256), 8, 4, 2, scale=2.5)


@pytest.mark.parametrize("groups,per", [(2, 5), (3, 20), (3, 341), (4, 1), (5, 64), (6, 32),
                                        (8, 32), (9, 113), (16, 64), (17, 60), (20, 3), (32, 32),
                                        (32, 1)])
@pytest.mark.parametrize("group_top", [1, 2])
def test_groups(groups, per, group_top):
    for tg in sorted({1, (groups + 1) // 2, groups}):
        for score, bias in (("sigmoid", balance(4, groups * per)), ("softmax", None)):
            check(logits(4, 6, groups * per), min(8, groups * per), score, bias, groups, tg,
                  group_top)


@pytest.mark.parametrize("k", [1, 2, 10, 31, 32])
def test_topk(k):
    check(logits(5, 5, 512), k, renorm=False)
    check(logits(5, 5, 32), k, "sigmoid", balance(5, 32))


def test_ties():
    x = torch.zeros(3, 100, device=DEV)
    x[1, ::3] = 1.0
    x[2, 50:] = -0.0            # equals +0
    for score in ("softmax", "sigmoid"):
        check(x, 9, score)
        check(x, 9, score, torch.zeros(100, device=DEV))
        check(x, 9, score, torch.zeros(100, device=DEV), 5, 2, 2)
    coarse = (logits(6, 40, 256) * 2).round() / 2
    check(coarse, 12, "sigmoid", (balance(6, 256) * 10).round() / 16, 8, 3, 2)


def test_masked_experts():
    """-inf and NaN are never chosen; a row can run out of experts, or have none."""
    x = logits(7, 8, 48)
    x[0, 3:] = -INF
    x[1] = -INF
    x[2, ::2] = float("nan")
    x[3] = float("nan")
    x[4, :40] = -INF
    x[5, 1:] = -INF
    x[6, 7] = INF
    x[7, 5] = INF
    x[7, 9] = INF
    bias = balance(7, 48)
    for kw in (dict(), dict(score="sigmoid"), dict(bias=bias), dict(score="sigmoid", bias=bias),
               dict(score="sigmoid", bias=bias, groups=6, top_groups=2, group_top=2),
               dict(groups=6, top_groups=3, group_top=1), dict(renorm=False)):
        check(x, 6, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_lowest_values(dtype):
    """Masks of the type's lowest value are ordinary logits: behind all others, and
    equal among themselves."""
    low = torch.finfo(DT[dtype]).min
    x = logits(8, 4, 32, dtype)
    x[0, 2:] = low
    x[1] = low
    x[2, ::2] = low
    for kw in (dict(), dict(score="sigmoid"), dict(bias=torch.zeros(32, device=DEV)),
               dict(score="sigmoid", bias=balance(8, 32), groups=4, top_groups=2, group_top=2)):
        check(x, 8, **kw)


def test_bias_that_is_not_finite():
    x, b = logits(9, 5, 40), balance(9, 40)
    b[3], b[4], b[5] = -INF, float("nan"), INF
    check(x, 6, "sigmoid", b)
    check(x, 6, "softmax", b, 4, 2, 1)


@pytest.mark.parametrize("dtype,bits", [("fp32", 0x7F800001), ("bf16", 0x7F81), ("fp16", 0x7C01)])
def test_signalling_nans_are_not_there(dtype, bits):
    x = logits(15, 5, 130, dtype)
    x.view(torch.int32 if dtype == "fp32" else torch.int16)[:, 3::5] = bits
    for kw in (dict(), dict(score="sigmoid"), dict(renorm=False),
               dict(score="sigmoid", bias=balance(15, 130), groups=10, top_groups=3, group_top=2)):
        check(x, 7, **kw)


def test_saturated_scores_keep_the_order_of_their_logits():
    x = torch.arange(64, device=DEV).float()[None] + 40.0
    ids, _ = run(x, 8, "sigmoid")
    assert ids.tolist() == [list(range(63, 55, -1))]


def test_negative_scores_rank_by_value():
    x = logits(10, 6, 96)
    check(x, 8, "sigmoid", balance(10, 96) - 3.0)
    check(x, 8, "sigmoid", balance(10, 96) - 3.0, 6, 2, 2)


def test_strided_rows_and_odd_addresses():
    for dtype in DT:
        wide = torch.full((7, 101), 50.0, dtype=DT[dtype], device=DEV)
        x = logits(11, 6, 96, dtype)
        wide[:6, 3:99] = x
        ids, w = run(wide[:6, 3:99], 5)
        ids2, w2 = run(x, 5)
        assert torch.equal(ids, ids2) and torch.equal(w, w2)


def test_rows_behind_the_last_stay():
    x = logits(12, 5, 64)
    ids = torch.full((9, 4), -7, dtype=torch.int32, device=DEV)
    w = torch.full((9, 4), -7.0, device=DEV)
    S.sifar_route(x, ids[2:7], w[2:7])
    for buf in (ids, w):
        assert (buf[:2] == -7).all() and (buf[7:] == -7).all()
    assert torch.equal(ids[2:7], run(x, 4)[0])


def test_no_tokens():
    run(torch.empty(0, 64, device=DEV), 4)


def test_far_rows():
    stride = (1 << 30) + 1
    buf = torch.empty(2 * stride + 64, dtype=torch.bfloat16, device=DEV)
    rows = torch.as_strided(buf, (3, 64), (stride, 1))
    rows.copy_(logits(13, 3, 64, "bf16"))
    check(rows, 6)


def test_streams_and_replays():
    x0 = logits(14, 33, 128)
    side = torch.cuda.Stream()
    x = torch.zeros_like(x0)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        x.copy_(x0)
        ids, w = run(x, 4)
    side.synchronize()
    want = run(x0, 4)
    assert torch.equal(ids, want[0]) and torch.equal(w, want[1])
    g = torch.cuda.CUDAGraph()
    bias = balance(14, 128)
    with torch.cuda.graph(g):
        gi, gw = run(x, 4, "sigmoid", bias, 8, 4, 2)
    for k in range(3):
        x.copy_(logits(20 + k, 33, 128))
        g.replay()
        ei, ew = run(x, 4, "sigmoid", bias, 8, 4, 2)
        torch.cuda.synchronize()
        assert torch.equal(gi, ei) and torch.equal(gw, ew)


@pytest.mark.parametrize("biased", [False, True])
def test_most_tokens(biased):
    x = logits(50, S.SIFAR_ROWS_MAX_TOKENS, 3)
    bias = torch.tensor([0.1, 0.0, -0.2], device=DEV) if biased else None
    ids, w = run(x, 1, "sigmoid", bias, renorm=False)
    s = torch.sigmoid(x.double().cpu())
    best = (s + bias.double().cpu() if biased else s).argmax(-1, keepdim=True)
    assert torch.equal(ids.cpu().long(), best)
    s = s.gather(1, best)
    assert ((w.double().cpu() - s).abs() <= s * (2.0 ** -24 + 1e-13)).all()
