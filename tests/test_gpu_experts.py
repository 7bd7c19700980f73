"""GPU: sifar_experts against its formula in 64 bits.

The bound on an output is counted. u = 2^-24 is half an fp32 step. g and u are sums of
`hidden` products in fp32: within (hidden + 4) u of sum|w x|. The activation's slope is at
most 1.13; its own arithmetic is off by 16 u, and by 3 u of the exponent's argument, of
itself. Between the products h is two bf16 elements (16-bit types), good to 2^-17 each, and
2^-17 of the weight times h is left out with fp16 weights. The second product adds
(inter + 8) u of sum|w h|, the sum over slots topk u. What is stored is off by half a step
of its type more."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import paper_2607_08973_amd as S
from test_gpu_block_norm import DT, half_step

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    S.load()
    yield
    torch.cuda.synchronize()


def formula(i, activation="silu", first_expert=0):
    """(out, bound) in 64 bits on the host."""
    x, w_in, w_out, weights = (i[n].double().cpu() for n in ("x", "w_in", "w_out", "weights"))
    T, H = x.shape
    E, _, I = w_out.shape
    topk = i["ids"].shape[1]
    out, err = torch.zeros(T, H, dtype=torch.float64), torch.zeros(T, H, dtype=torch.float64)
    for t, ids in enumerate(i["ids"].cpu().tolist()):
        for j, e in enumerate(ids):
            e -= first_expert
            if not 0 <= e < E:
                continue
            y, ey = w_in[e] @ x[t], (H + 4) * U * (w_in[e].abs() @ x[t].abs())
            g, u, eg, eu = y[:I], y[I:], ey[:I], ey[I:]
            z = g if activation == "silu" else math.sqrt(8 / math.pi) * (g + 0.044715 * g ** 3)
            a = g * torch.sigmoid(z)
            ea = 1.13 * eg + a.abs() * (16 * U + 3 * U * z.abs())
            h = a * u
            eh = ea * u.abs() + (a.abs() + ea) * eu
            if x.numel() and i["x"].dtype != torch.float32:
                eh = eh + 2.0 ** -16 * h.abs()
            v, w = w_out[e], weights[t, j].abs()
            out[t] += weights[t, j] * (v @ h)
            err[t] += w * (v.abs() @ eh + (I + 8 + topk) * U * (v.abs() @ h.abs()))
    return out, err + 2.0 ** -126


def check(i, out, **kw):
    want, err = formula(i, **kw)
    g = out.double().cpu()
    bad = ~((g - want).abs() <= err + half_step(out.dtype, want.abs() + err))
    assert not bad.any(), (bad.nonzero()[:4], g[bad][:4], want[bad][:4], err[bad][:4])


def inputs(seed, T, E, topk, H, I, dtype="bf16", total=None, ids=None):
    r = np.random.default_rng([2607, 92, seed, T, E, H])
    n = lambda *s: torch.from_numpy(r.standard_normal(s, dtype=np.float32))
    dt = DT[dtype]
    if ids is None:
        ids = np.argsort(r.random((T, total or E)), 1)[:, :topk]
    w = torch.from_numpy(r.random((T, topk), dtype=np.float32) + 0.1)
    return dict(x=n(T, H).to(dt).to(DEV), w_in=(n(E, 2 * I, H) / H ** 0.5).to(dt).to(DEV),
                w_out=(n(E, H, I) / I ** 0.5).to(dt).to(DEV),
                ids=torch.from_numpy(np.asarray(ids, np.int32)).to(DEV).contiguous(),
                weights=w.to(DEV))


def run(i, stream=None, **kw):
    T, topk = i["ids"].shape
    out = torch.full(i["x"].shape, 7.0, dtype=i["x"].dtype, device=DEV)
    ws = torch.full((S.sifar_experts_workspace(T, topk, i["w_out"].shape[2]),), 255,
                    dtype=torch.uint8, device=DEV)  # NaNs, and indices far out of range
    S.sifar_experts(**i, out=out, workspace=ws, stream=stream, **kw)
    torch.cuda.synchronize()
    return out


def run_and_check(i, **kw):
    out = run(i, **kw)
    check(i, out, **kw)
    return out


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("H,I", [(8, 8), (16, 64), (64, 24), (520, 264), (1000, 136), (32, 1032)])
@pytest.mark.parametrize("activation", ["silu", "gelu"])
def test_sizes_types_and_activations(dtype, H, I, activation):
    run_and_check(inputs(1, 5, 6, 2, H, I, dtype), activation=activation)


@pytest.mark.parametrize("T,E,topk", [(1, 1, 1), (1, 128, 8), (2, 3, 3), (16, 4, 1), (17, 1, 1),
                                      (33, 2, 1), (40, 3, 2), (64, 8, 2), (65, 1, 1), (100, 2, 2),
                                      (128, 16, 8), (32, 40, 32), (128, 1, 1), (3, 1024, 5)])
def test_tokens_experts_and_slots(T, E, topk):
    run_and_check(inputs(2, T, E, topk, 72, 40))


@pytest.mark.parametrize("first", [0, 3, 20, 1000])
def test_experts_of_other_ranks(first):
    """Slots of other ranks' experts and empty ones count for nothing; a token without any
    here is zeros."""
    i = inputs(3, 9, 5, 3, 64, 48, total=25)
    i["ids"][2] = -1
    i["ids"][3] = torch.tensor([4, -1, 2 ** 31 - 1])
    i["ids"][4] = torch.tensor([-(2 ** 31), 5, 24])
    out = run_and_check(i, first_expert=first)
    assert (out[2] == 0).all()
    if first == 1000:
        assert (out == 0).all()


def test_nobody_names_an_expert():
    i = inputs(4, 4, 5, 2, 64, 48)
    i["ids"].fill_(-1)
    i["weights"].fill_(float("nan"))
    assert (run(i) == 0).all()


def test_the_same_expert_twice():
    """One token's slots may name one expert several times; each counts."""
    i = inputs(5, 3, 4, 3, 64, 48, ids=[[1, 1, 1], [2, 0, 2], [3, 3, 0]])
    run_and_check(i)
    i = inputs(6, 40, 3, 25, 64, 48, ids=np.random.default_rng(6).integers(0, 3, (40, 25)))
    run_and_check(i)  # 1000 slots: hundreds of columns of an expert


def test_a_weight_that_is_zero_or_negative():
    i = inputs(7, 6, 4, 2, 64, 48)
    i["weights"][:, 0] = 0
    i["weights"][2:, 1] *= -3
    run_and_check(i)


def test_only_what_is_named_is_read():
    """Experts that nobody named may hold anything."""
    i = inputs(8, 4, 8, 2, 64, 48, ids=[[1, 2], [2, 6], [6, 1], [1, 2]])
    want = run_and_check(i)
    for e in (0, 3, 4, 5, 7):
        i["w_in"][e] = float("nan")
        i["w_out"][e] = float("inf")
    assert torch.equal(run(i), want)


def test_values_that_fp16_cannot_hold():
    """h beyond fp16's largest number, brought back by w_out."""
    i = inputs(9, 3, 2, 1, 64, 48, "fp16")
    i["w_in"].mul_(60)
    i["x"].mul_(30)
    i["w_out"].div_(4000)
    h, _ = formula(i)
    assert torch.isfinite(h).all()
    g = i["w_in"][0].double() @ i["x"][0].double()
    assert float((g[:48] * g[48:]).abs().max()) > 65504
    run_and_check(i)


def test_extreme_gates():
    """Gates where the exponential is 0 or infinite."""
    for activation in ("silu", "gelu"):
        i = inputs(10, 4, 2, 1, 64, 48, "fp32")
        i["w_in"][:, :48].mul_(150)
        run_and_check(i, activation=activation)


def test_one_token_does_not_disturb_another():
    """NaN in a token's row stays in it."""
    i = inputs(11, 20, 3, 2, 64, 48)
    want = run(i)
    i["x"][7] = float("nan")
    got = run(i)
    assert got[7].isnan().all()
    keep = [t for t in range(20) if t != 7]
    assert torch.equal(got[keep], want[keep])


def test_strided_rows_and_rows_behind_the_last():
    i = inputs(12, 5, 4, 2, 64, 48)
    want = run(i)
    x = torch.full((8, 96), float("nan"), dtype=torch.bfloat16, device=DEV)
    x[:5, 16:80] = i["x"]
    out = torch.full((8, 96), 9.0, dtype=torch.bfloat16, device=DEV)
    w_in = torch.full((4, 120, 64), float("nan"), dtype=torch.bfloat16, device=DEV)
    w_in[:, :96] = i["w_in"]
    ws = torch.zeros(S.sifar_experts_workspace(5, 2, 48), dtype=torch.uint8, device=DEV)
    S.sifar_experts(x[:5, 16:80], i["ids"], i["weights"], w_in[:, :96], i["w_out"], out[:5, 16:80], ws)
    assert torch.equal(out[:5, 16:80], want)
    assert (out[5:] == 9.0).all() and (out[:, :16] == 9.0).all() and (out[:, 80:] == 9.0).all()


def test_offsets_beyond_32_bits():
    """Experts 1.2e9 elements apart: the third's matrices lie 4.8 GB in."""
    far = 1_200_000_000
    buf = torch.empty(2 * far + 20000, dtype=torch.bfloat16, device=DEV)
    i = inputs(13, 4, 3, 2, 64, 48, ids=[[2, 0], [1, 2], [2, 1], [0, 1]])
    for name, at, shape in (("w_in", 0, (3, 96, 64)), ("w_out", 8192, (3, 64, 48))):
        w = torch.as_strided(buf, shape, (far, shape[2], 1), at)
        w.copy_(i[name])
        i[name] = w
    run_and_check(i)


def test_equal_inputs_give_equal_bits():
    i = inputs(14, 50, 7, 4, 264, 136)
    assert torch.equal(run(i), run(i))


def test_streams_and_graphs():
    """Graphs that share a workspace, replayed with other ids in between: the plan is made
    anew each time."""
    steps = [inputs(15, 9, 6, 2, 64, 48), inputs(16, 9, 6, 2, 64, 48)]
    ws = torch.zeros(S.sifar_experts_workspace(9, 2, 48), dtype=torch.uint8, device=DEV)
    outs = [torch.zeros_like(i["x"]) for i in steps]
    graphs = []
    for i, out in zip(steps, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            S.sifar_experts(**i, out=out, workspace=ws)
        graphs.append(g)
    r = np.random.default_rng(17)
    for k in range(4):
        for i, out, g in zip(steps, outs, graphs):
            i["ids"].copy_(torch.from_numpy(r.integers(-1, 6, (9, 2)).astype(np.int32)))
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, run(i)), k
    check(steps[0], outs[0])
    out = run(steps[1], stream=torch.cuda.Stream())
    assert torch.equal(out, outs[1])
