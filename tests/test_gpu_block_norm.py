"""GPU: sifar_block_norm against its formula in 64 bits.

The bound on an output is counted, not chosen. u = 2^-24 is half an fp32 step.
A mean square is a sum of at most 64 squares a lane, 6 butterfly steps and 16
waves: 90 roundings, and the square root halves a relative error, so 1/sqrt(...)
is within 45 u + its own 4 operations; with scale, weight and gate each norm's
factor is within 64 u. The partials' sum is off by (parts - 1) u sum|x_p| and the
scaled residual by 2 u of its terms; both then pass through the second norm, whose
mean they shift by at most rms(error) / rms(value). What is stored is off by half
a step of its type more (and half a subnormal step at the bottom)."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2607_08973_amd as S

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    S.load()
    yield
    torch.cuda.synchronize()


def _f64(t):
    return None if t is None else t.detach().double().cpu()


def _rms(t):
    return t.square().mean(-1, keepdim=True).sqrt()


def formula(x, residual, post, gate, norm, bs, rs, off, eps):
    """(r', bound on its error, y, bound) in 64 bits, before the outputs' rounding."""
    x, residual, post, gate, norm = map(_f64, (x, residual, post, gate, norm))
    x = x if x.dim() == 3 else x[None]
    a, err = x.sum(0), (x.shape[0] - 1) * U * x.abs().sum(0)
    if post is not None:
        inv = 1.0 / (a.square().mean(-1, keepdim=True) + eps).sqrt()
        w = (off + post) * inv
        err = w.abs() * err + (a * w).abs() * (64 * U + _rms(err) * inv)
        a = a * w
    g = bs * (1.0 if gate is None else gate)
    a, err = a * g, err * abs(g) if isinstance(g, float) else err * g.abs()
    err = err + 4 * U * a.abs()
    if residual is not None:
        err = err + 2 * U * (a.abs() + (rs * residual).abs())
        a = a + rs * residual
    if norm is None:
        return a, err, None, None
    inv = 1.0 / (a.square().mean(-1, keepdim=True) + eps).sqrt()
    w = (off + norm) * inv
    return a, err, a * w, w.abs() * err + (a * w).abs() * (64 * U + _rms(err) * inv)


def half_step(t, value):
    f = torch.finfo(t)
    return value.abs() * (f.eps / 2) + f.smallest_normal * f.eps / 2


def check(got, want, err):
    g = got.double().cpu()
    bad = ~((g - want).abs() <= err + half_step(got.dtype, want.abs() + err))
    assert not bad.any(), (bad.nonzero()[:4], g[bad][:4], want[bad][:4])


def inputs(seed, T, H, dtype, residual="same", parts=1, post=True, gate="none", off=0.0):
    r = np.random.default_rng([2607, seed, T, H])
    n = lambda *s: torch.from_numpy(r.standard_normal(s))
    dt = DT[dtype]
    x = (n(parts, T, H) * 0.5).to(dt).to(DEV)
    res = None if residual == "none" else n(T, H).to(
        torch.float32 if residual == "fp32" else dt).to(DEV)
    w = lambda: (1.0 - off + 0.1 * n(H)).to(dt).to(DEV)
    g = {"none": None, "channel": n(H).to(dt).to(DEV), "token": n(T, H).to(dt).to(DEV)}[gate]
    rdt = res.dtype if res is not None else (torch.float32 if residual == "fp32" else dt)
    return dict(x=x if parts > 1 else x[0], residual=res, post=w() if post else None, gate=g,
                norm=w(), rdt=rdt)


def run(i, bs=1.0, rs=1.0, off=0.0, eps=1e-6, norm=True, stream=None):
    T, H = i["x"].shape[-2:]
    out = torch.full((T, H), 7.0, dtype=i["rdt"], device=DEV)
    y = torch.full((T, H), 7.0, dtype=i["x"].dtype, device=DEV) if norm else None
    S.sifar_block_norm(i["x"], i["residual"], out, i["post"], i["gate"],
                       i["norm"] if norm else None, y, bs, rs, off, eps, stream)
    return out, y


def check_run(i, out, y, bs=1.0, rs=1.0, off=0.0, eps=1e-6):
    r, e, yy, ey = formula(i["x"], i["residual"], i["post"], i["gate"],
                           i["norm"] if y is not None else None, bs, rs, off, eps)
    check(out, r, e)
    if y is not None:
        check(y, yy, ey)


# one row's vectors: fewer than a wave, one wave, ragged waves, two, four and eight a lane
@pytest.mark.parametrize("H", [8, 512, 520, 1000, 4096, 8192, 8200, 16392, 32776, 65536])
@pytest.mark.parametrize("dtype,residual", [("bf16", "same"), ("bf16", "fp32"), ("fp16", "same"),
                                            ("fp16", "fp32"), ("fp32", "same")])
def test_row_lengths_and_types(H, dtype, residual):
    T = 3 if H > 512 else 7
    i = inputs(1, T, H, dtype, residual, gate="token")
    check_run(i, *run(i))


@pytest.mark.parametrize("T", [1, 2, 5, 130, 1030])
@pytest.mark.parametrize("H", [64, 576])
def test_row_counts(T, H):
    i = inputs(2, T, H, "bf16", gate="channel")
    check_run(i, *run(i))


@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("gate", ["none", "channel", "token"])
@pytest.mark.parametrize("residual", ["none", "same", "fp32"])
@pytest.mark.parametrize("norm", [False, True])
def test_optional_operands_and_scales(post, gate, residual, norm):
    i = inputs(3, 5, 1544, "bf16", residual, parts=3, post=post, gate=gate, off=1.0)
    kw = dict(bs=0.37, rs=0.5, off=1.0, eps=1e-5)
    check_run(i, *run(i, norm=norm, **kw), **kw)


@pytest.mark.parametrize("parts", [2, 5, 8])
@pytest.mark.parametrize("H", [512, 4104, 16392, 40968])
def test_partials(parts, H):
    i = inputs(4, 3, H, "bf16", parts=parts)
    check_run(i, *run(i))


def test_partials_are_summed_in_rank_order():
    """A sum that cancels in rank order only: 2^30 - 2^30 + 1, then + 2^-20."""
    x = torch.zeros(4, 1, 64, dtype=torch.float32, device=DEV)
    for p, v in enumerate((2.0 ** 30, -(2.0 ** 30), 1.0, 2.0 ** -20)):
        x[p] = v
    out = torch.zeros(1, 64, device=DEV)
    S.sifar_block_norm(x, None, out)
    assert (out == 1.0 + 2.0 ** -20).all()


def test_matches_the_all_reduce_epilogue():
    """The plain pre-norm case on an all-reduce's output is sifar_reduce_rmsnorm's: the
    same residual stream bit for bit, y within a step (it is normalised unrounded)."""
    N, T, H = 4, 3, 1024
    r = np.random.default_rng(5)
    n = lambda *s: torch.from_numpy(r.standard_normal(s)).to(torch.bfloat16).to(DEV)
    x, res, w = n(N, T, H), n(T, H), n(H)
    a, y0 = torch.empty_like(res), torch.empty_like(res)
    with S.Sifar(nranks=N, hidden=H, max_tokens=T, reduces_per_step=1) as s:
        s.produce(x, T)
        s.reduce(a, T)
        s.check()
    want = res.clone()
    with S.Sifar(nranks=N, hidden=H, max_tokens=T, reduces_per_step=1, epilogue=1,
                 rms_eps=1e-6) as s:
        s.produce(x, T)
        s.reduce_rmsnorm(want, w, y0, T)
        s.check()
    out, y = torch.empty_like(res), torch.empty_like(res)
    S.sifar_block_norm(a, res, out, norm_weight=w, y=y, eps=1e-6)
    assert torch.equal(out, want)
    # half a step of r' through the norm and two roundings of y
    err = (2.0 ** -8 * 3 + 1e-6) * (y0.double().abs() + y.double().abs()) + 1e-6
    assert ((y.double() - y0.double()).abs() <= err).all()


def test_strided_rows_and_rows_behind_the_last():
    """Views of wider buffers; what lies between and behind the rows stays as it was."""
    T, H, W = 5, 264, 320
    i = inputs(6, T, H, "bf16", parts=2, gate="token")
    wide = lambda t: torch.full((*t.shape[:-2], T + 3, W), 9.0, dtype=t.dtype, device=DEV)
    buf = {k: wide(i[k]) for k in ("x", "residual", "gate")}
    for k, b in buf.items():
        b[..., :T, :H] = i[k]
    out, y = wide(i["residual"]), wide(i["residual"])
    S.sifar_block_norm(buf["x"][:, :T, :H], buf["residual"][:T, :H], out[:T, :H], i["post"],
                       buf["gate"][:T, :H], i["norm"], y[:T, :H])
    check_run(i, out[:T, :H], y[:T, :H])
    for b in (out, y):
        assert (b[T:] == 9.0).all() and (b[:, H:] == 9.0).all()


def test_interleaved_outputs():
    """residual_out and y as the halves of one buffer's rows."""
    i = inputs(7, 6, 128, "bf16")
    both = torch.zeros(6, 256, dtype=torch.bfloat16, device=DEV)
    S.sifar_block_norm(i["x"], i["residual"], both[:, :128], i["post"], None, i["norm"],
                       both[:, 128:])
    check_run(i, both[:, :128], both[:, 128:])


@pytest.mark.parametrize("H", [256, 4096, 16392, 40968])
def test_in_place(H):
    """residual_out over the residual and y over x: the same bits as apart."""
    i = inputs(8, 9, H, "bf16", gate="token")
    out, y = run(i)
    x, res = i["x"].clone(), i["residual"].clone()
    S.sifar_block_norm(x, res, res, i["post"], i["gate"], i["norm"], x)
    assert torch.equal(res, out) and torch.equal(x, y)
    g = i["gate"].clone()
    out2 = torch.empty_like(out)
    S.sifar_block_norm(i["x"], i["residual"], out2, i["post"], g, i["norm"], g)
    assert torch.equal(out2, out) and torch.equal(g, y)


def test_zero_rows_and_values_that_are_not_numbers():
    """A row of zeros stays zero; an infinity or NaN stays in its own row."""
    i = inputs(9, 6, 512, "bf16", residual="none")
    clean_out, clean_y = run(i)
    i["x"] = i["x"].clone()
    i["x"][1] = 0.0
    i["x"][3, 5] = float("inf")
    i["x"][4, 7] = float("nan")
    out, y = run(i)
    assert (out[1] == 0).all() and (y[1] == 0).all()
    assert not torch.isfinite(y[3]).all() and torch.isnan(y[4]).all()
    for t in (0, 2, 5):
        assert torch.equal(out[t], clean_out[t]) and torch.equal(y[t], clean_y[t])


def test_no_tokens():
    z = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device=DEV)
    S.sifar_block_norm(z(0, 64), z(0, 64), z(0, 64), z(64), None, z(64), z(0, 64))


def test_equal_bits_for_a_row_alone_and_in_a_batch():
    """A token's result does not depend on the batch it is in."""
    for H in (256, 4096):
        i = inputs(10, 40, H, "bf16")
        out, y = run(i)
        for t in (0, 17, 39):
            one = dict(i, x=i["x"][t:t + 1], residual=i["residual"][t:t + 1])
            o1, y1 = run(one)
            assert torch.equal(o1[0], out[t]) and torch.equal(y1[0], y[t])


def test_streams_and_replays():
    """On a stream of its own behind the work that makes its inputs; captured and
    replayed on new inputs, with eager calls between the replays."""
    i = inputs(11, 8, 2048, "bf16")
    side = torch.cuda.Stream()
    x = torch.zeros_like(i["x"])
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        x.copy_(i["x"])
        out, y = run(dict(i, x=x))
    side.synchronize()
    check_run(i, out, y)
    g = torch.cuda.CUDAGraph()
    ins = dict(i, x=i["x"].clone(), residual=i["residual"].clone())
    with torch.cuda.graph(g):
        gout, gy = run(ins)
    for k in range(3):
        new = inputs(20 + k, 8, 2048, "bf16")
        ins["x"].copy_(new["x"])
        ins["residual"].copy_(new["residual"])
        g.replay()
        eager = run(ins)
        torch.cuda.synchronize()
        assert torch.equal(gout, eager[0]) and torch.equal(gy, eager[1])


def test_far_rows():
    """Rows past 2^31 elements and 2^32 bytes from the first."""
    H, T = 256, 3
    stride = (1 << 30) + 256 * 8
    buf = torch.empty(2 * stride + H, dtype=torch.bfloat16, device=DEV)
    rows = torch.as_strided(buf, (T, H), (stride, 1))
    i = inputs(12, T, H, "bf16")
    rows.copy_(i["x"])
    out, y = run(dict(i, x=rows))
    check_run(i, out, y)


def test_most_rows():
    i = inputs(60, S.SIFAR_ROWS_MAX_TOKENS, 8, "bf16", gate="channel")
    out, y = run(i)
    check_run(i, out, y)


@pytest.mark.parametrize("H", [6136, 6144, 8192, 12288, 16384])
@pytest.mark.parametrize("parts", [1, 2])
def test_rows_of_many_lanes(H, parts):
    """Around the lengths from which one partial's rows take fewer lanes."""
    i = inputs(61, 3, H, "bf16", "fp32", parts=parts, gate="token")
    out, y = run(i)
    check_run(i, out, y)
