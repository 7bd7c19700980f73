"""GPU: sifar_cache_append against its formula in 64 bits.

The bound on a rotated element is counted. u = 2^-24 is half an fp32 step. What is left of
an angle behind its quadrant goes to fp32 once and is multiplied by pi / 2 once (a
constant that is off by less than u): 3 u of at most pi / 4. The series are off by 2e-9
and end in two roundings of numbers up to 1: cosine and sine within 5 u, and 6 u with
rotary_scale. In 64 bits the angle itself is off by 2^-51 of its size (a product, the
constant 2 / pi, a product). Two products and their sum add 2 u: an element is within
(8 u + 2^-51 |angle|) scale (|a| + |b|), and half a step of its type where it is stored.
Copied elements are the same bits."""
from __future__ import annotations

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


def rotated(x, positions, inv_freq, interleaved, scale):
    """(formula in 64 bits, bound) of x [T][H][D] on the host."""
    x = x.detach().double().cpu()
    n = inv_freq.shape[0]
    if n == 0:
        return x, torch.zeros_like(x)
    angle = positions.double().cpu()[:, None] * inv_freq.double().cpu()
    c, s = scale * torch.cos(angle)[:, None], scale * torch.sin(angle)[:, None]
    off = ((8 * U + 2.0 ** -51 * angle.abs()) * abs(scale))[:, None]
    at = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    a, b = x[..., at[0]], x[..., at[1]]
    want, err = x.clone(), torch.zeros_like(x)
    want[..., at[0]], want[..., at[1]] = a * c - b * s, a * s + b * c
    err[..., at[0]] = err[..., at[1]] = off * (a.abs() + b.abs())
    return want, err


def check(got, want, err):
    g = got.detach().double().cpu()
    same = err == 0  # copied
    assert torch.equal(g[same], want[same])
    bad = ~same & ~((g - want).abs() <= err + half_step(got.dtype, want.abs() + err))
    assert not bad.any(), (bad.nonzero()[:4], g[bad][:4], want[bad][:4])


def inputs(seed, T, Hq, Hk, D, page, dtype="bf16", sequences=None, width=6, furthest=None,
           layout="slots"):
    """Tokens of random sequences at positions of their own; a table of distinct pages."""
    r = np.random.default_rng([2607, 90, seed, T, D])
    n = lambda *s: torch.from_numpy(r.standard_normal(s)).to(DT[dtype]).to(DEV)
    sequences = sequences or T
    reach = min(width * page, furthest or width * page)
    slots = r.permutation(sequences * reach)[:T] if sequences * reach < 10 ** 6 else (
        r.integers(0, sequences * reach, T))
    pool = sequences * width + 3
    pages = torch.from_numpy(r.permutation(pool)[:sequences * width].astype(np.int32)).view(
        sequences, width).to(DEV)
    both = n(2, pool, page, Hk, D)
    if layout == "heads":
        both = both.permute(0, 1, 3, 2, 4).contiguous().permute(0, 1, 3, 2, 4)
    elif layout == "both":
        both = both.transpose(0, 1).contiguous().transpose(0, 1)
    x = n(T, Hq + 2 * Hk, D)
    i32 = lambda v: torch.from_numpy(v.astype(np.int32)).to(DEV)
    return dict(q=x[:, :Hq], k=x[:, Hq:Hq + Hk], v=x[:, Hq + Hk:], positions=i32(slots % reach),
                sequence=i32(slots // reach), pages=pages, k_cache=both[0], v_cache=both[1])


def freqs(rotary, base=10000.0):
    return (base ** (-torch.arange(0, rotary, 2).double() / max(rotary, 1))).float().to(DEV)


def run_and_check(i, rotary, interleaved=False, scale=1.0, **kw):
    f = freqs(rotary)
    k0, v0 = i["k_cache"].clone(), i["v_cache"].clone()
    q_out = torch.full(i["q"].shape, 7.0, dtype=i["q"].dtype, device=DEV)
    S.sifar_cache_append(**i, q_out=q_out, inv_freq=f if rotary else None, interleaved=interleaved,
                         rotary_scale=scale, **kw)
    torch.cuda.synchronize()
    check(q_out, *rotated(i["q"], i["positions"], f, interleaved, scale))
    page = k0.shape[1]
    at = i["positions"].long()
    seq = i["sequence"].long() if i["sequence"] is not None else torch.arange(at.numel(), device=DEV)
    row, slot = i["pages"][seq, at // page].long(), at % page
    check(i["k_cache"][row, slot], *rotated(i["k"], i["positions"], f, interleaved, scale))
    assert torch.equal(i["v_cache"][row, slot], i["v"])
    for c, before in ((i["k_cache"], k0), (i["v_cache"], v0)):  # every other slot as it was
        now = c.clone()
        now[row, slot] = before[row, slot]
        assert torch.equal(now.view(torch.int16 if c.element_size() == 2 else torch.int32),
                           before.view(torch.int16 if c.element_size() == 2 else torch.int32))


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("D,rotary", [(8, 8), (8, 2), (64, 64), (80, 40), (96, 32), (128, 128),
                                      (128, 8), (192, 128), (256, 256), (256, 0), (104, 6)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_head_dims_and_rotated_parts(dtype, D, rotary, interleaved):
    run_and_check(inputs(1, 5, 6, 2, D, 16, dtype), rotary, interleaved, scale=1.25)


@pytest.mark.parametrize("T", [1, 2, 63, 257])
@pytest.mark.parametrize("Hq,Hk", [(1, 1), (8, 8), (40, 5), (71, 1)])
def test_tokens_and_heads(T, Hq, Hk):
    run_and_check(inputs(2, T, Hq, Hk, 64, 8, sequences=min(T, 9), width=20), 64)


@pytest.mark.parametrize("page", [1, 7, 16, 24, 128])
@pytest.mark.parametrize("layout", ["slots", "heads", "both"])
def test_pages_and_layouts(page, layout):
    run_and_check(inputs(3, 11, 4, 2, 128, page, layout=layout), 128)


def test_most_heads():
    run_and_check(inputs(4, 2, 1024, 1024, 24, 2), 16)


def test_far_positions():
    """A million positions on, and at the end of 31 bits: angles keep their exactness."""
    i = inputs(5, 16, 4, 2, 128, 65536, "fp32", sequences=1, width=2, furthest=131072)
    table = torch.full((1, 32768), -1, dtype=torch.int32, device=DEV)
    for first in (15, 32766):
        t = dict(i, positions=i["positions"] + first * 65536, pages=table.clone())
        t["pages"][0, first:first + 2] = i["pages"][0]
        run_and_check(t, 128)
        assert int(t["positions"].max()) > 2 ** (20 if first == 15 else 31) - 65536


def test_without_queries_and_without_sequence():
    i = inputs(6, 7, 3, 2, 64, 16)
    i["sequence"] = None
    i["positions"] = torch.arange(7, dtype=torch.int32, device=DEV) * 13
    run_and_check(i, 64)
    before = i["k_cache"].clone()
    i["k_cache"].zero_()
    i["v_cache"].zero_()
    del i["q"]
    S.sifar_cache_append(**i, inv_freq=freqs(64))
    keep = i["k_cache"] != 0
    assert torch.equal(i["k_cache"][keep], before[keep]) and int(keep.sum()) > 7 * 2 * 60


def test_queries_in_place_and_strided_rows():
    i = inputs(7, 9, 4, 2, 64, 16, "fp16")
    q0, f = i["q"].clone(), freqs(64)
    S.sifar_cache_append(**i, q_out=i["q"], inv_freq=f)  # a view of the projection's rows
    check(i["q"], *rotated(q0, i["positions"], f, False, 1.0))
    wide = torch.full((12, 400), 9.0, dtype=torch.float16, device=DEV)
    out = wide[:9, 16:16 + 256].unflatten(1, (4, 64))
    i["q"] = q0
    S.sifar_cache_append(**i, q_out=out, inv_freq=f)
    check(out, *rotated(q0, i["positions"], f, False, 1.0))
    assert (wide[9:] == 9.0).all() and (wide[:, :16] == 9.0).all() and (wide[:, 272:] == 9.0).all()


def test_padding_and_pages_that_are_not_there():
    """Negative positions leave everything as it was; positions without a page (the table
    says so, or ends before) and unknown sequences leave the cache as it was."""
    i = inputs(8, 10, 4, 2, 64, 16, sequences=10, width=4)
    p = torch.tensor([5, -1, 17, -(2 ** 31), 40, 63, 64, 2 ** 31 - 1, 3, 9], dtype=torch.int32)
    i["positions"] = p.to(DEV)
    s = torch.tensor([0, 1, 2, 3, 4, 5, 6, 7, -1, 10], dtype=torch.int32)
    i["sequence"] = s.to(DEV)
    pool = i["k_cache"].shape[0]
    i["pages"][2, 1] = -1
    i["pages"][4, 2] = pool
    k0, v0 = i["k_cache"].clone(), i["v_cache"].clone()
    q_out = torch.full(i["q"].shape, 7.0, dtype=i["q"].dtype, device=DEV)
    S.sifar_cache_append(**i, q_out=q_out, inv_freq=freqs(64))
    want, err = rotated(i["q"], i["positions"].clamp(min=0), freqs(64), False, 1.0)
    live = p >= 0
    check(q_out[live.to(DEV)], want[live], err[live])
    assert (q_out[~live.to(DEV)] == 7.0).all()
    for c, before, x in ((i["k_cache"], k0, i["k"]), (i["v_cache"], v0, i["v"])):
        for t in (0, 5):  # the only two with a slot
            row = int(i["pages"][t, int(p[t]) // 16])
            assert not torch.equal(c[row, int(p[t]) % 16], before[row, int(p[t]) % 16])
            c[row, int(p[t]) % 16] = before[row, int(p[t]) % 16]
        assert torch.equal(c, before)


def test_offsets_beyond_32_bits():
    """Pages 1.2e9 elements apart: the third lies 4.8 GB in."""
    far, D = 1_200_000_000, 64
    cache = torch.empty(2 * far + 4096, dtype=torch.bfloat16, device=DEV)
    view = lambda at: torch.as_strided(cache, (3, 16, 1, D), (far, D, D, 1), at)
    kc, vc = view(0), view(2048)
    kc.zero_(), vc.zero_()
    i = inputs(9, 3, 2, 1, D, 16, sequences=3, width=1)
    i.update(k_cache=kc, v_cache=vc, positions=torch.tensor([3, 9, 15], dtype=torch.int32, device=DEV),
             sequence=None, pages=torch.tensor([[2], [1], [0]], dtype=torch.int32, device=DEV))
    run_and_check(i, D)


def test_elements_keep_their_bits():
    """NaN payloads, infinities and signed zeros of values and of what is not rotated."""
    i = inputs(10, 2, 2, 1, 32, 16)
    bits = torch.tensor([0x7FC1, -0x3F, 0x7F80, -0x80, -0x8000, 1, 0x7F81, 0x7FFF],
                        dtype=torch.int16, device=DEV)
    for name in ("q", "k", "v"):
        i[name][..., 8:16] = bits.view(torch.bfloat16)
    for interleaved in (False, True):
        q_out = torch.empty_like(i["q"])
        S.sifar_cache_append(**i, q_out=q_out, inv_freq=freqs(8), interleaved=interleaved)
        at = i["positions"].long()
        row = i["pages"][i["sequence"].long(), at // 16].long()
        for got in (q_out, i["k_cache"][row, at % 16], i["v_cache"][row, at % 16]):
            assert (got[..., 8:16].contiguous().view(torch.int16) == bits).all()


def test_another_stream_and_a_graph():
    i, f = inputs(11, 6, 4, 2, 64, 16), freqs(64)
    q_out = torch.zeros(i["q"].shape, dtype=torch.bfloat16, device=DEV)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    S.sifar_cache_append(**i, q_out=q_out, inv_freq=f, stream=st)
    torch.cuda.synchronize()
    check(q_out, *rotated(i["q"], i["positions"], f, False, 1.0))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        S.sifar_cache_append(**i, q_out=q_out, inv_freq=f)
    for k in range(3):
        i["positions"].copy_((i["positions"] + 7) % 96)
        i["q"].copy_(torch.randn(i["q"].shape, device=DEV).to(torch.bfloat16))
        q_out.zero_()
        g.replay()
        torch.cuda.synchronize()
        check(q_out, *rotated(i["q"], i["positions"], f, False, 1.0))
        at = i["positions"].long()
        row = i["pages"][i["sequence"].long(), at // 16].long()
        assert torch.equal(i["v_cache"][row, at % 16], i["v"])
