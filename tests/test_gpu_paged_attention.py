"""GPU: sifar_paged_attention against its formula in 64 bits.

The bound on an output is counted. u = 2^-24 is half an fp32 step. A score is a sum of D
products in fp32: within (D + 2) u of scale sum|q k|; scaling it to base 2, taking the
maximum off and the exponential itself add 8 u and 3 u of its size. Bounded scores (tanh)
shrink errors and add 16 u of the cap. So a weight is within e_p of itself, e_p being
what its score is off by; the maximum's own error cancels, and

    |out - exact| <= sum_p w_p e_p (|v_p| + |out|) + n u (sum_p w_p |v_p| + |out|)

with w the exact weights and n the roundings on the way of a summand: one for each tile
of 32 positions a wave takes and for each rescaling, the joins of four waves and of all
chunks, counted by length / 16 + 64. 16-bit elements have each weight as two of their kind,
which leaves 2^-16. What is stored is off by half a step of its type more. lse is off by
the largest e_p, and 8 u of itself and of the largest score in base 2."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import paper_2607_08973_amd as S
from test_gpu_block_norm import DT, half_step

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
INF = float("inf")


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    S.load()
    yield
    torch.cuda.synchronize()


def formula(i, t, max_length=None, scale=None, window=0, softcap=0.0):
    """Row t: (out, bound, lse, bound) in 64 bits on the host."""
    q = i["q"][t].double().cpu()
    Hq, D = q.shape
    kc, vc, pages = i["k_cache"], i["v_cache"], i["pages"][t].cpu()
    page, Hk = kc.shape[1], kc.shape[2]
    n = max(0, min(int(i["lengths"][t]), pages.numel() * page, max_length or 1 << 40))
    at = torch.arange(max(0, n - window) if window else 0, n)
    row = pages[at // page].long()
    at = at[(row >= 0) & (row < kc.shape[0])]
    row = pages[at // page].long().to(DEV)
    k = kc[row, (at % page).to(DEV)].double().cpu().transpose(0, 1)  # [Hk][n][D]
    v = vc[row, (at % page).to(DEV)].double().cpu().transpose(0, 1)
    g = Hq // Hk
    k, v = k.repeat_interleave(g, 0), v.repeat_interleave(g, 0)
    scale = D ** -0.5 if scale is None else scale
    x = scale * (k @ q[:, :, None])[..., 0]
    e = (D + 2) * U * abs(scale) * (k.abs() @ q.abs()[:, :, None])[..., 0] + 11 * U * x.abs() + 8 * U
    if softcap:
        x = softcap * torch.tanh(x / softcap)
        e = e + 16 * U * softcap
    sink = i.get("sinks")
    sink = torch.full((Hq,), -INF, dtype=torch.float64) if sink is None else sink.double().cpu()
    top = torch.maximum(x.amax(-1), sink) if at.numel() else sink
    e = e + 3 * U * (top[:, None] - x).abs().nan_to_num(0.0, 0.0, 0.0)
    lse = torch.logsumexp(torch.cat([x, sink[:, None]], 1), 1)
    w = torch.where(torch.isinf(lse)[:, None], 0.0, torch.exp(x - lse[:, None]))
    out = (w[:, None] @ v)[:, 0]
    rough = at.numel() / 16 + 64
    tiny = 2.0 ** -16 if i["q"].dtype != torch.float32 else 0.0
    err = ((w * (e + tiny + rough * U))[:, None] @ v.abs())[:, 0] + (
        (w * e).sum(-1, keepdim=True) + rough * U) * out.abs()
    # fp32's own smallest step: of products with weights below it
    err = err + 2.0 ** -126
    span = x.abs().amax(-1) if at.numel() else torch.zeros(Hq, dtype=torch.float64)
    off = (e.amax(-1) if at.numel() else 0.0) + 8 * U * (lse.abs().nan_to_num(0.0, 0.0, 0.0) + span) \
        + rough * U
    return out, err, lse, off


def check(i, out, lse, rows=None, **kw):
    for t in range(out.shape[0]) if rows is None else rows:
        want, err, wl, el = formula(i, t, **kw)
        g = out[t].double().cpu()
        bad = ~((g - want).abs() <= err + half_step(out.dtype, want.abs() + err))
        assert not bad.any(), (t, bad.nonzero()[:4], g[bad][:4], want[bad][:4])
        if lse is not None:
            l = lse[t].double().cpu()
            none = torch.isinf(wl)
            assert torch.equal(l[none], wl[none])
            assert ((l - wl).abs()[~none] <= (el + 0 * wl)[~none]).all(), (t, l, wl)


def inputs(seed, lengths, Hq, Hk, D, page, dtype="bf16", width=None, layout="slots", spread=2.0,
           sinks=False):
    r = np.random.default_rng([2607, 91, seed, len(lengths), D])
    n = lambda *s: torch.from_numpy(r.standard_normal(s, dtype=np.float32)).to(DT[dtype]).to(DEV)
    T = len(lengths)
    counts = [-(-max(x, 0) // page) for x in lengths]
    width = width or max(1, max(counts))
    pool = sum(counts) + 3
    order = r.permutation(pool).astype(np.int32)
    pages = np.full((T, width), -1, np.int32)
    at = 0
    for t, c in enumerate(counts):
        c = min(c, width)
        pages[t, :c] = order[at:at + c]
        at += c
    both = n(2, pool, page, Hk, D)
    if layout == "heads":
        both = both.permute(0, 1, 3, 2, 4).contiguous().permute(0, 1, 3, 2, 4)
    elif layout == "both":
        both = both.transpose(0, 1).contiguous().transpose(0, 1)
    q = torch.from_numpy(spread * r.standard_normal((T, Hq, D))).to(DT[dtype]).to(DEV)
    s = torch.from_numpy(r.standard_normal(Hq, dtype=np.float32)).to(DEV) if sinks else None
    return dict(q=q, k_cache=both[0], v_cache=both[1], pages=torch.from_numpy(pages).to(DEV),
                lengths=torch.tensor(lengths, dtype=torch.int32, device=DEV), sinks=s)


def run(i, max_length=None, stream=None, lse=True, **kw):
    T, Hq, D = i["q"].shape
    Hk, page = i["k_cache"].shape[2], i["k_cache"].shape[1]
    out = torch.full((T, Hq, D), 7.0, dtype=i["q"].dtype, device=DEV)
    l = torch.full((T, Hq), 7.0, device=DEV) if lse else None
    n = S.sifar_paged_attention_workspace(T, Hq, Hk, D,
                                          max_length or i["pages"].shape[1] * page)
    ws = torch.full((n,), 255, dtype=torch.uint8, device=DEV) if n else None  # NaNs
    S.sifar_paged_attention(**i, out=out, workspace=ws, max_length=max_length, lse=l, stream=stream,
                            **kw)
    torch.cuda.synchronize()
    return out, l


def run_and_check(i, **kw):
    out, lse = run(i, **kw)
    kw.pop("stream", None)
    check(i, out, lse, **kw)
    return out, lse


# one position, tiles' and chunks' edges, several chunks
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("D", [8, 64, 80, 128, 136, 256])
def test_lengths_dims_and_types(D, dtype):
    run_and_check(inputs(1, [1, 2, 15, 16, 17, 31, 32, 33, 127, 128, 129, 255, 256, 257, 300, 1000],
                         4, 2, D, 16, dtype, sinks=D == 80))


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_more_than_the_caches_keep(D, dtype):
    """Tables with room for so much that keys and values are loaded past the caches, and chunks
    of one tile to a dozen for each wave."""
    i = inputs(22, [1, 31, 33, 255, 700, 1537, 3001, 9000], 4, 2, D, 512, dtype,
               width=-(-2 ** 27 // (8 * 2 * 2 * D * 512 * i_size(dtype))) + 1)
    run_and_check(i)
    run_and_check(i, window=1200, softcap=20.0)


def i_size(dtype):
    return 4 if dtype == "fp32" else 2


@pytest.mark.parametrize("Hq,Hk", [(1, 1), (3, 3), (5, 1), (15, 5), (16, 1), (17, 1), (34, 2),
                                   (64, 1), (48, 16)])
def test_head_groups(Hq, Hk):
    run_and_check(inputs(2, [5, 700], Hq, Hk, 64, 16))


@pytest.mark.parametrize("page", [1, 3, 16, 24, 100, 512])
@pytest.mark.parametrize("layout", ["slots", "heads", "both"])
def test_pages_and_layouts(page, layout):
    run_and_check(inputs(3, [1, 99, 100, 101, 517], 4, 2, 128, page, "fp16", layout=layout))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kw", [
    dict(window=1), dict(window=64), dict(window=300), dict(window=5000), dict(softcap=1.0),
    dict(softcap=50.0, window=17), dict(scale=1.0), dict(scale=-0.3), dict(scale=0.0)], ids=str)
def test_windows_caps_and_scales(kw, dtype):
    run_and_check(inputs(4, [1, 16, 64, 65, 333, 900], 4, 2, 64, 16, dtype, sinks=True), **kw)


def test_a_long_sequence_beside_short_ones():
    run_and_check(inputs(5, [3, 20001, 1, 4096, 0, 2049], 8, 2, 128, 64))
    run_and_check(inputs(6, [33000], 2, 1, 64, 32, "fp16"), window=30001)


def test_many_sequences():
    """So many that none is shared: one launch."""
    r = np.random.default_rng(7)
    i = inputs(7, [int(x) for x in r.integers(0, 256, 1500)], 4, 2, 64, 16)
    out, lse = run(i, max_length=256)
    check(i, out, lse, rows=list(range(0, 1500, 13)), max_length=256)
    # and so many that are, by length
    i = inputs(8, [int(x) for x in r.integers(0, 5000, 300)], 4, 4, 64, 16)
    out, lse = run(i)
    check(i, out, lse, rows=list(range(0, 300, 7)))


@pytest.mark.parametrize("sinks", [False, True])
@pytest.mark.parametrize("width", [2, 40])
def test_rows_without_a_position(sinks, width):
    """Length zero and below, pages that are not there: zeros, and lse -inf or the sink."""
    i = inputs(9, [0, 5, -3, 20], 4, 2, 64, 16, sinks=sinks, width=width)
    i["pages"][3] = torch.tensor([-1, 1 << 20] + [-5] * (width - 2), dtype=torch.int32, device=DEV)
    out, lse = run_and_check(i)
    for t in (0, 2, 3):
        assert (out[t] == 0).all()
        if not sinks:
            assert (lse[t] == -INF).all()


def test_pages_that_are_not_there_in_between():
    i = inputs(10, [200, 600], 4, 2, 128, 16)
    i["pages"][0, 3] = -1
    i["pages"][0, 12] = i["k_cache"].shape[0]
    i["pages"][1, ::2] = -7
    run_and_check(i)


def test_lengths_beyond_what_is_known():
    """Cut to max_length and to the table."""
    i = inputs(11, [100, 64, 30], 4, 2, 64, 16, width=4)
    i["lengths"][1] = 2 ** 31 - 1
    run_and_check(i)
    run_and_check(i, max_length=33)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("value", [float("nan"), INF, -INF])
@pytest.mark.parametrize("D", [64, 80, 256])
def test_what_is_not_read_has_no_influence(dtype, value, D):
    """NaN and infinities behind lengths, before windows, and in the first page's first slot,
    which stands in for positions that are not there."""
    i = inputs(12, [5, 37, 300], 4, 2, D, 16, dtype)
    kw = dict(window=280)
    want = run(i, **kw)
    used = torch.zeros(i["k_cache"].shape[:2], dtype=torch.bool)
    for t, n in enumerate(i["lengths"].tolist()):
        for p in range(max(0, n - 280), n):
            used[int(i["pages"][t, p // 16]), p % 16] = True
    free = (~used).nonzero()
    for c in ("k_cache", "v_cache"):
        i[c][free[:, 0].to(DEV), free[:, 1].to(DEV)] = value
    if used[0, 0]:  # make the stand-in poisonous too
        other = int((~used).all(1).nonzero()[0])
        i["pages"][i["pages"] == 0] = other
        for c in ("k_cache", "v_cache"):
            i[c][other] = i[c][0]
            i[c][0] = value
    got = run(i, **kw)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_scores_that_are_not_finite():
    """-inf has no weight, a row of them nothing; NaN and +inf make their own head's row NaN."""
    i = inputs(13, [50, 50, 50], 4, 4, 64, 16, "fp32")
    p = i["pages"]
    i["q"][:, 0] = i["q"][:, 0].abs()
    i["k_cache"][int(p[0, 1]), 3, 0] = -INF      # one position of head 0
    i["k_cache"][p[1, :4].long(), :, 0] = -INF   # all of them
    i["k_cache"][int(p[2, 0]), 5, 1, 7] = float("nan")
    i["q"][2, 2] = i["q"][2, 2].abs()
    i["k_cache"][int(p[2, 2]), 1, 2] = INF
    out, lse = run(i)
    keep = [x for x in range(50) if x != 16 + 3]
    k = i["k_cache"][p[0].long()].flatten(0, 1)[:50, 0].double().cpu()[keep]
    v = i["v_cache"][p[0].long()].flatten(0, 1)[:50, 0].double().cpu()[keep]
    w = torch.softmax(k @ i["q"][0, 0].double().cpu() / 8.0, 0)
    assert ((out[0, 0].double().cpu() - w @ v).abs() < 1e-5).all()
    assert (out[1, 0] == 0).all() and lse[1, 0] == -INF
    for h in (1, 2):
        assert out[2, h].isnan().all() and lse[2, h].isnan()
    for t, h in ((0, 1), (0, 3), (1, 1), (1, 2), (2, 0), (2, 3)):
        want, err, wl, el = formula(i, t)
        assert ((out[t, h].double().cpu() - want[h]).abs() <= err[h] + half_step(
            torch.float32, want[h].abs())).all()


def test_weights_spread_over_all_exponents():
    """One position outweighs the others by 2^40, or all weigh the same: both ends of the
    running maximum, which grows in every tile of one row and never in another."""
    for dtype in ("bf16", "fp16", "fp32"):
        i = inputs(14, [1000, 1000, 1000], 1, 1, 64, 16, dtype, spread=0.0)
        i["q"][:, 0, 0] = 8.0
        order = torch.arange(1000, device=DEV)
        for t, x in enumerate((order / 50.0, -order / 50.0, (order == 517) * 27.0)):
            rows = i["pages"][t].long()[order // 16]
            i["k_cache"][rows, order % 16] = 0
            i["k_cache"][rows, order % 16, 0, 0] = x.to(i["q"].dtype)
        run_and_check(i)


def test_fp16_sums_of_many_small_weights():
    """60000 positions 2^-15 of the largest hold two thirds of the weight: 16-bit weights
    would round them to multiples of 2^-24."""
    n = 60000
    i = inputs(15, [n], 1, 1, 64, 64, "fp16", spread=0.0)
    i["k_cache"].zero_()
    i["q"][0, 0, 0] = 10.0
    i["k_cache"][int(i["pages"][0, 0]), 0, 0, 0] = 8.3
    i["v_cache"].copy_(i["v_cache"].abs())
    run_and_check(i)


def test_matches_what_was_appended():
    """Keys and values by sifar_cache_append, token by token, attended to after each."""
    page, D = 16, 64
    i = inputs(16, [40], 4, 2, D, page)
    r = np.random.default_rng(16)
    k, v = (torch.from_numpy(r.standard_normal((40, 2, D))).to(torch.bfloat16).to(DEV) for _ in "kv")
    f = (10000.0 ** (-torch.arange(0, D, 2).double() / D)).float().to(DEV)
    q_out = torch.empty_like(i["q"])
    for p in range(40):
        S.sifar_cache_append(k[p:p + 1], v[p:p + 1],
                             torch.tensor([p], dtype=torch.int32, device=DEV), i["pages"],
                             i["k_cache"], i["v_cache"], q=i["q"], q_out=q_out, inv_freq=f)
        if p % 13 == 0 or p == 39:
            run_and_check(dict(i, q=q_out, lengths=torch.tensor([p + 1], dtype=torch.int32,
                                                                device=DEV)))


def test_queries_in_place_and_strided_rows():
    i = inputs(17, [40, 700, 9], 4, 2, 64, 16, "fp16")
    want, _ = run(i)
    wide = torch.full((5, 400), 9.0, dtype=torch.float16, device=DEV)
    view = wide[:3, 16:16 + 256].unflatten(1, (4, 64))
    view.copy_(i["q"])
    n = S.sifar_paged_attention_workspace(3, 4, 2, 64, i["pages"].shape[1] * 16)
    ws = torch.zeros(n, dtype=torch.uint8, device=DEV)
    S.sifar_paged_attention(**dict(i, q=view), out=view, workspace=ws)
    assert torch.equal(view, want)
    assert (wide[3:] == 9.0).all() and (wide[:, :16] == 9.0).all() and (wide[:, 272:] == 9.0).all()


def test_offsets_beyond_32_bits():
    far, D = 1_200_000_000, 64
    cache = torch.empty(2 * far + 4096, dtype=torch.bfloat16, device=DEV)
    view = lambda at: torch.as_strided(cache, (3, 16, 1, D), (far, D, D, 1), at)
    i = inputs(18, [48], 2, 1, D, 16)
    i.update(k_cache=view(0), v_cache=view(2048),
             pages=torch.tensor([[2, 0, 1]], dtype=torch.int32, device=DEV))
    for c in ("k_cache", "v_cache"):
        i[c].copy_(torch.randn(i[c].shape, device=DEV).to(torch.bfloat16))
    run_and_check(i)


def test_equal_inputs_give_equal_bits():
    i = inputs(19, [5000, 17, 900], 8, 2, 128, 16)
    a, b = run(i), run(i)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_streams_and_graphs():
    """Two captured graphs that share a workspace, replayed one after the other with eager
    calls between, lengths growing as a decode's do; and a call on a stream of its own."""
    steps = [inputs(20, [100, 700, 1, 0], 8, 2, 64, 16, width=60),
             inputs(21, [900, 5, 300, 33], 8, 2, 64, 16, width=60)]
    n = S.sifar_paged_attention_workspace(4, 8, 2, 64, 960)
    ws = torch.zeros(n, dtype=torch.uint8, device=DEV)
    outs = [torch.zeros_like(i["q"]) for i in steps]
    graphs = []
    for i, out in zip(steps, outs):
        i["pages"].copy_(torch.arange(240, device=DEV).view(4, 60) % i["k_cache"].shape[0])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            S.sifar_paged_attention(**i, out=out, workspace=ws)
        graphs.append(g)
    for k in range(4):
        for i, out, g in zip(steps, outs, graphs):
            i["lengths"] += 37
            g.replay()
            eager, _ = run(i, lse=False)
            assert torch.equal(out, eager), k
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        for i, out in zip(steps, outs):
            assert torch.equal(out, run(i, lse=False)[0])
    check(steps[0], outs[0], None)
    torch.cuda.synchronize()
    out, _ = run(steps[1], stream=torch.cuda.Stream())
    assert torch.equal(out, outs[1])
