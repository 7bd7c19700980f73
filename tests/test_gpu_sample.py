"""GPU: sifar_sample against its definition in 64 bits.

Tokens have to be equal. A probability is a 64-bit weight over a sum that is off by
at most one unit of 2^-42 of the largest weight (which it holds) a token, rounded
once to fp32: 2^-24 + vocab * 2^-42 of its value."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

import paper_2607_08973_amd as S

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
INF, NAN = math.inf, math.nan


@pytest.fixture(autouse=True, scope="module")
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    S.load()
    yield
    torch.cuda.synchronize()


def one(x, u, tau, k, p, m):
    """(token, prob) of one row of 64-bit logits."""
    live = np.flatnonzero(x > -INF)
    if not live.size:
        return -1, 0.0
    live = live[np.argsort(-x[live], kind="stable")]
    if not tau > 0:
        return live[0], 1.0
    x = x[live]
    z = np.zeros(x.size)
    with np.errstate(over="ignore", invalid="ignore"):
        z[x < x[0]] = (x[x < x[0]] - x[0]) / tau
    live, z = live[z >= -60 * math.log(2)], z[z >= -60 * math.log(2)]
    w = np.exp(z)
    n = live.size
    if k > 0:
        n = min(n, int(k))
    if p < 1:
        mass = np.cumsum(w[:n])
        n = min(n, 1 + int(np.searchsorted(mass, p * mass[-1], "left")))
    if m > 0:
        n = min(n, int((z >= math.log(min(m, 1.0))).sum()))   # w >= m, where w rounds to 1 too
    order = np.argsort(live[:n])
    live, w = live[:n][order], w[:n][order]
    mass = np.cumsum(w)
    u = u if u > 0 else 0.0
    i = min(int(np.searchsorted(mass, u * mass[-1], "right")), n - 1)
    return live[i], w[i] / mass[-1]


def run(x, uniform, **kw):
    T, V = x.shape
    f = lambda v, dt=torch.float32: None if v is None else torch.as_tensor(v, dtype=dt).expand(
        T).contiguous().to(DEV)
    out = torch.full((T,), -9, dtype=torch.int32, device=DEV)
    probs = torch.full((T,), -9.0, device=DEV)
    ws = torch.empty(S.sifar_sample_workspace(T, V), dtype=torch.uint8, device=DEV)
    ws.fill_(0xA5)
    S.sifar_sample(x, f(uniform), out, ws, probs, f(kw.get("temperature")),
                   f(kw.get("top_k"), torch.int32), f(kw.get("top_p")), f(kw.get("min_p")))
    return out, probs


def check(x, uniform, **kw):
    out, probs = run(x, uniform, **kw)
    T, V = x.shape
    xs = x.double().cpu().numpy()
    get = lambda k, d: np.broadcast_to(
        np.asarray(torch.as_tensor(kw.get(k, d), dtype=torch.float32), np.float64), (T,))
    u = np.broadcast_to(np.asarray(torch.as_tensor(uniform, dtype=torch.float32), np.float64), (T,))
    args = [u, get("temperature", 1.0), get("top_k", 0), get("top_p", 1.0), get("min_p", 0.0)]
    want = [one(xs[t], *(a[t] for a in args)) for t in range(T)]
    token = np.array([w[0] for w in want])
    prob = np.array([w[1] for w in want])
    got, gp = out.cpu().numpy(), probs.double().cpu().numpy()
    assert np.array_equal(got, token), [(t, got[t], token[t]) for t in
                                        np.flatnonzero(got != token)[:4]]
    assert (np.abs(gp - prob) <= prob * (2.0 ** -24 + V * 2.0 ** -42) + 2.0 ** -150).all()


def rng(*seed):
    return np.random.default_rng([2607, *seed])


def logits(seed, T, V, dtype="fp32", shape="flat"):
    r = rng(seed, T, V)
    x = r.standard_normal((T, V)) * (1.5 if shape == "flat" else 2.5)
    if shape == "peaked":
        x += (r.random((T, V)) < 40 / V) * (6 + 4 * r.random((T, V)))
    return torch.from_numpy(x).to(DT[dtype]).to(DEV)


VOCABS = [1, 2, 63, 1000, 1023, 1024, 1025, 5000, 50257, 131075]


@pytest.mark.parametrize("V", VOCABS)
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("shape", ["flat", "peaked"])
def test_filters(V, dtype, shape):
    """Every filter alone and together, each row its own values."""
    T = 6 if V > 5000 else 24
    x, r = logits(1, T, V, dtype, shape), rng(1, T, V)
    u, tau = r.random(T), 0.5 + r.random(T)
    tau[1::5] = 0.0
    k, p, m = r.integers(1, 100, T), 0.5 + 0.499 * r.random(T), 0.2 * r.random(T)
    check(x, u)
    check(x, u, temperature=tau)
    check(x, u, temperature=tau, top_k=k)
    check(x, u, temperature=tau, top_p=p)
    check(x, u, temperature=tau, min_p=m)
    check(x, u, temperature=tau, top_k=k, top_p=p, min_p=m)
    check(x, u, temperature=tau, top_k=k * 60, top_p=p)


@pytest.mark.parametrize("V", [5, 1500])
def test_every_part_of_the_unit_interval(V):
    """One row drawn with 512 numbers over the whole interval: each token as often as
    it should be, at every filter."""
    x = logits(2, 1, V).expand(512, V)
    u = (np.arange(512) + 0.37) / 512
    for kw in (dict(), dict(top_k=3), dict(top_p=0.8), dict(min_p=0.1),
               dict(top_k=V, top_p=0.6, min_p=0.01)):
        check(x.contiguous(), u, **kw)


@pytest.mark.parametrize("V,levels", [(4000, 1), (4000, 2), (130000, 1), (130000, 3)])
def test_ties(V, levels):
    """Rows of few values: thresholds fall between equal logits, and the lower
    indices stay; more candidates than any list holds."""
    r = rng(3, V, levels)
    T = 12
    x = torch.from_numpy(r.integers(0, levels, (T, V)).astype(np.float32)).to(DEV)
    x[1, ::2] *= -1.0                                  # -0 and 0 are equal
    u = r.random(T)
    check(x, u)
    check(x, u, top_k=r.integers(1, V, T))
    check(x, u, top_p=r.random(T))
    check(x, u, top_k=r.integers(1, V, T), top_p=0.1 + 0.8 * r.random(T))
    check(x, u, min_p=0.5)
    check(x, u, temperature=0.0)


def test_exact_borders():
    """Equal weights, where running sums meet targets exactly."""
    x = torch.zeros(6, 4, device=DEV)
    u = [0.0, 0.25, 0.5, 0.75, 1.0 - 2.0 ** -24, 0.25 - 2.0 ** -26]
    out, probs = run(x, u)
    assert out.tolist() == [0, 1, 2, 3, 3, 0] and (probs == 0.25).all()
    out, probs = run(x, u, top_p=0.5)
    assert out.tolist() == [0, 0, 1, 1, 1, 0] and (probs == 0.5).all()
    out, probs = run(x, u, top_p=0.5000001)
    assert out.tolist() == [0, 0, 1, 2, 2, 0]
    check(x, u, top_k=3, top_p=2.0 / 3)


def test_nothing_is_there():
    for V in (3, 3000):
        x = logits(4, 6, V)
        x[0] = -INF
        x[1] = NAN
        x[2, 1:] = -INF
        x[3, ::2] = NAN
        x[4, : V // 2] = -INF
        for kw in (dict(), dict(temperature=0.0), dict(top_k=2), dict(top_p=0.9), dict(min_p=0.1),
                   dict(top_k=5, top_p=0.5, min_p=0.2)):
            check(x, rng(4, V).random(6), **kw)


@pytest.mark.parametrize("dtype,bits", [("fp32", 0x7F800001), ("fp32", 0xFFA00000 - (1 << 32)),
                                        ("bf16", 0x7F81), ("bf16", 0xFF81 - (1 << 16)),
                                        ("fp16", 0x7C01), ("fp16", 0xFD00 - (1 << 16))])
@pytest.mark.parametrize("V", [900, 70000])
def test_signalling_nans_are_not_there(dtype, bits, V):
    x = logits(45, 3, V, dtype)
    raw = x.view(torch.int32 if dtype == "fp32" else torch.int16)
    raw[:, 5::7] = bits
    raw[1, : V // 2] = bits
    for kw in (dict(), dict(temperature=0.0), dict(top_k=9), dict(top_p=0.95),
               dict(top_k=V, top_p=0.9), dict(min_p=0.05), dict(temperature=INF)):
        check(x, [0.1, 0.6, 0.95], **kw)


def test_infinite_logits_share_the_weight():
    x = logits(5, 4, 2500)
    x[0, 7] = INF
    x[1, [3, 1100, 2400]] = INF
    x[2, :] = -INF
    x[2, 2000] = INF
    for kw in (dict(), dict(temperature=0.0), dict(top_k=2), dict(top_p=0.5), dict(min_p=0.3),
               dict(temperature=INF), dict(temperature=INF, top_p=0.3, min_p=1.0)):
        check(x, [0.7, 0.5, 0.1, 0.9], **kw)


@pytest.mark.parametrize("dtype", list(DT))
def test_masks_of_the_lowest_value(dtype):
    low = torch.finfo(DT[dtype]).min
    x = logits(6, 6, 3000, dtype)
    x[0, 1:] = low
    x[1] = low
    x[2, :2990] = low
    x[3, ::2] = low
    x[4, :2999] = low
    u = [0.0, 0.5, 0.0, 0.3, 0.99, 0.0]
    for kw in (dict(), dict(temperature=0.0), dict(temperature=0.7, top_k=50),
               dict(temperature=1.5, top_p=0.95), dict(min_p=0.01)):
        check(x, u, **kw)


@pytest.mark.parametrize("tau", [1e-45, 1e-30, 1e-3, 30.0, 1e30, INF, -1.0, NAN, 0.0])
def test_temperatures(tau):
    x, r = logits(7, 8, 4100), rng(7)
    for kw in (dict(), dict(top_k=7), dict(top_p=0.6), dict(min_p=0.3), dict(min_p=1.0),
               dict(top_k=2000, top_p=0.9, min_p=1e-6)):
        check(x, r.random(8), temperature=tau, **kw)


def test_values_at_and_past_the_ends_of_their_ranges():
    x, u = logits(8, 8, 2100), rng(8).random(8)
    for k in (-5, 0, 1, 2, 2100, 2 ** 31 - 1):
        check(x, u, top_k=k)
    for p in (-1.0, 0.0, 1e-30, 1.0 - 2.0 ** -24, 1.0, 2.0, NAN):
        check(x, u, top_p=p)
    for m in (-1.0, 0.0, 1e-38, 0.999, 1.0, 3.0, NAN):
        check(x, u, min_p=m)
    for v in (0.0, 2.0 ** -149, 1.0 - 2.0 ** -24, 1.0, 7.0, -1.0, NAN):
        check(x, v)
        check(x, v, top_k=40, top_p=0.9)


def test_far_behind_the_likeliest():
    """Weights near and below the cut at 2^-60: kept at 2^-59.9, gone at 2^-60.1."""
    x = torch.full((2, 3000), -INF, device=DEV)
    x[:, 2000] = 0.0
    x[0, 10] = -59.9 * math.log(2)
    x[1, 10] = -60.1 * math.log(2)
    out, _ = run(x, 0.0)
    assert out.tolist() == [10, 2000]


def test_rows_of_a_wider_buffer_and_odd_addresses():
    for dtype in DT:
        x = logits(9, 5, 3001, dtype)
        wide = torch.full((6, 3011), 99.0, dtype=DT[dtype], device=DEV)
        wide[:5, 5:3006] = x
        u = rng(9).random(5)
        for kw in (dict(), dict(top_k=9), dict(top_p=0.9)):
            a, b = run(wide[:5, 5:3006], u, **kw), run(x, u, **kw)
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_outputs_behind_the_last_row_stay_and_probs_are_optional():
    x, u = logits(10, 3, 2000), torch.tensor([0.1, 0.5, 0.9], device=DEV)
    out = torch.full((7,), -9, dtype=torch.int32, device=DEV)
    need = S.sifar_sample_workspace(3, 2000)
    ws = torch.full((need + 64,), 7, dtype=torch.uint8, device=DEV)
    S.sifar_sample(x, u, out[2:5], ws[:need])
    assert torch.equal(out[2:5], run(x, [0.1, 0.5, 0.9])[0])
    assert (out[:2] == -9).all() and (out[5:] == -9).all() and (ws[need:] == 7).all()


def test_no_rows():
    run(torch.empty(0, 100, device=DEV), 0.5)


def test_a_row_does_not_depend_on_its_batch():
    x, r = logits(11, 300, 3000, "bf16"), rng(11)
    u, p = r.random(300), 0.9 * r.random(300)
    out, probs = run(x, u, top_p=p)
    for t in (0, 150, 299):
        a, b = run(x[t:t + 1], u[t:t + 1], top_p=p[t:t + 1])
        assert a[0] == out[t] and b[0] == probs[t]
    again = run(x, u, top_p=p)
    assert torch.equal(again[0], out) and torch.equal(again[1], probs)


def test_far_rows():
    stride = (1 << 30) + 5
    buf = torch.empty(2 * stride + 2000, dtype=torch.bfloat16, device=DEV)
    rows = torch.as_strided(buf, (3, 2000), (stride, 1))
    rows.copy_(logits(12, 3, 2000, "bf16"))
    check(rows, [0.2, 0.5, 0.8], top_p=0.9)


def test_largest_vocabulary():
    V = S.SIFAR_SAMPLE_MAX_VOCAB
    x = logits(13, 2, V)
    for kw in (dict(), dict(top_k=2000), dict(top_p=0.7), dict(top_k=50, top_p=0.9, min_p=0.05)):
        check(x, [0.3, 0.999], **kw)


@pytest.mark.parametrize("T,V", [(1, 65536), (3, 70001), (65, 66000), (2, 262144)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_nucleus_of_large_rows(T, V, dtype):
    """Few rows of many logits, whose passes are spread over workgroups: flat and peaked
    rows side by side, greedy and masked ones among them; with min-p, which cuts a
    nucleus short, and where a top-k for some rows keeps the passes in one workgroup."""
    x = logits(30, T, V, dtype)
    x[T // 2] = logits(31, 1, V, dtype, "peaked")[0]
    x[T - 1, : V // 3] = -INF
    r = rng(30, T, V)
    tau = 0.7 + 0.6 * r.random(T)
    tau[2::7] = 0.0
    if T > 4:
        x[4] = -INF
    u, p = r.random(T), 0.3 + 0.699 * r.random(T)
    check(x, u, temperature=tau, top_p=p)
    check(x, u, temperature=tau, top_p=p, min_p=0.02)
    check(x, u, temperature=tau, top_p=p, top_k=0)


def test_nucleus_of_rows_with_few_values():
    """A window that no list holds: many equal logits at the border."""
    x = torch.from_numpy(rng(32).integers(0, 3, (4, 70000)).astype(np.float32)).to(DEV)
    x[1] = 5.0
    check(x, [0.1, 0.5, 0.9, 0.99], top_p=[0.3, 0.5, 0.9, 0.999])


def test_spread_rows_replay():
    T, V = 3, 70000
    r = rng(33)
    x, u = logits(33, T, V), torch.from_numpy(r.random(T)).float().to(DEV)
    p = torch.full((T,), 0.9, device=DEV)
    ws = [torch.full((S.sifar_sample_workspace(256, V),), 0x5A, dtype=torch.uint8, device=DEV)
          for _ in range(2)]
    out = [torch.empty(T, dtype=torch.int32, device=DEV) for _ in range(2)]
    S.sifar_sample(x, u, out[0], ws[0], top_p=p)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        S.sifar_sample(x, u, out[0], ws[0], top_p=p)
    for k in range(4):
        x.copy_(logits(34 + k, T, V, shape=("flat", "peaked")[k & 1]))
        u.copy_(torch.from_numpy(r.random(T)))
        g.replay()
        S.sifar_sample(x, u, out[1], ws[1], top_p=p)
        torch.cuda.synchronize()
        assert torch.equal(out[0], out[1])
        check(x, u.cpu(), top_p=0.9)


def test_streams_and_replays():
    x0, r = logits(14, 9, 5000), rng(14)
    u = torch.from_numpy(r.random(9)).float().to(DEV)
    p = torch.full((9,), 0.8, device=DEV)
    side = torch.cuda.Stream()
    x = torch.zeros_like(x0)
    ws = [torch.empty(S.sifar_sample_workspace(9, 5000), dtype=torch.uint8, device=DEV)
          for _ in range(2)]
    out = [torch.empty(9, dtype=torch.int32, device=DEV) for _ in range(2)]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        x.copy_(x0)
        S.sifar_sample(x, u, out[0], ws[0], top_p=p)
    side.synchronize()
    S.sifar_sample(x0, u, out[1], ws[1], top_p=p)
    assert torch.equal(out[0], out[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        S.sifar_sample(x, u, out[0], ws[0], top_p=p)
    for k in range(3):
        x.copy_(logits(20 + k, 9, 5000))
        u.copy_(torch.from_numpy(r.random(9)))
        g.replay()
        S.sifar_sample(x, u, out[1], ws[1], top_p=p)
        torch.cuda.synchronize()
        assert torch.equal(out[0], out[1])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_spread_rows_at_the_ends_of_their_ranges(dtype):
    """Rows whose passes may be spread: infinite logits, masks of both kinds, and
    temperatures at which the passes cannot be bounded."""
    V = 70000
    x, u = logits(40, 9, V, dtype), [0.7, 0.5, 0.1, 0.9, 0.3, 0.99, 0.0, 0.6, 0.4]
    x[0, 7] = INF
    x[1, [3, 1100, 69999]] = INF
    x[2] = -INF
    x[2, 66000] = INF
    x[3] = torch.finfo(DT[dtype]).min
    x[4, : V - 3] = torch.finfo(DT[dtype]).min
    x[5] = NAN
    x[6, ::2] = NAN
    x[7] = -3.0
    for p in (0.6, 0.9999, 0.0, [1.0, 0.5] * 4 + [0.7]):
        check(x, u, top_p=p)
        check(x, u, top_p=p, min_p=0.2)
        check(x, u, top_p=p, temperature=[1e-45, 1e-30, 1e-3, 30.0, 1e30, INF, -1.0, NAN, 200.0])
        check(x, u, top_p=p, temperature=[INF, 1e30, 1e-45, 2.0, 0.5, 1.0, 50.0, 1e-3, INF])


def test_most_rows():
    T = S.SIFAR_ROWS_MAX_TOKENS
    x = logits(41, T, 3)
    u = torch.from_numpy(rng(41).random(T).astype(np.float32))
    x64, at = x.double().cpu(), u.double()
    out, _ = run(x, u)
    mass = torch.softmax(x64, -1).cumsum(-1)
    assert torch.equal(out.cpu().long(), (mass[:, :2] <= at[:, None]).sum(-1))
    out, _ = run(x, u, top_k=2)
    least = 2 - x64.flip(-1).argmin(-1, keepdim=True)   # of equal ones, the last leaves
    mass = torch.softmax(x64.scatter(1, least, -INF), -1).cumsum(-1)
    want = (mass[:, :2] <= at[:, None]).sum(-1)
    want = torch.where((want == 2) & (least[:, 0] == 2), 1, want)
    assert torch.equal(out.cpu().long(), want)
    out, probs = run(x, u, temperature=0.0)
    assert torch.equal(out.cpu().long(), x64.argmax(-1)) and (probs == 1).all()
