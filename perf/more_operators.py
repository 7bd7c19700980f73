"""The blocks of a decode step's layers, as a user's program calls them, beside their plain forms.

``append``   the new tokens' keys and values into a paged cache, rotated by their positions on the
             way, and the queries rotated beside them (``sifar_cache_append``)
``attend``   attention of one new token of each sequence over that cache
             (``sifar_paged_attention``)
``experts``  a mixture-of-experts layer for a few tokens, from the router's ids and weights
             (``sifar_experts``)

With ``own`` false ``run`` computes them with elementary torch operations in 32 bits; the angles
of the rotation in 64.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
BASE = 500000.0  # of the rotation's frequencies


# ---- cases -------------------------------------------------------------------------------------

def _append(name, tokens, sequences, q_heads, kv_heads, dim, page, dtype="bf16", rotary=0,
            interleaved=0, furthest=4096):
    """Tokens are spread evenly over the sequences and follow one another in each, the last of
    them up to position `furthest`."""
    c = dict(op="append", tokens=tokens, sequences=sequences, q_heads=q_heads, kv_heads=kv_heads,
             dim=dim, page=page, dtype=dtype, rotary=rotary or dim, interleaved=interleaved,
             furthest=furthest)
    return dict(c, name=name) if name else c


def _attend(name, tokens, length, q_heads, kv_heads, dim, page, dtype="bf16", ragged=0, window=0,
            softcap=0.0, sinks=0):
    c = dict(op="attend", tokens=tokens, length=length, q_heads=q_heads, kv_heads=kv_heads,
             dim=dim, page=page, dtype=dtype, ragged=ragged, window=window, softcap=softcap,
             sinks=sinks)
    return dict(c, name=name) if name else c


def _experts(name, tokens, experts, topk, hidden, inter, dtype="bf16", ranks=1,
             activation="silu"):
    """`experts` of experts * ranks are here, those of the rank in the middle."""
    c = dict(op="experts", tokens=tokens, experts=experts, topk=topk, hidden=hidden, inter=inter,
             dtype=dtype, ranks=ranks, activation=activation)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one request's next token, latency only
        _append("append-t1-h32x8-d128", 1, 1, 32, 8, 128, 16),
        # an odd decode batch in half precision, pairs of neighbours, part of a head rotated,
        # positions up to a million
        _append("append-t77-h12x4-d96-far", 77, 77, 12, 4, 96, 24, "fp16", 32, 1, 1048576),
        # a prefill of four prompts
        _append("append-t8192-h32x8-d128", 8192, 4, 32, 8, 128, 64),
        # the first tokens of a request: latency only
        _attend("attend-t1-l33-h32x8-d128", 1, 33, 32, 8, 128, 16),
        # one request with a long context
        _attend("attend-t1-l131072-h32x8-d128", 1, 131072, 32, 8, 128, 64),
        # a serving batch of ragged contexts
        _attend("attend-t64-l8192-h64x8-d128", 64, 8192, 64, 8, 128, 16, ragged=1),
        # heads without groups in 32 bits
        _attend("attend-t16-l2000-h16x16-d64-fp32", 16, 2000, 16, 16, 64, 32, "fp32"),
        # odd heads, pages and lengths; window, bounded scores and a sink per head
        _attend("attend-t5-l777-h12x4-d80-fp16", 5, 777, 12, 4, 80, 24, "fp16", 1, 512, 30.0, 1),
        # one token through 8 of 128 small experts, latency
        _experts("experts-t1-e128-k8-h2048", 1, 128, 8, 2048, 768),
        # a batch that reaches most of 64 experts, a token or two for each
        _experts("experts-t16-e64-k6-h4096", 16, 64, 6, 4096, 1408),
        # a larger batch over a few large experts
        _experts("experts-t64-e8-k2-h4096", 64, 8, 2, 4096, 8192),
        # one of three ranks' experts, odd sizes, half precision
        _experts("experts-t7-e20-k4-h1000-fp16", 7, 20, 4, 1000, 520, "fp16", 3, "gelu"),
    ]


def _spread(rng, lo, hi):
    """A whole number of lo..hi, even over its logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def _heads(rng):
    kv = rng.choice([1, 2, 4, 8, 16])
    return kv * rng.choice([g for g in (1, 2, 3, 4, 5, 6, 7, 8, 12, 16) if g * kv <= 64]), kv


def draw(rng):
    op = rng.choice(["append", "attend", "experts"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    page = rng.choice([1, 8, 16, 16, 24, 32, 64, 128])
    dim = rng.choice([64, 80, 96, 128, 128, 128, 192, 256])
    q_heads, kv_heads = _heads(rng)
    if op == "append":
        while True:
            tokens = _spread(rng, 1, 8192)
            sequences = rng.choice([1, tokens, _spread(rng, 1, tokens)])
            each = -(-tokens // sequences)
            furthest = _spread(rng, max(each, 512), 1048576)
            if (tokens * (q_heads + 2 * kv_heads) * dim * SIZE[dtype] <= 8192 * 48 * 128 * 2
                    and sequences * furthest // page <= 1 << 23
                    and (each + 2 * page) * sequences * kv_heads * dim <= 1 << 27):
                break
        rotary = rng.choice([dim, dim, dim // 2, 32])
        return _append(None, tokens, sequences, q_heads, kv_heads, dim, page, dtype, rotary,
                       rng.randint(0, 1), furthest)
    if op == "attend":
        while True:
            tokens, length = _spread(rng, 1, 256), _spread(rng, 1, 131072)
            if tokens * length * kv_heads * dim * 2 * SIZE[dtype] <= 1 << 29:
                break
        return _attend(None, tokens, length, q_heads, kv_heads, dim, page, dtype,
                       rng.randint(0, 1), rng.choice([0, 0, 0, _spread(rng, 16, 4096)]),
                       rng.choice([0.0, 0.0, 30.0]), rng.choice([0, 0, 1]))
    while True:
        tokens, experts, ranks = _spread(rng, 1, 64), _spread(rng, 4, 256), rng.choice([1, 1, 2, 4])
        hidden, inter = 8 * _spread(rng, 64, 512), 8 * _spread(rng, 32, 1024)
        topk = rng.randint(1, min(8, experts))
        if experts * 3 * hidden * inter * SIZE[dtype] <= 1 << 30:
            break
    return _experts(None, tokens, experts, topk, hidden, inter, dtype, ranks,
                    rng.choice(["silu", "silu", "gelu"]))


# ---- inputs ------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _pages(g, counts, width):
    """A table [sequences][width] of pages that lie anywhere in their pool, -1 behind each
    sequence's own, and the pool's size: a quarter more than is taken, and a few."""
    total = int(sum(counts))
    pool = total + total // 4 + 4
    order = torch.randperm(pool, generator=g, device=DEV).int()
    n = torch.tensor(counts, device=DEV)
    at = torch.arange(width, device=DEV)
    first = torch.cumsum(n, 0) - n
    return torch.where(at < n[:, None], order[(first[:, None] + at).clamp(max=pool - 1)], -1), pool


def _append_inputs(case, seed):
    """Projections N(0,1) in one buffer of a row's q, k and v, with one channel in 64 of the keys
    ten times as large; positions that end between half of `furthest` and it; the cache holds what
    was there before."""
    g, dt = _gen(seed), DT[case["dtype"]]
    T, Hq, Hk, D, S = (case[k] for k in ("tokens", "q_heads", "kv_heads", "dim", "sequences"))
    x = torch.randn((T, Hq + 2 * Hk, D), generator=g, device=DEV)
    x[:, Hq:Hq + Hk, ::64] *= 10.0
    x = x.to(dt)
    each = -(-T // S)
    t = torch.arange(T, device=DEV)
    sequence, nth = t // each, t % each
    last = torch.rand((S,), generator=g, device=DEV) * 0.5 + 0.5
    start = (last * (case["furthest"] - each)).long()
    position = start[sequence] + nth
    # pages that the new tokens lie in are the only ones of the pool that a table names here
    page, width = case["page"], -(-case["furthest"] // case["page"])
    per = -(-each // page) + 1
    pool = S * per + 4
    order = torch.randperm(pool, generator=g, device=DEV).int()
    pages = torch.full((S, width), -1, dtype=torch.int32, device=DEV)
    at = (start // page)[:, None] + torch.arange(per, device=DEV)
    pages.scatter_(1, at.clamp(max=width - 1), order[:S * per].view(S, per))
    pages[:, -1] = order[torch.arange(1, S + 1, device=DEV) * per - 1]
    cache = torch.randn((2, pool, page, Hk, D), generator=g, device=DEV).to(dt)
    R = case["rotary"]
    inv_freq = (BASE ** (-torch.arange(0, R, 2, device=DEV).double() / R)).float()
    return dict(q=x[:, :Hq], k=x[:, Hq:Hq + Hk], v=x[:, Hq + Hk:], positions=position.int(),
                sequence=sequence.int(), pages=pages, k_cache=cache[0], v_cache=cache[1],
                inv_freq=inv_freq)


def _attend_inputs(case, seed):
    """Queries and keys whose scores spread by a few units, so that some positions carry most of
    the weight, as in a model; the pool holds other sequences' values behind a sequence's last."""
    g, dt = _gen(seed), DT[case["dtype"]]
    T, L, Hq, Hk, D = (case[k] for k in ("tokens", "length", "q_heads", "kv_heads", "dim"))
    lengths = torch.full((T,), L, dtype=torch.int64, device=DEV)
    if case["ragged"]:
        lengths = 1 + (torch.rand((T,), generator=g, device=DEV) * L).long().clamp(max=L - 1)
        lengths[T // 2] = L
    page = case["page"]
    pages, pool = _pages(g, [-(-n // page) for n in lengths.tolist()], -(-L // page))
    q = (2.0 * torch.randn((T, Hq, D), generator=g, device=DEV)).to(dt)
    k = torch.randn((pool, page, Hk, D), generator=g, device=DEV).to(dt)
    v = torch.randn((pool, page, Hk, D), generator=g, device=DEV).to(dt)
    sinks = torch.randn((Hq,), generator=g, device=DEV) if case["sinks"] else None
    return dict(q=q, k_cache=k, v_cache=v, pages=pages, lengths=lengths.int(), sinks=sinks)


def _experts_inputs(case, seed):
    """Normed activations N(0,1), weights that keep their scale, a router that likes some experts
    more, its softmax over the chosen as weights."""
    g, dt = _gen(seed), DT[case["dtype"]]
    T, E, k, H, I = (case[n] for n in ("tokens", "experts", "topk", "hidden", "inter"))
    x = torch.randn((T, H), generator=g, device=DEV).to(dt)
    w_in = torch.empty((E, 2 * I, H), dtype=dt, device=DEV).normal_(0.0, H ** -0.5, generator=g)
    w_out = torch.empty((E, H, I), dtype=dt, device=DEV).normal_(0.0, I ** -0.5, generator=g)
    logits = torch.randn((T, E * case["ranks"]), generator=g, device=DEV)
    logits = logits + 0.5 * torch.randn((E * case["ranks"],), generator=g, device=DEV)
    best, ids = torch.sort(logits, dim=-1, descending=True)
    e = torch.exp(best[:, :k] - best[:, :1])
    return dict(x=x, w_in=w_in, w_out=w_out, ids=ids[:, :k].int().contiguous(),
                weights=e / e.sum(-1, keepdim=True), first=case["ranks"] // 2 * E)


_INPUTS = {"append": _append_inputs, "attend": _attend_inputs, "experts": _experts_inputs}


def prepare(case, seed):
    s = dict(_INPUTS[case["op"]](case, seed), case=case)
    T, dt = case["tokens"], DT[case["dtype"]]
    if case["op"] == "append":
        s["q_out"] = torch.empty((T, case["q_heads"], case["dim"]), dtype=dt, device=DEV)
    elif case["op"] == "attend":
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((T, case["q_heads"]), dtype=torch.float32, device=DEV)
    else:
        s["out"] = torch.empty_like(s["x"])
    if own and case["op"] != "append":
        import paper_2607_08973_amd as S
        if case["op"] == "attend":
            n = S.sifar_paged_attention_workspace(T, case["q_heads"], case["kv_heads"],
                                                  case["dim"], case["length"])
        else:
            n = S.sifar_experts_workspace(T, case["topk"], case["inter"])
        s["workspace"] = torch.empty(n, dtype=torch.uint8, device=DEV)
    return s


# ---- one pass ----------------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if own:
        return {"append": _own_append, "attend": _own_attend, "experts": _own_experts}[op](s)
    return {"append": _plain_append, "attend": _plain_attend, "experts": _plain_experts}[op](s)


def _own_append(s):
    import paper_2607_08973_amd as S
    S.sifar_cache_append(s["k"], s["v"], s["positions"], s["pages"], s["k_cache"], s["v_cache"],
                         q=s["q"], q_out=s["q_out"], inv_freq=s["inv_freq"],
                         interleaved=s["case"]["interleaved"], sequence=s["sequence"])
    return s["q_out"], s["k_cache"], s["v_cache"]


def _own_attend(s):
    import paper_2607_08973_amd as S
    c = s["case"]
    S.sifar_paged_attention(s["q"], s["k_cache"], s["v_cache"], s["pages"], s["lengths"], s["out"],
                            s["workspace"], max_length=c["length"], window=c["window"],
                            softcap=c["softcap"], sinks=s["sinks"], lse=s["lse"])
    return s["out"], s["lse"]


def _own_experts(s):
    import paper_2607_08973_amd as S
    S.sifar_experts(s["x"], s["ids"], s["weights"], s["w_in"], s["w_out"], s["out"],
                    s["workspace"], activation=s["case"]["activation"], first_expert=s["first"])
    return s["out"]


def _rotated(x, cos, sin, interleaved):
    """x [tokens][heads][dim] in 32 bits, its first 2 * cos.shape[-1] elements rotated."""
    n = cos.shape[-1]
    head, rest = x[..., :2 * n], x[..., 2 * n:]
    cos, sin = cos[:, None], sin[:, None]
    if interleaved:
        a, b = head[..., 0::2], head[..., 1::2]
        head = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = head[..., :n], head[..., n:]
        head = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([head, rest], -1)


def _plain_append(s):
    angle = s["positions"].double()[:, None] * s["inv_freq"].double()
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    turn = s["case"]["interleaved"]
    s["q_out"].copy_(_rotated(s["q"].float(), cos, sin, turn))
    page = s["case"]["page"]
    at = s["positions"].long()
    row = s["pages"][s["sequence"].long(), at // page].long()
    s["k_cache"][row, at % page] = _rotated(s["k"].float(), cos, sin, turn).to(s["k"].dtype)
    s["v_cache"][row, at % page] = s["v"]
    return s["q_out"], s["k_cache"], s["v_cache"]


def _plain_attend(s):
    c = s["case"]
    T, Hq, D = s["q"].shape
    Hk, L = c["kv_heads"], c["length"]
    rows = s["pages"].clamp(min=0).long()
    k = s["k_cache"][rows].flatten(1, 2)[:, :L].permute(0, 2, 1, 3).float()  # [T][Hk][L][D]
    v = s["v_cache"][rows].flatten(1, 2)[:, :L].permute(0, 2, 1, 3).float()
    q = s["q"].view(T, Hk, Hq // Hk, D).float()
    x = torch.matmul(q, k.transpose(-1, -2)) * D ** -0.5  # [T][Hk][group][L]
    if c["softcap"]:
        x = c["softcap"] * torch.tanh(x / c["softcap"])
    at, n = torch.arange(L, device=x.device), s["lengths"][:, None]
    there = at < n
    if c["window"]:
        there = there & (at >= n - c["window"])
    x = torch.where(there[:, None, None], x, -math.inf)
    m = x.amax(-1, keepdim=True)
    sink = None if s["sinks"] is None else s["sinks"].view(1, Hk, Hq // Hk, 1)
    if sink is not None:
        m = torch.maximum(m, sink)
    w = torch.exp(x - m)
    total = w.sum(-1, keepdim=True)
    if sink is not None:
        total = total + torch.exp(sink - m)
    out = torch.matmul(w, v) / total
    return (out.reshape(T, Hq, D).to(s["q"].dtype),
            (m + torch.log(total)).reshape(T, Hq))


def _act(x, activation):
    if activation == "silu":
        return x / (1.0 + torch.exp(-x))
    return 0.5 * x * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x * x * x)))


def _plain_experts(s):
    """Where the slots are fewer than the experts, each slot's own weights; otherwise all experts
    on all tokens, weighted by what the router gave."""
    c, x = s["case"], s["x"].float()
    (T, H), k, E, I = x.shape, c["topk"], c["experts"], c["inter"]
    at = s["ids"].long() - s["first"]
    here = (at >= 0) & (at < E)
    w, at = torch.where(here, s["weights"], 0.0), torch.where(here, at, 0)
    if T * k < E:
        e = at.reshape(-1)
        xs = x.repeat_interleave(k, 0)[:, :, None]
        y = torch.matmul(s["w_in"][e].float(), xs)[..., 0]  # [T * k][2 I]
        h = _act(y[:, :I], c["activation"]) * y[:, I:]
        y = torch.matmul(s["w_out"][e].float(), h[:, :, None])[..., 0]
        return (y.view(T, k, H) * w[..., None]).sum(1).to(s["x"].dtype)
    y = torch.matmul(s["w_in"].float(), x.t())  # [E][2 I][T]
    h = _act(y[:, :I], c["activation"]) * y[:, I:]
    y = torch.matmul(s["w_out"].float(), h)  # [E][H][T]
    share = torch.zeros((T, E), device=x.device).scatter_add_(1, at, w)
    return (y * share.t()[:, None]).sum(0).t().to(s["x"].dtype).contiguous()


# ---- work and the definition in 64 bits --------------------------------------------------------

def work(case):
    """Every input read once, every output written once. Of the experts' weights those that a
    token reaches, as many as an even router would; of a cache the positions that are there."""
    T, e = case["tokens"], SIZE[case["dtype"]]
    if case["op"] == "append":
        row = (case["q_heads"] + 2 * case["kv_heads"]) * case["dim"]
        return {"bytes": 2 * T * row * e + 12 * T + 2 * case["rotary"],
                "flops": 3 * T * (case["q_heads"] + case["kv_heads"]) * case["rotary"]}
    if case["op"] == "attend":
        L = case["length"]
        if case["ragged"]:
            L = (L + 1) / 2
        L = min(L, case["window"]) if case["window"] else L
        H, D = case["q_heads"], case["dim"]
        return {"bytes": int(2 * T * (L * case["kv_heads"] + H) * D * e + 4 * T * (L / case["page"] + H)),
                "flops": int(4 * T * L * H * D)}
    E, k, H, I = case["experts"], case["topk"], case["hidden"], case["inter"]
    reached = E * (1.0 - (1.0 - k / (E * case["ranks"])) ** T)
    return {"bytes": int(reached * 3 * I * H * e + 2 * T * H * e + 8 * T * k),
            "flops": int(6 * T * k / case["ranks"] * I * H)}


def exact(case, seed):
    s = _INPUTS[case["op"]](case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "experts": _exact_experts}[
        case["op"]](case, s)


def _exact_append(case, s):
    """As complex numbers: a pair times e^(i angle)."""
    n, page = case["rotary"] // 2, case["page"]
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV),
                       torch.outer(s["positions"].double(), s["inv_freq"].double()))[:, None]

    def rotate(x):
        y = x.double().clone()
        a, b = ((slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if case["interleaved"] else
                (slice(0, n), slice(n, 2 * n)))
        z = torch.complex(y[..., a].contiguous(), y[..., b].contiguous()) * turn
        y[..., a], y[..., b] = z.real, z.imag
        return y

    kc, vc = s["k_cache"].double(), s["v_cache"].double()
    slot = s["pages"].long()[s["sequence"].long(), s["positions"].long() // page] * page \
        + s["positions"].long() % page
    kc.flatten(0, 1).index_copy_(0, slot, rotate(s["k"]))
    vc.flatten(0, 1).index_copy_(0, slot, s["v"].double())
    return rotate(s["q"]), kc, vc


def _exact_attend(case, s):
    """Sequence by sequence and head by head of the cache."""
    T, H, D = s["q"].shape
    G, page = H // case["kv_heads"], case["page"]
    out = torch.empty((T, H, D), dtype=torch.float64, device=DEV)
    lse = torch.empty((T, H), dtype=torch.float64, device=DEV)
    lengths = s["lengths"].tolist()
    for t, n in enumerate(lengths):
        lo = max(0, n - case["window"]) if case["window"] else 0
        p = torch.arange(lo, n, device=DEV)
        rows = s["pages"][t].long()[p // page]
        for g in range(case["kv_heads"]):
            k, v = (s[c][rows, p % page, g].double() for c in ("k_cache", "v_cache"))
            x = s["q"][t, g * G:(g + 1) * G].double() @ k.t() / math.sqrt(D)
            if case["softcap"]:
                x = torch.tanh(x / case["softcap"]) * case["softcap"]
            if s["sinks"] is not None:
                x = torch.cat([x, s["sinks"][g * G:(g + 1) * G, None].double()], 1)
            total = torch.logsumexp(x, 1)
            out[t, g * G:(g + 1) * G] = torch.exp(x - total[:, None])[:, :n - lo] @ v
            lse[t, g * G:(g + 1) * G] = total
    return out, lse


def _exact_experts(case, s):
    """Expert by expert, its own tokens only."""
    out = torch.zeros((case["tokens"], case["hidden"]), dtype=torch.float64, device=DEV)
    I, ids = case["inter"], s["ids"] - s["first"]
    for e in range(case["experts"]):
        t, slot = torch.nonzero(ids == e, as_tuple=True)
        if t.numel() == 0:
            continue
        y = s["x"][t].double() @ s["w_in"][e].double().t()
        a, b = y[:, :I], y[:, I:]
        z = a if case["activation"] == "silu" else math.sqrt(8.0 / math.pi) * (
            a + 0.044715 * a ** 3)
        h = a * torch.sigmoid(z) * b
        out.index_add_(0, t, s["weights"][t, slot].double()[:, None] *
                       (h @ s["w_out"][e].double().t()))
    return out
