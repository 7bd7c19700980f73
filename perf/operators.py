"""The row operators of a decode step, as a user's program calls them, beside their plain forms.

``block_norm``  what surrounds a block in layers that normalise before and after it: the block's
                output (one tensor, or up to eight ranks' partials to be summed), its own norm, a
                gate and a scale, the residual stream, and the next block's norm
                (``sifar_block_norm``)
``route``       a token's experts from its router logits: softmax or sigmoid scores, a bias for
                balance, groups, top-k, renormalised weights (``sifar_route``)
``sample``      a token from its logits and one given random number: temperature, top-k, top-p,
                min-p (``sifar_sample``)

With ``own`` false ``run`` computes them with elementary torch operations in 32 bits; in 64 where
an order or a running sum decides which index comes out.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
EPS = 1e-6
CUT = -60.0 * math.log(2.0)  # a token 2^-60 below the likeliest is never drawn


# ---- cases -------------------------------------------------------------------------------------

def _norm(name, tokens, hidden, dtype="bf16", residual="same", parts=1, post=1, gate="none",
          branch_scale=1.0, residual_scale=1.0, offset=0.0):
    c = dict(op="block_norm", tokens=tokens, hidden=hidden, dtype=dtype, residual=residual,
             parts=parts, post=post, gate=gate, branch_scale=branch_scale,
             residual_scale=residual_scale, offset=offset)
    return dict(c, name=name) if name else c


def _route(name, tokens, experts, topk, dtype="fp32", score="softmax", bias=0, groups=1,
           top_groups=1, group_top=1, renorm=1, scale=1.0):
    c = dict(op="route", tokens=tokens, experts=experts, topk=topk, dtype=dtype, score=score,
             bias=bias, groups=groups, top_groups=top_groups, group_top=group_top, renorm=renorm,
             scale=scale)
    return dict(c, name=name) if name else c


def _sample(name, tokens, vocab, dtype="fp32", filters="", shape="peaked", masked=0):
    c = dict(op="sample", tokens=tokens, vocab=vocab, dtype=dtype, filters=filters, shape=shape,
             masked=masked)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of a decode step: norm after the block and before the next one, latency only
        _norm("norm-t1-h4096-bf16", 1, 4096, offset=1.0),
        # a decode batch whose block output is still eight ranks' partials
        _norm("norm-t64-h8192-n8-bf16", 64, 8192, parts=8, gate="channel"),
        # a prefill with the residual stream in 32 bits
        _norm("norm-t4096-h5120-res32", 4096, 5120, residual="fp32", branch_scale=0.25),
        # a gate per token, ragged rows, in half precision
        _norm("norm-t77-h3896-fp16", 77, 3896, dtype="fp16", gate="token", residual_scale=0.5),
        # one token through 256 experts with balance bias and groups, latency only
        _route("route-t1-e256-bias", 1, 256, 8, score="sigmoid", bias=1, groups=8, top_groups=4,
               group_top=2, scale=2.5),
        # a prefill through 512 experts, logits straight from a 16-bit projection
        _route("route-t16384-e512-bf16", 16384, 512, 10, dtype="bf16"),
        # a prefill through bias and groups
        _route("route-t8192-e256-bias", 8192, 256, 8, score="sigmoid", bias=1, groups=8,
               top_groups=4, group_top=2, scale=2.5),
        # an odd batch, an odd number of experts, weights as they are
        _route("route-t333-e60", 333, 60, 4, renorm=0),
        # one request, no filter: latency only
        _sample("sample-t1-v32000", 1, 32000),
        # a small batch with every filter, each request its own values
        _sample("sample-t8-v128256-kpm", 8, 128256, filters="kpm"),
        # a large batch drawn by nucleus from flat rows: the nucleus holds thousands of tokens
        _sample("sample-t256-v151936-p-flat", 256, 151936, dtype="bf16", filters="p",
                shape="flat"),
        # an odd vocabulary, grammar masks, temperature and min-p
        _sample("sample-t33-v50257-m", 33, 50257, dtype="fp16", filters="m", masked=1),
    ]


def _spread(rng, lo, hi):
    """A whole number of lo..hi, even over its logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["block_norm", "route", "sample"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op == "block_norm":
        while True:
            tokens, hidden = _spread(rng, 1, 4096), 8 * _spread(rng, 16, 2048)
            parts = rng.choice([1, 1, 2, 4, 8])
            if tokens * hidden * (parts + 3) <= 4096 * 5120 * 4:
                break
        return _norm(None, tokens, hidden, dtype, rng.choice(["same", "same", "fp32", "none"]),
                     parts, rng.randint(0, 1), rng.choice(["none", "channel", "token"]),
                     rng.choice([1.0, 0.25]), rng.choice([1.0, 0.5]), rng.choice([0.0, 1.0]))
    if op == "route":
        score, bias = rng.choice(["softmax", "sigmoid"]), rng.randint(0, 1)
        if rng.random() < 0.5:
            groups = rng.choice([2, 4, 8])
            experts = groups * _spread(rng, 4, 64)
            top_groups = rng.randint(1, groups)
            topk = rng.randint(1, min(12, top_groups * experts // groups))
        else:
            groups = top_groups = 1
            experts = _spread(rng, 8, 512)
            topk = rng.randint(1, min(12, experts))
        return _route(None, _spread(rng, 1, 16384), experts, topk, dtype, score, bias, groups,
                      top_groups, rng.choice([1, 2]), rng.randint(0, 1), rng.choice([1.0, 2.5]))
    while True:
        tokens, vocab = _spread(rng, 1, 256), _spread(rng, 1000, 262144)
        if tokens * vocab <= 256 * 151936:
            break
    return _sample(None, tokens, vocab, dtype, rng.choice(["", "k", "p", "m", "kp", "kpm"]),
                   rng.choice(["peaked", "flat"]), rng.randint(0, 1))


# ---- inputs ------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _norm_inputs(case, seed):
    """Decode activations N(0,1) * 0.5 with 0.1 % outliers x 50 (in each partial), a residual
    stream N(0,1) and norm weights N(1, 0.02), all less the offset that the norm adds."""
    g, dt = _gen(seed), DT[case["dtype"]]
    T, H, P = case["tokens"], case["hidden"], case["parts"]
    x = torch.randn((P, T, H), generator=g, device=DEV) * 0.5
    x = torch.where(torch.rand((P, T, H), generator=g, device=DEV) < 0.001, x * 50.0, x).to(dt)
    weights = (1.0 - case["offset"] + 0.02 * torch.randn((2, H), generator=g, device=DEV)).to(dt)
    rdt = torch.float32 if case["residual"] == "fp32" else dt
    residual = torch.randn((T, H), generator=g, device=DEV).to(rdt)
    gate = torch.rand((1 if case["gate"] == "channel" else T, H), generator=g, device=DEV).to(dt)
    return dict(x=x, post=weights[0] if case["post"] else None, weight=weights[1],
                residual=None if case["residual"] == "none" else residual,
                gate=None if case["gate"] == "none" else gate, rdt=rdt)


def _route_inputs(case, seed):
    """Router logits N(0, 1.5) with a common part per expert, a balance bias of a tenth of a
    sigmoid score's range (a tenth of a uniform softmax score for softmax)."""
    g, E = _gen(seed), case["experts"]
    x = 1.5 * torch.randn((case["tokens"], E), generator=g, device=DEV)
    x = (x + 0.5 * torch.randn((E,), generator=g, device=DEV)).to(DT[case["dtype"]])
    bias = torch.randn((E,), generator=g, device=DEV)
    return x, bias * (0.1 if case["score"] == "sigmoid" else 0.1 / E) if case["bias"] else None


def _sample_inputs(case, seed):
    """Logits: a bulk N(0, 2.5) and, in peaked rows, some forty tokens lifted out of it as a
    language model's are; grammar masks put -inf on nine of ten tokens of every third row.
    Every request has filters of its own, one in eight is greedy."""
    g, T, V = _gen(seed), case["tokens"], case["vocab"]
    x = torch.randn((T, V), generator=g, device=DEV) * (2.5 if case["shape"] == "peaked" else 1.5)
    if case["shape"] == "peaked":
        x += (torch.rand((T, V), generator=g, device=DEV) < 40.0 / V) * (
            6.0 + 4.0 * torch.rand((T, V), generator=g, device=DEV))
    if case["masked"]:
        x[::3].masked_fill_(torch.rand((len(range(0, T, 3)), V), generator=g, device=DEV) < 0.9,
                            -math.inf)
    r = lambda lo, hi: lo + (hi - lo) * torch.rand((T,), generator=g, device=DEV)
    s = dict(logits=x.to(DT[case["dtype"]]), uniform=r(0.0, 1.0), temperature=r(0.6, 1.2),
             top_k=r(1.0, 100.0).int(), top_p=r(0.7, 0.99), min_p=r(0.02, 0.1))
    s["temperature"][5::8] = 0.0
    for key, letter in (("top_k", "k"), ("top_p", "p"), ("min_p", "m")):
        if letter not in case["filters"]:
            s[key] = None
    return s


def prepare(case, seed):
    T = case["tokens"]
    s = dict(case=case)
    if case["op"] == "block_norm":
        s.update(_norm_inputs(case, seed))
        s["residual_out"] = torch.empty((T, case["hidden"]), dtype=s["rdt"], device=DEV)
        s["y"] = torch.empty((T, case["hidden"]), dtype=s["x"].dtype, device=DEV)
    elif case["op"] == "route":
        s["logits"], s["bias"] = _route_inputs(case, seed)
        s["ids"] = torch.empty((T, case["topk"]), dtype=torch.int32, device=DEV)
        s["weights"] = torch.empty((T, case["topk"]), dtype=torch.float32, device=DEV)
    else:
        s.update(_sample_inputs(case, seed))
        s["tokens"] = torch.empty((T,), dtype=torch.int32, device=DEV)
        s["probs"] = torch.empty((T,), dtype=torch.float32, device=DEV)
        if own:
            import paper_2607_08973_amd as S
            s["workspace"] = torch.empty(S.sifar_sample_workspace(T, case["vocab"]),
                                         dtype=torch.uint8, device=DEV)
    return s


# ---- one pass ----------------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if own:
        return {"block_norm": _own_norm, "route": _own_route, "sample": _own_sample}[op](s)
    return {"block_norm": _plain_norm, "route": _plain_route, "sample": _plain_sample}[op](s)


def _own_norm(s):
    import paper_2607_08973_amd as S
    c = s["case"]
    S.sifar_block_norm(s["x"], s["residual"], s["residual_out"], post_weight=s["post"],
                       gate=s["gate"], norm_weight=s["weight"], y=s["y"],
                       branch_scale=c["branch_scale"], residual_scale=c["residual_scale"],
                       weight_offset=c["offset"], eps=EPS)
    return s["residual_out"], s["y"]


def _own_route(s):
    import paper_2607_08973_amd as S
    c = s["case"]
    S.sifar_route(s["logits"], s["ids"], s["weights"], score=c["score"], bias=s["bias"],
                  groups=c["groups"], top_groups=c["top_groups"], group_top=c["group_top"],
                  renorm=c["renorm"], scale=c["scale"])
    return s["ids"], s["weights"]


def _own_sample(s):
    import paper_2607_08973_amd as S
    S.sifar_sample(s["logits"], s["uniform"], s["tokens"], s["workspace"], probs=s["probs"],
                   temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                   min_p=s["min_p"])
    return s["tokens"], s["probs"]


def _plain_norm(s):
    c = s["case"]
    a = s["x"][0].float()
    for p in range(1, c["parts"]):
        a = a + s["x"][p].float()
    if s["post"] is not None:
        a = a * torch.rsqrt((a * a).mean(-1, keepdim=True) + EPS) * (s["post"].float()
                                                                     + c["offset"])
    if s["gate"] is not None:
        a = a * s["gate"].float()
    a = a * c["branch_scale"]
    if s["residual"] is not None:
        a = a + s["residual"].float() * c["residual_scale"]
    y = a * torch.rsqrt((a * a).mean(-1, keepdim=True) + EPS) * (s["weight"].float()
                                                                 + c["offset"])
    return a.to(s["rdt"]), y.to(s["x"].dtype)


def _plain_route(s):
    """Scores in 64 bits: a score next to another's decides which expert is chosen."""
    c = s["case"]
    x = s["logits"].double()
    T, E = x.shape
    there = x > -math.inf
    if c["score"] == "softmax":
        m = x.amax(-1, keepdim=True)
        e = torch.where(there, torch.where(x == m, 1.0, torch.exp(x - m)), 0.0)
        score = e / e.sum(-1, keepdim=True).clamp(min=1.0)
    else:
        score = torch.where(there, 1.0 / (1.0 + torch.exp(-x)), 0.0)
    choice = score if s["bias"] is None else score + s["bias"].double()
    there = there & (choice > -math.inf)
    key = torch.where(there, x if s["bias"] is None else choice, -math.inf)
    if c["groups"] > 1:
        per = E // c["groups"]
        best = torch.sort(torch.where(there, choice, -math.inf).view(T, c["groups"], per), -1,
                          descending=True)[0][..., :c["group_top"]]
        rank = best[..., 0]
        if c["group_top"] == 2 and per > 1:
            rank = rank + torch.where(best[..., 1] > -math.inf, best[..., 1], 0.0)
        order = torch.sort(rank, dim=-1, descending=True, stable=True)[1][:, :c["top_groups"]]
        stay = torch.zeros((T, c["groups"]), dtype=torch.bool, device=x.device)
        stay.scatter_(1, order, True)
        there = there & stay.repeat_interleave(per, 1)
        key = torch.where(there, key, -math.inf)
    ids = torch.sort(key, dim=-1, descending=True, stable=True)[1][:, :c["topk"]]
    ok = there.gather(1, ids)
    w = torch.where(ok, score.gather(1, ids), 0.0)
    if c["renorm"]:
        total = w.sum(-1, keepdim=True)
        w = torch.where(total > 0, w / total, 0.0)
    return torch.where(ok, ids, -1).int(), (w * c["scale"]).float()


def _plain_sample(s):
    """Running sums in 64 bits: a sum next to a border decides which token comes out."""
    x = s["logits"].float()
    T, V = x.shape
    x = torch.where(x > -math.inf, x, -math.inf)
    xs, order = torch.sort(x, dim=-1, descending=True, stable=True)
    top = xs[:, :1].double()
    t = s["temperature"].double()[:, None]
    greedy = ~(t > 0)
    z = (xs.double() - top) / torch.where(greedy, 1.0, t)
    z = torch.where(xs == top, 0.0, z)
    w = torch.where((xs > -math.inf) & (z >= CUT), torch.exp(z), 0.0)
    at = torch.arange(V, device=x.device)
    keep = w > 0
    if s["top_k"] is not None:
        k = s["top_k"][:, None]
        keep &= (at < k) | (k <= 0)
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        wk = torch.where(keep, w, 0.0)
        run_ = torch.cumsum(wk, -1)
        before = torch.cat([torch.zeros_like(run_[:, :1]), run_[:, :-1]], -1)
        keep &= (before < p * run_[:, -1:]) | (p >= 1) | (at == 0)
    if s["min_p"] is not None:
        keep &= (w >= s["min_p"].double()[:, None].clamp(max=1.0))
    w = torch.where(keep, w, 0.0)
    w = torch.zeros_like(w).scatter_(1, order, w)  # in the order of the tokens again
    run_ = torch.cumsum(w, -1)
    total = run_[:, -1:]
    token = (run_ <= s["uniform"].double()[:, None] * total).sum(-1, keepdim=True).clamp(max=V - 1)
    prob = w.gather(1, token) / total
    token = torch.where(greedy, order[:, :1], token)
    prob = torch.where(greedy, 1.0, prob)
    none = xs[:, :1] == -math.inf
    return (torch.where(none, -1, token)[:, 0].int(), torch.where(none, 0.0, prob)[:, 0].float())


# ---- work and the definition in 64 bits --------------------------------------------------------

def work(case):
    """Every input read once, every output written once. Operations: a partial's addition, two
    sums of squares, scales and weights of an element; an exponential (16) and what the choice
    compares for a logit."""
    T, e = case["tokens"], SIZE[case["dtype"]]
    if case["op"] == "block_norm":
        H, er = case["hidden"], 4 if case["residual"] == "fp32" else e
        gate = {"none": 0, "channel": H, "token": T * H}[case["gate"]]
        moved = T * H * (case["parts"] * e + er * (1 if case["residual"] == "none" else 2) + e)
        return {"bytes": moved + (gate + (1 + case["post"]) * H) * e,
                "flops": T * H * (case["parts"] + 10)}
    if case["op"] == "route":
        E = case["experts"]
        return {"bytes": T * E * e + 4 * E * case["bias"] + 8 * T * case["topk"],
                "flops": T * E * 20}
    return {"bytes": T * case["vocab"] * e + T * (16 + 4 * len(case["filters"])),
            "flops": T * case["vocab"] * 20}


def exact(case, seed):
    if case["op"] == "block_norm":
        s = _norm_inputs(case, seed)
        h = lambda t: None if t is None else t.double().cpu().numpy()
        x, post, weight, res, gate = (h(s[k]) for k in ("x", "post", "weight", "residual", "gate"))
        a = x.sum(0)
        if post is not None:
            a *= (post + case["offset"]) / np.sqrt(np.square(a).mean(-1, keepdims=True) + EPS)
        a *= case["branch_scale"] * (1.0 if gate is None else gate)
        if res is not None:
            a += case["residual_scale"] * res
        y = a * (weight + case["offset"]) / np.sqrt(np.square(a).mean(-1, keepdims=True) + EPS)
        return torch.from_numpy(a), torch.from_numpy(y)
    if case["op"] == "route":
        return _exact_route(case, seed)
    return _exact_sample(case, seed)


def _exact_route(case, seed):
    logits, bias = _route_inputs(case, seed)
    x = logits.double().cpu().numpy()
    T, E = x.shape
    if case["score"] == "softmax":
        score = np.exp(x - x.max(1, keepdims=True))
        score /= score.sum(1, keepdims=True)
    else:
        score = 1.0 / (1.0 + np.exp(-x))
    choice = score + (0.0 if bias is None else bias.double().cpu().numpy())
    rank = x.copy() if bias is None else choice.copy()
    G, per = case["groups"], E // case["groups"]
    if G > 1:
        part = np.sort(choice.reshape(T, G, per), -1)
        worth = part[..., -min(case["group_top"], per):].sum(-1)
        drop = np.argsort(-worth, 1, kind="stable")[:, case["top_groups"]:]
        out = np.zeros((T, G), bool)
        np.put_along_axis(out, drop, True, 1)
        rank[np.repeat(out, per, 1)] = -np.inf
    ids = np.argsort(-rank, 1, kind="stable")[:, :case["topk"]]
    w = np.take_along_axis(score, ids, 1)
    if case["renorm"]:
        w /= w.sum(1, keepdims=True)
    return torch.from_numpy(ids.astype(np.int32)), torch.from_numpy(w * case["scale"])


def _exact_sample(case, seed):
    s = {k: None if v is None else v.double().cpu().numpy()
         for k, v in _sample_inputs(case, seed).items()}
    tokens, probs = [], []
    for t in range(case["tokens"]):
        x, tau = s["logits"][t], s["temperature"][t]
        live = np.flatnonzero(x > -np.inf)
        if live.size == 0:
            tokens.append(-1)
            probs.append(0.0)
            continue
        x = x[live]
        if not tau > 0:
            tokens.append(int(live[np.argmax(x)]))
            probs.append(1.0)
            continue
        z = (x - x.max()) / tau
        live, z = live[z >= CUT], z[z >= CUT]
        if any(s[k] is not None for k in ("top_k", "top_p")):
            first = np.argsort(-z, kind="stable")
            n = first.size
            if s["top_k"] is not None and s["top_k"][t] > 0:
                n = min(n, int(s["top_k"][t]))
            if s["top_p"] is not None and s["top_p"][t] < 1:
                mass = np.cumsum(np.exp(z[first[:n]]))
                n = min(n, 1 + int(np.searchsorted(mass, s["top_p"][t] * mass[-1], "left")))
            pick = np.sort(first[:n])
            live, z = live[pick], z[pick]
        if s["min_p"] is not None:
            live, z = live[np.exp(z) >= s["min_p"][t]], z[np.exp(z) >= s["min_p"][t]]
        mass = np.cumsum(np.exp(z))
        i = min(int(np.searchsorted(mass, s["uniform"][t] * mass[-1], "right")), live.size - 1)
        tokens.append(int(live[i]))
        probs.append(float(np.exp(z[i]) / mass[-1]))
    return torch.tensor(tokens, dtype=torch.int32), torch.tensor(probs, dtype=torch.float64)
