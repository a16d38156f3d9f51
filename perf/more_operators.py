"""Cases of the operators of a mixture-of-experts layer and of 8-bit layers.

A program that serves a model whose experts are 8-bit integers with a scale for
each channel runs, for every layer, the choice of experts from the router's
logits, the experts' products on the carriers of the activations, the gated
activation between them, and the sum of the experts' outputs by the routing
weights.  Layers that all tokens pass through take the same product without
routes.  Calls have one token, a decode batch, or a prompt.  The dense products
have layer shapes of the benchmark; the others are generic.  ``draw`` spreads over
the same ranges.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def listed():
    return [
        # the router of one token: the smallest call, launch and latency
        {"name": "route_token", "op": "route", "dtype": "fp32", "tokens": 1, "experts": 128, "top": 8,
         "scoring": "softmax", "bias": False, "groups": 1, "kept": 1, "group_top": 1, "renorm": True, "scale": 1.0,
         "pad": 0},
        # a prompt through a router with a balance bias and groups, BF16 logits, rows of padding behind it
        {"name": "route_prompt", "op": "route", "dtype": "bf16", "tokens": 8191, "experts": 256, "top": 8,
         "scoring": "sigmoid", "bias": True, "groups": 8, "kept": 4, "group_top": 2, "renorm": True, "scale": 2.5,
         "pad": 57},
        # one token through a dense layer (queries, keys and values)
        {"name": "w8_token", "op": "w8", "dtype": "bf16", "rows": 1, "n": 6144, "k": 4096, "bias": False},
        # an odd decode batch through a dense layer of long rows
        {"name": "w8_batch", "op": "w8", "dtype": "fp16", "rows": 45, "n": 4096, "k": 14336, "bias": True},
        # several prompts through the widest dense layer
        {"name": "w8_prompt", "op": "w8", "dtype": "bf16", "rows": 7013, "n": 28672, "k": 8192, "bias": False},
        # one token through its experts
        {"name": "experts_token", "op": "experts", "dtype": "bf16", "tokens": 1, "top": 8, "experts": 64, "n": 4096,
         "k": 2048, "fan": True, "bias": False},
        # an odd decode batch through its experts' second layer (a row of activations for each route)
        {"name": "experts_batch", "op": "experts", "dtype": "fp16", "tokens": 61, "top": 6, "experts": 96, "n": 2048,
         "k": 1408, "fan": False, "bias": True},
        # a prompt through its experts
        {"name": "experts_prompt", "op": "experts", "dtype": "bf16", "tokens": 8191, "top": 4, "experts": 48,
         "n": 4096, "k": 4096, "fan": True, "bias": False},
        # between the experts' products of one token
        {"name": "gated_token", "op": "gated", "dtype": "bf16", "rows": 8, "width": 2048, "act": "silu", "fused": True},
        # between the products of several prompts
        {"name": "gated_prompt", "op": "gated", "dtype": "fp16", "rows": 7013, "width": 14336, "act": "gelu",
         "fused": True},
        # one token's experts joined
        {"name": "combine_token", "op": "combine", "dtype": "bf16", "tokens": 1, "top": 8, "width": 4096,
         "base": True},
        # a prompt's experts joined with a shared expert's output; some routes have no expert
        {"name": "combine_prompt", "op": "combine", "dtype": "fp16", "tokens": 8191, "top": 6, "width": 4104,
         "base": True},
    ]


def _log_uniform(rng: random.Random, lo: float, hi: float) -> int:
    return max(1, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.99)))))


def draw(rng: random.Random):
    """One more call of the same ranges: 1 to 8192 tokens, 8 to 512 experts, dense
    layers of up to 28672 rows of 16384, experts of up to 4096 by 4096."""
    op = rng.choice(["route", "route", "w8", "w8", "experts", "experts", "gated", "combine"])
    dtype = rng.choice(["bf16", "fp16"])
    if op == "route":
        experts = rng.choice([8, 16, 40, 60, 64, 72, 96, 128, 160, 200, 256, 384, 512])
        groups = rng.choice([1, 1] + [g for g in (2, 4, 5, 8, 16) if experts % g == 0 and experts // g >= 2])
        kept = rng.randint(1, groups)
        return {"op": op, "dtype": rng.choice(["bf16", "fp16", "fp32"]), "tokens": _log_uniform(rng, 1, 8192),
                "experts": experts, "top": rng.randint(1, min(12, kept * (experts // groups))),
                "scoring": rng.choice(["softmax", "sigmoid"]), "bias": rng.random() < 0.5, "groups": groups,
                "kept": kept, "group_top": rng.choice([1, 2]), "renorm": rng.random() < 0.7,
                "scale": rng.choice([1.0, 2.5]), "pad": rng.choice([0, 0, rng.randint(1, 40)])}
    if op == "w8":
        n, k = _log_uniform(rng, 200, 28672), 16 * _log_uniform(rng, 16, 1024)
        return {"op": op, "dtype": rng.choice(["bf16", "fp16", "fp32"]),
                "rows": _log_uniform(rng, 1, min(8192, 2**40 // (n * k))), "n": n, "k": k, "bias": rng.random() < 0.3}
    if op == "experts":
        experts = rng.choice([8, 16, 40, 64, 96, 128])
        n, k = _log_uniform(rng, 200, 4096), 16 * _log_uniform(rng, 16, 256)
        top = rng.randint(1, 8)
        tokens = _log_uniform(rng, 1, min(8192, 2**39 // (n * k * top)))
        return {"op": op, "dtype": dtype, "tokens": tokens, "top": top, "experts": experts, "n": n, "k": k,
                "fan": rng.random() < 0.5, "bias": rng.random() < 0.3}
    if op == "gated":
        width = 8 * _log_uniform(rng, 32, 1792)
        return {"op": op, "dtype": dtype, "rows": _log_uniform(rng, 1, min(32768, 2**27 // (2 * width))),
                "width": width, "act": rng.choice(["silu", "gelu"]), "fused": rng.random() < 0.6}
    width, top = 8 * _log_uniform(rng, 32, 1024), rng.randint(1, 8)
    return {"op": op, "dtype": dtype, "tokens": _log_uniform(rng, 1, min(8192, 2**27 // (width * top))), "top": top,
            "width": width, "base": rng.random() < 0.6}


# ---------------------------------------------------------------- inputs


def _generator(seed: int):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _rand(g, *shape):
    return torch.rand(shape, generator=g, device="cuda")


def _carriers(g, rows, k):
    """8-bit activations and their scales: a token has a scale of its own, some
    channels are large."""
    x = _randn(g, rows, k) * torch.where(_rand(g, k) < 0.005, 12.0, 1.0)
    top = x.abs().amax(1, keepdim=True).clamp_min(1e-6)
    return torch.round(x * (127.0 / top)).to(torch.int8), (top[:, 0] / 127.0) * (0.5 + 3.0 * _rand(g, rows))


def _weights(g, n, k):
    w = _randn(g, n, k)
    top = w.abs().amax(1, keepdim=True)
    return torch.round(w * (127.0 / top)).to(torch.int8), top[:, 0] * (0.02 / 127.0) * torch.exp2(_rand(g, n) - 0.5)


def _popular(g, tokens, experts, top):
    """Distinct experts of every token, some experts more in demand than others."""
    taste = 0.7 * _randn(g, experts) - torch.log(-torch.log(_rand(g, tokens, experts).clamp(1e-9, 1.0 - 1e-6)))
    return taste.topk(top, 1).indices.to(torch.int32)


def _plan(chosen, experts):
    """Routes grouped by expert: where each expert's begin, and the routes in order."""
    flat = chosen.flatten().long()
    key = torch.where((flat >= 0) & (flat < experts), flat, experts)
    order = torch.sort(key, stable=True).indices
    ends = torch.zeros(experts + 1, dtype=torch.long, device=flat.device).scatter_add_(0, key, torch.ones_like(key))
    ends = ends.cumsum(0)
    offsets = torch.cat((torch.zeros_like(ends[:1]), ends[:experts]))
    order = torch.where(torch.arange(flat.numel(), device=flat.device) < offsets[-1], order, -1)
    return torch.cat((offsets, order)).to(torch.int32)


def _inputs(case, seed):
    g = _generator(seed)
    dtype = DTYPES[case["dtype"]]
    if case["op"] == "route":
        t, e = case["tokens"], case["experts"]
        logits = 1.5 * _randn(g, t + case["pad"], e) + 0.5 * _randn(g, e)
        return {"logits": logits.to(dtype), "bias": 0.1 * _randn(g, e) if case["bias"] else None,
                "live": torch.full((1,), t, dtype=torch.int32, device="cuda") if case["pad"] else None}
    if case["op"] == "w8":
        x8, dx = _carriers(g, case["rows"], case["k"])
        w8, dw = _weights(g, case["n"], case["k"])
        return {"x8": x8, "dx": dx, "w8": w8, "dw": dw, "bias": _randn(g, case["n"]).to(dtype) if case["bias"] else None}
    if case["op"] == "experts":
        t, e, n, k = case["tokens"], case["experts"], case["n"], case["k"]
        x8, dx = _carriers(g, t if case["fan"] else t * case["top"], k)
        w8 = torch.empty((e, n, k), dtype=torch.int8, device="cuda")
        dw = torch.empty((e, n), device="cuda")
        for i in range(e):
            w8[i], dw[i] = _weights(g, n, k)
        return {"x8": x8, "dx": dx, "w8": w8, "dw": dw, "plan": _plan(_popular(g, t, e, case["top"]), e),
                "bias": _randn(g, e, n).to(dtype) if case["bias"] else None}
    if case["op"] == "gated":
        r, w = case["rows"], case["width"]
        if case["fused"]:  # the product that made them leaves both halves of a row side by side
            gate, up = (2.0 * _randn(g, r, 2 * w)).to(dtype).split(w, 1)
        else:
            gate, up = (2.0 * _randn(g, r, w)).to(dtype), (2.0 * _randn(g, r, w)).to(dtype)
        return {"gate": gate, "up": up}
    t, k, w = case["tokens"], case["top"], case["width"]
    chosen = _popular(g, t, 32, k)
    lost = _rand(g, t, k) < 0.02
    y = _randn(g, t * k, w)
    # what no expert has written holds anything
    y[lost.flatten()] = math.nan
    weights = torch.softmax(_randn(g, t, k), 1)
    return {"y": y.to(dtype), "weights": torch.where(lost, 0.0, weights), "chosen": torch.where(lost, -1, chosen),
            "base": _randn(g, t, w).to(dtype) if case["base"] else None}


def prepare(case, seed):
    return {"case": dict(case), **_inputs(case, seed)}


# ---------------------------------------------------------------- one pass


def run(s):
    c = s["case"]
    if own:
        import paper_2608_06763_amd as cq
        if c["op"] == "route":
            return cq.cq_route(s["logits"], c["top"], scoring=c["scoring"], bias=s["bias"], groups=c["groups"],
                               kept_groups=c["kept"], group_top=c["group_top"], renormalize=c["renorm"],
                               scale=c["scale"], live=s["live"])
        if c["op"] == "w8":
            return cq.cq_gemm_w8(s["x8"], s["dx"], s["w8"], s["dw"], bias=s["bias"], y_dtype=DTYPES[c["dtype"]])
        if c["op"] == "experts":
            return cq.cq_gemm_routed_w8(s["x8"], s["dx"], s["w8"], s["dw"], s["plan"],
                                        fan=c["top"] if c["fan"] else 1, bias=s["bias"], y_dtype=DTYPES[c["dtype"]])
        if c["op"] == "gated":
            return cq.cq_gated(s["gate"], s["up"], act=c["act"])
        return cq.cq_combine(s["y"], s["weights"], s["chosen"], 32, base=s["base"])
    if c["op"] == "route":
        return _plain_route(s, c)
    if c["op"] == "w8":
        y = (s["x8"].float() @ s["w8"].float().t()) * s["dx"][:, None] * s["dw"]
        if s["bias"] is not None:
            y = y + s["bias"].float()
        return y.to(DTYPES[c["dtype"]])
    if c["op"] == "experts":
        return _plain_experts(s, c)
    if c["op"] == "gated":
        x = s["gate"].float()
        if c["act"] == "silu":
            x = x / (1.0 + torch.exp(-x))
        else:
            x = 0.5 * x * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x * x * x)))
        return (x * s["up"].float()).to(s["gate"].dtype)
    t, k = s["chosen"].shape
    taken = (s["chosen"] >= 0) & (s["chosen"] < 32)
    rows = torch.where(taken[..., None], s["y"].view(t, k, -1).float(), 0.0)
    out = (rows * s["weights"][..., None]).sum(1)
    if s["base"] is not None:
        out = out + s["base"].float()
    return out.to(s["y"].dtype)


def _plain_route(s, c):
    """Scores in 64 bits: neighbours in a token's order are often closer than 32 tell apart."""
    l = s["logits"].double()
    tokens, experts = l.shape
    if c["scoring"] == "softmax":
        score = torch.exp(l - l.amax(1, keepdim=True))
        score = score / score.sum(1, keepdim=True)
    else:
        score = 1.0 / (1.0 + torch.exp(-l))
    choice = score if s["bias"] is None else score + s["bias"].double()
    if c["kept"] < c["groups"]:
        member = choice.view(tokens, c["groups"], -1)
        best = torch.sort(member, dim=2, descending=True).values[..., :c["group_top"]].sum(2)
        rank = torch.sort(best, dim=1, descending=True, stable=True).indices[:, :c["kept"]]
        kept = torch.zeros_like(best, dtype=torch.bool).scatter_(1, rank, True)
        choice = torch.where(kept[..., None], member, -math.inf).view(tokens, experts)
    chosen = torch.sort(choice, dim=1, descending=True, stable=True).indices[:, :c["top"]]
    weights = score.gather(1, chosen)
    if c["renorm"]:
        weights = weights / weights.sum(1, keepdim=True)
    weights = weights * c["scale"]
    if s["live"] is not None:
        dead = torch.arange(tokens, device=l.device)[:, None] >= s["live"]
        chosen, weights = torch.where(dead, -1, chosen), torch.where(dead, 0.0, weights)
    return chosen.to(torch.int32), weights.float(), _plan(chosen, experts)


def _plain_experts(s, c):
    experts, n, _ = s["w8"].shape
    plan, fan = s["plan"].long(), c["top"] if c["fan"] else 1
    order, ends = plan[experts + 1:], plan[:experts + 1].tolist()
    y = torch.empty((order.numel(), n), dtype=DTYPES[c["dtype"]], device=order.device)
    for e in range(experts):
        if ends[e] == ends[e + 1]:
            continue
        routes = order[ends[e]:ends[e + 1]]
        rows = routes // fan
        part = (s["x8"][rows].float() @ s["w8"][e].float().t()) * s["dx"][rows][:, None] * s["dw"][e]
        if s["bias"] is not None:
            part = part + s["bias"][e].float()
        y[routes] = part.to(y.dtype)
    return y


# ---------------------------------------------------------------- what a pass cannot do without


def work(case):
    size = 4.0 if case["dtype"] == "fp32" else 2.0
    if case["op"] == "route":
        t, e, k = case["tokens"] + case["pad"], case["experts"], case["top"]
        return {"bytes": t * e * size + 12.0 * t * k + 4.0 * e * (1 + case["bias"]), "flops": 8.0 * t * e}
    if case["op"] == "w8":
        m, n, k = case["rows"], case["n"], case["k"]
        return {"bytes": 1.0 * (m + n) * k + 4.0 * (m + n) + m * n * size + case["bias"] * n * size,
                "flops": 2.0 * m * n * k}
    if case["op"] == "experts":
        t, e, n, k, top = (case[x] for x in ("tokens", "experts", "n", "k", "top"))
        hit = e * (1.0 - (1.0 - top / e) ** t)  # experts that any token takes, all equally popular
        return {"bytes": hit * n * (k + 4.0 + case["bias"] * size) + t * (1 if case["fan"] else top) * (k + 4.0) +
                t * top * (n * size + 4.0), "flops": 2.0 * t * top * n * k}
    if case["op"] == "gated":
        n = 1.0 * case["rows"] * case["width"]
        return {"bytes": 3.0 * n * size, "flops": 6.0 * n}
    n = 1.0 * case["tokens"] * case["width"]
    return {"bytes": n * size * (case["top"] + 1 + case["base"]) + 8.0 * case["tokens"] * case["top"],
            "flops": 2.0 * n * case["top"]}


# ---------------------------------------------------------------- the same in 64 bits


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "route":
        return _exact_route(case, s)
    if case["op"] == "w8":
        y = torch.mm(s["x8"].double() * s["dx"].double()[:, None], (s["w8"].double() * s["dw"].double()[:, None]).t())
        return y if s["bias"] is None else y + s["bias"].double()
    if case["op"] == "experts":
        e, n = case["experts"], case["n"]
        plan = s["plan"].tolist()
        x = s["x8"].double() * s["dx"].double()[:, None]
        if case["fan"]:
            x = x.repeat_interleave(case["top"], 0)
        y = torch.zeros((len(plan) - e - 1, n), dtype=torch.float64, device="cuda")
        for i in range(e):
            at = plan[e + 1 + plan[i]:e + 1 + plan[i + 1]]
            if at:
                y[at] = x[at] @ (s["w8"][i].double() * s["dw"][i].double()[:, None]).t()
                if s["bias"] is not None:
                    y[at] += s["bias"][i].double()
        return y
    if case["op"] == "gated":
        x = s["gate"].double()
        if case["act"] == "silu":
            return s["up"].double() * x * torch.sigmoid(x)
        # 1 + tanh(z) = 2 sigmoid(2 z)
        return s["up"].double() * x * torch.sigmoid(math.sqrt(8.0 / math.pi) * x * (1.0 + 0.044715 * x**2))
    out = torch.zeros((case["tokens"], case["width"]), dtype=torch.float64, device="cuda")
    if case["base"]:
        out += s["base"].double()
    for j in range(case["top"]):
        row = torch.nan_to_num(s["y"][j::case["top"]].double())
        out += row * (s["weights"][:, j].double() * (s["chosen"][:, j] >= 0))[:, None]
    return out


def _exact_route(case, s):
    l = s["logits"].cpu().double().numpy()
    tokens, e, k, g = l.shape[0], case["experts"], case["top"], case["groups"]
    if case["scoring"] == "softmax":
        top = l.max(1, keepdims=True)
        score = np.exp(l - (top + np.log(np.exp(l - top).sum(1, keepdims=True))))
    else:
        score = np.exp(-np.logaddexp(0.0, -l))
    # without a bias the order is that of the logits; scores only matter where they are added
    choice = score + s["bias"].cpu().double().numpy() if case["bias"] else l
    closed = np.zeros((tokens, e), bool)
    if case["kept"] < g:
        adds = choice if case["bias"] or case["group_top"] == 1 else score
        member = -np.sort(-adds.reshape(tokens, g, e // g), 2)[..., :case["group_top"]]
        value = member.sum(2)
        index = np.lexsort((np.broadcast_to(np.arange(g), value.shape), -value), axis=1)
        left = np.ones((tokens, g), bool)
        np.put_along_axis(left, index[:, :case["kept"]], False, 1)
        closed = np.repeat(left, e // g, 1)
    at = np.broadcast_to(np.arange(e), choice.shape)
    chosen = np.lexsort((at, -choice, closed), axis=1)[:, :k]
    weights = np.take_along_axis(score, chosen, 1)
    if case["renorm"]:
        weights = weights / weights.sum(1, keepdims=True)
    weights = weights * case["scale"]
    chosen[case["tokens"]:], weights[case["tokens"]:] = -1, 0.0
    routes = [[] for _ in range(e)]
    for r, x in enumerate(chosen.ravel().tolist()):
        if x >= 0:
            routes[x].append(r)
    ends = np.cumsum([0] + [len(x) for x in routes])
    order = np.concatenate([np.asarray(x, np.int64) for x in routes] + [np.full(chosen.size - ends[-1], -1)])

    def whole(a):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()

    return whole(chosen), torch.from_numpy(weights).cuda(), whole(np.concatenate((ends, order)))
