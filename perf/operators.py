"""Cases of the operators between the packed products of a decoder block.

A program that serves a model whose linear layers are packed by this framework
runs, between two of them, a norm with the residual stream, the rotation of
queries and keys with the append to a paged cache, and the attention that reads
the cache: for one token of one or many sequences, for a batch that shares a
long prefix, for prompts and for chunks of them.  Activations are BF16 or FP16.
The listed cases are such calls at the layer shapes of the benchmark (32 query
heads over 8 key heads of 128, width 4096) and at generic ones; ``draw`` spreads
over the same ranges.  Sequence lengths are ragged and follow from the case
alone, since a serving program knows them on the host.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    return [
        # one token between two blocks: the smallest call, launch and latency
        {"name": "norm_token", "op": "norm", "dtype": "bf16", "tokens": 1, "width": 4096, "post": False,
         "gate": False},
        # several prompts through norms on both sides of a gated block
        {"name": "norm_prompts", "op": "norm", "dtype": "bf16", "tokens": 7013, "width": 8192, "post": True,
         "gate": True},
        # the new token of one sequence
        {"name": "append_token", "op": "append", "dtype": "bf16", "tokens": 1, "heads": 32, "kv_heads": 8, "dim": 128,
         "rot": 128, "interleaved": False, "page": 16},
        # an odd decode batch, half of each head rotated, neighbouring pairs
        {"name": "append_batch", "op": "append", "dtype": "fp16", "tokens": 61, "heads": 40, "kv_heads": 8, "dim": 64,
         "rot": 32, "interleaved": True, "page": 32},
        # a prompt's keys and values
        {"name": "append_prompt", "op": "append", "dtype": "bf16", "tokens": 8191, "heads": 64, "kv_heads": 8,
         "dim": 128, "rot": 128, "interleaved": False, "page": 64},
        # one sequence early in its answer
        _attn("token_short", batch=1, q_max=1, cached=300),
        # a decode batch of sequences of very different lengths, capped scores
        _attn("token_batch", batch=45, q_max=1, cached=8000, dtype="fp16", softcap=30.0, page=16),
        # one sequence with a long history
        _attn("token_long", batch=1, q_max=1, cached=200000, page=64),
        # several prompts at once, sliding window, bias by distance
        _attn("prompts_ragged", batch=7, q_max=2300, cached=0, dtype="fp16", heads=16, kv_heads=16, dim=64,
              slopes=True, window=1000),
        # a long prompt
        _attn("prompt", batch=1, q_max=8192, cached=0, page=64),
        # a few sequences behind one system prompt
        _attn("shared_few", op="shared", batch=9, q_max=1, cached=200, shared=1500),
        # many samples of one long document
        _attn("shared_many", op="shared", batch=90, q_max=1, cached=1200, shared=24000, page=64),
    ]


def _attn(name, op="attn", dtype="bf16", heads=32, kv_heads=8, dim=128, page=32, softcap=0.0, window=0, slopes=False,
          bidir=0, shared=0, lens=1, **sizes):
    case = {"op": op, "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page,
            "softcap": softcap, "window": window, "slopes": slopes, "bidir": bidir, "shared": shared, "lens": lens}
    case.update(sizes)
    if name:
        case["name"] = name
    return case


def _log_uniform(rng: random.Random, lo: float, hi: float) -> int:
    return max(1, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.99)))))


def draw(rng: random.Random):
    """One more call of the same ranges: 1 to 8192 new tokens, histories of up
    to 200000 tokens, 1 to 128 sequences, heads of 64, 128 or 256."""
    op = rng.choice(["norm", "append", "token", "token", "prompt", "prompt", "shared"])
    dtype = rng.choice(["bf16", "fp16"])
    if op == "norm":
        return {"op": "norm", "dtype": dtype, "tokens": _log_uniform(rng, 1, 8192),
                "width": 8 * _log_uniform(rng, 64, 1024), "post": rng.random() < 0.5, "gate": rng.random() < 0.5}
    dim = rng.choice([64, 128, 128, 256])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16])
    heads = kv_heads * rng.choice([1, 2, 4, 4, 5, 7, 8])
    page = rng.choice([16, 32, 64, 128])
    if op == "append":
        return {"op": "append", "dtype": dtype, "tokens": _log_uniform(rng, 1, min(8192, 2**26 // (heads * dim))),
                "heads": heads, "kv_heads": kv_heads, "dim": dim, "rot": rng.choice([dim, dim, dim // 2]),
                "interleaved": rng.random() < 0.3, "page": page}
    kind = {"dtype": dtype, "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page,
            "softcap": rng.choice([0.0, 0.0, 50.0]), "lens": rng.randrange(1 << 20)}
    # elements of the keys that all sequences hold, and scores in all
    keys, scores = 2**28 // (kv_heads * dim), 2**30 // heads
    if op == "prompt":
        q_max = _log_uniform(rng, 2, 4096)
        cached = rng.choice([0, 0, _log_uniform(rng, 1, 16384)])
        batch = _log_uniform(rng, 1, 16)
        batch = max(1, min(batch, keys // (q_max + cached), scores // (q_max * (q_max + cached)), 8192 // q_max))
        return _attn(None, batch=batch, q_max=q_max, cached=cached, window=rng.choice([0, 0, 500]),
                     slopes=rng.random() < 0.3, bidir=rng.choice([0, 0, min(q_max, 100)]), **kind)
    batch = _log_uniform(rng, 1, 128)
    if op == "shared":
        shared = _log_uniform(rng, 100, min(32768, keys, scores // batch))
        cached = _log_uniform(rng, 1, max(1, min(2000, keys // batch)))
        return _attn(None, op="shared", batch=batch, q_max=1, cached=cached, shared=shared, **kind)
    cached = _log_uniform(rng, 1, min(200000, keys // batch, scores // batch))
    return _attn(None, batch=batch, q_max=1, cached=cached, window=rng.choice([0, 0, 0, 1000]),
                 slopes=rng.random() < 0.3, **kind)


# ---------------------------------------------------------------- inputs


def _lengths(case):
    """New and cached tokens of each sequence, ragged over a factor of about
    eight; the first has the most of both."""
    rng = random.Random(case["lens"])
    new, old = [case["q_max"]], [case["cached"]]
    for _ in range(case["batch"] - 1):
        new.append(_log_uniform(rng, max(1, case["q_max"] / 8), case["q_max"]))
        old.append(_log_uniform(rng, max(1, case["cached"] / 8), case["cached"]) if case["cached"] else 0)
    return new, old


def _generator(seed: int):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape, dtype):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _inputs(case, seed):
    g = _generator(seed)
    dtype = DTYPES[case["dtype"]]
    if case["op"] == "norm":
        t, h = case["tokens"], case["width"]
        # the stream has a scale per token and a few large channels
        stream = torch.randn((t, h), generator=g, device="cuda")
        stream *= 1.0 + 4.0 * torch.rand((t, 1), generator=g, device="cuda")
        stream *= torch.where(torch.rand((h,), generator=g, device="cuda") < 0.005, 20.0, 1.0)
        return {"y": _randn(g, t, h, dtype=dtype), "stream": stream.to(dtype),
                "weight": (1.0 + 0.2 * torch.randn((h,), generator=g, device="cuda")).to(dtype),
                "post": _randn(g, h, dtype=dtype) if case["post"] else None,
                "gate": torch.rand((t, h), generator=g, device="cuda").to(dtype) if case["gate"] else None}
    heads, kv_heads, dim, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    if case["op"] == "append":
        t, rot = case["tokens"], case["rot"]
        pages = -(-t // page) + 5
        # the product that made them leaves queries, keys and values of a token side by side
        qkv = _randn(g, t, heads + 2 * kv_heads, dim, dtype=dtype)
        angle = torch.arange(t + 100, device="cuda")[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, device="cuda") / rot)
        order = torch.randperm(pages, generator=g, device="cuda")
        i = torch.arange(t, device="cuda") + 3
        return {"q": qkv[:, :heads], "k": qkv[:, heads:heads + kv_heads], "v": qkv[:, heads + kv_heads:],
                "cos": angle.cos(), "sin": angle.sin(), "positions": (i + 64).to(torch.int32),
                "slots": (order[i // page] * page + i % page).to(torch.int32),
                "k_cache": torch.zeros((pages, kv_heads, page, dim), dtype=dtype, device="cuda"),
                "v_cache": torch.zeros((pages, kv_heads, page, dim), dtype=dtype, device="cuda")}
    new, old = _lengths(case)
    total = sum(new)
    lens = [a + b for a, b in zip(new, old)]
    width = -(-max(lens) // page)
    front = -(-case["shared"] // page)
    pages = sum(-(-n // page) for n in lens) + front
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    used = (torch.tensor(lens, device="cuda")[:, None] + (page - 1)) // page
    column = torch.arange(width, device="cuda")[None]
    taken = column < used
    first = torch.cumsum(used, 0) - used + front
    tables = torch.where(taken, order[(first + column).clamp_max(pages - 1)], 0).to(torch.int32)
    # keys have a few large channels, values a mean of their own
    keys = torch.randn((pages, kv_heads, page, dim), generator=g, device="cuda")
    keys *= torch.where(torch.rand((kv_heads, 1, dim), generator=g, device="cuda") < 0.03, 4.0, 1.0)
    values = torch.randn((pages, kv_heads, page, dim), generator=g, device="cuda")
    values += 0.3 * torch.randn((kv_heads, 1, dim), generator=g, device="cuda")
    qkv = _randn(g, total, heads + 2 * kv_heads, dim, dtype=dtype)
    starts = torch.tensor([0] + new, device="cuda").cumsum(0).to(torch.int32)
    state = {"q": qkv[:, :heads], "k_cache": keys.to(dtype), "v_cache": values.to(dtype), "tables": tables,
             "q_starts": starts if case["q_max"] > 1 else None,
             "kv_lens": torch.tensor(lens, device="cuda", dtype=torch.int32), "max_q": max(new), "max_kv": max(lens),
             "softcap": case["softcap"], "window": case["window"], "slopes": None, "bidir": None}
    if case["slopes"]:
        state["slopes"] = 2.0 ** (-8.0 * (torch.arange(heads, device="cuda") + 1.0) / heads)
    if case["bidir"]:
        state["bidir"] = torch.randint(0, case["bidir"] + 1, (len(new),), generator=g, device="cuda").to(torch.int32)
    if case["op"] == "shared":
        state["prefix_table"], state["prefix_len"] = order[:front].contiguous(), case["shared"]
    return state


def prepare(case, seed):
    return {"op": case["op"], "interleaved": case.get("interleaved", False), **_inputs(case, seed)}


# ---------------------------------------------------------------- one pass

EPS = 1e-5


def run(s):
    if own:
        import paper_2608_06763_amd as cq
        if s["op"] == "norm":
            return cq.cq_norm_residual(s["stream"], s["weight"], EPS, y=s["y"], post_weight=s["post"], gate=s["gate"],
                                       alpha=0.5)
        if s["op"] == "append":
            q = cq.cq_rope_append(s["q"], s["k"], s["v"], s["cos"], s["sin"], s["positions"], s["slots"], s["k_cache"],
                                  s["v_cache"], interleaved=s["interleaved"])
            return [q, s["k_cache"], s["v_cache"]]
        if s["op"] == "shared":
            return cq.cq_attn_shared_prefix(s["q"], s["k_cache"], s["v_cache"], s["prefix_table"], s["prefix_len"],
                                            s["tables"], s["kv_lens"], s["max_kv"], q_starts=s["q_starts"],
                                            max_q=s["max_q"], softcap=s["softcap"])
        return cq.cq_attn_paged(s["q"], s["k_cache"], s["v_cache"], s["tables"], s["kv_lens"], s["max_kv"],
                                q_starts=s["q_starts"], max_q=s["max_q"], softcap=s["softcap"], window=s["window"],
                                slopes=s["slopes"], bidir=s["bidir"])
    if s["op"] == "norm":
        return _plain_norm(s)
    if s["op"] == "append":
        return _plain_append(s)
    return _plain_attention(s)


def _plain_norm(s):
    u = s["y"].float()
    if s["post"] is not None:
        u = u * torch.rsqrt((u * u).mean(1, keepdim=True) + EPS) * s["post"].float()
    if s["gate"] is not None:
        u = u * s["gate"].float()
    r = s["stream"].float() + 0.5 * u
    h = r * torch.rsqrt((r * r).mean(1, keepdim=True) + EPS) * s["weight"].float()
    return h.to(s["y"].dtype), r.to(s["y"].dtype)


def _plain_rotate(x, cos, sin, interleaved):
    rot = 2 * cos.shape[-1]
    x = x.float()
    a, rest = x[..., :rot], x[..., rot:]
    if interleaved:
        x1, x2 = a[..., 0::2], a[..., 1::2]
        a = torch.stack((x1 * cos - x2 * sin, x2 * cos + x1 * sin), -1).flatten(-2)
    else:
        x1, x2 = a[..., :rot // 2], a[..., rot // 2:]
        a = torch.cat((x1 * cos - x2 * sin, x2 * cos + x1 * sin), -1)
    return torch.cat((a, rest), -1)


def _plain_append(s):
    at = s["positions"].long()
    cos, sin = s["cos"][at][:, None], s["sin"][at][:, None]
    slots, page = s["slots"].long(), s["k_cache"].shape[2]
    q = _plain_rotate(s["q"], cos, sin, s["interleaved"]).to(s["q"].dtype)
    k = _plain_rotate(s["k"], cos, sin, s["interleaved"]).to(s["q"].dtype)
    s["k_cache"][slots // page, :, slots % page] = k
    s["v_cache"][slots // page, :, slots % page] = s["v"]
    return [q, s["k_cache"], s["v_cache"]]


def _plain_pages(cache, tables, tokens):
    """The pages of each table side by side, FP32 [..., kv heads, tokens, dim]."""
    x = cache[tables.long()].transpose(-4, -3).flatten(-3, -2)
    return x[..., :tokens, :].float()


def _plain_attention(s):
    q, dtype = s["q"], s["q"].dtype
    total, heads, dim = q.shape
    kv_heads, batch, max_q = s["k_cache"].shape[1], s["kv_lens"].numel(), s["max_q"]
    group = heads // kv_heads
    lens = s["kv_lens"].long()
    starts = s["q_starts"]
    starts = torch.arange(batch + 1, device=q.device) if starts is None else starts.long()
    local = torch.arange(max_q, device=q.device)
    token = starts[:-1, None] + local
    # queries padded to the longest, [batch, kv heads, group * max_q, dim]
    x = q[token.clamp_max(total - 1)].float().view(batch, max_q, kv_heads, group, dim)
    x = x.permute(0, 2, 3, 1, 4).reshape(batch, kv_heads, group * max_q, dim)
    keys, values = (_plain_pages(s[c], s["tables"], s["max_kv"]) for c in ("k_cache", "v_cache"))
    score = (x @ keys.transpose(-1, -2)) * dim**-0.5
    score = score.view(batch, kv_heads, group, max_q, -1)
    if s["softcap"]:
        score = s["softcap"] * torch.tanh(score / s["softcap"])
    i = (lens - (starts[1:] - starts[:-1]))[:, None, None] + local[:, None]
    j = torch.arange(s["max_kv"], device=q.device)
    if s["slopes"] is not None:
        score = score + s["slopes"].view(kv_heads, group, 1, 1) * (j - i)[:, None, None]
    seen = j <= i
    if s["window"]:
        seen = seen & (j > i - s["window"])
    if s["bidir"] is not None:
        seen = seen | (j < s["bidir"].long()[:, None, None])
    seen = seen & (j < lens[:, None, None]) & (i >= 0)
    score = torch.where(seen[:, None, None], score, -math.inf)
    if "prefix_table" in s:
        front, front_v = (_plain_pages(s[c], s["prefix_table"], s["prefix_len"]) for c in ("k_cache", "v_cache"))
        rows = x.transpose(0, 1).reshape(kv_heads, -1, dim)
        before = (rows @ front.transpose(-1, -2)) * dim**-0.5
        if s["softcap"]:
            before = s["softcap"] * torch.tanh(before / s["softcap"])
        before = before.view(kv_heads, batch, group, max_q, -1).transpose(0, 1)
        score = torch.cat((before, score), -1)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(torch.isinf(top), 0.0, top))
    norm = p.sum(-1, keepdim=True)
    p = p / torch.where(norm > 0, norm, 1.0)
    n = s.get("prefix_len", 0)
    out = p[..., n:].reshape(batch, kv_heads, group * max_q, -1) @ values
    out = out.view(batch, kv_heads, group, max_q, dim)
    if n:
        before = p[..., :n].transpose(0, 1).reshape(kv_heads, -1, n) @ front_v
        out = out + before.view(kv_heads, batch, group, max_q, dim).transpose(0, 1)
    # back to one row for each token
    out = out.permute(0, 3, 1, 2, 4).reshape(batch * max_q, heads, dim)
    row = torch.arange(total, device=q.device)
    of = torch.searchsorted(starts[1:].contiguous(), row, right=True)
    return out[of * max_q + row - starts[of]].to(dtype)


# ---------------------------------------------------------------- what a pass cannot do without


def _seen(case):
    """Visible (query, own key) pairs of a head, and own keys that any query sees."""
    pairs = keys = 0
    for n, c in zip(*_lengths(case)):
        w = case["window"] or n + c
        full = min(n, max(0, n + c - w))  # queries whose window is whole
        rest = n - full
        pairs += full * w + rest * (c + 1) + rest * (rest - 1) // 2
        # tokens of a prefix that its own tokens see ahead of them, on average half of its most
        pairs += min(case["bidir"] // 2, n) ** 2 // 2 if not c else 0
        keys += min(n + c, w + n - 1)
    return pairs, keys


def work(case):
    if case["op"] == "norm":
        n = case["tokens"] * case["width"]
        return {"bytes": 2.0 * (n * (5 if case["gate"] else 4) + case["width"] * (2 if case["post"] else 1)),
                "flops": n * (7.0 + 4.0 * case["post"] + case["gate"])}
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    if case["op"] == "append":
        t = case["tokens"]
        return {"bytes": t * (4.0 * (heads + 2 * kv_heads) * dim + 4.0 * case["rot"] + 8.0),
                "flops": t * 3.0 * (heads + kv_heads) * case["rot"]}
    new, _ = _lengths(case)
    total = sum(new)
    pairs, keys = _seen(case)
    pairs += total * case["shared"]
    keys += case["shared"]
    return {"bytes": 4.0 * total * heads * dim + 4.0 * keys * kv_heads * dim, "flops": 4.0 * pairs * heads * dim}


# ---------------------------------------------------------------- the same in 64 bits


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "norm":
        y, r = s["y"].double(), s["stream"].double()
        if s["post"] is not None:
            y = y / (y.pow(2).mean(1, keepdim=True) + EPS).sqrt() * s["post"].double()
        if s["gate"] is not None:
            y = y * s["gate"].double()
        r = r + y / 2
        return r / (r.pow(2).mean(1, keepdim=True) + EPS).sqrt() * s["weight"].double(), r
    if case["op"] == "append":
        at, rot = s["positions"].long(), case["rot"]
        turn = torch.complex(s["cos"][at].double(), s["sin"][at].double())[:, None]
        out = []
        for x in (s["q"], s["k"]):
            x = x.double().clone()
            lo, hi = (slice(0, rot, 2), slice(1, rot, 2)) if case["interleaved"] else \
                (slice(0, rot // 2), slice(rot // 2, rot))
            z = torch.complex(x[..., lo], x[..., hi]) * turn
            x[..., lo], x[..., hi] = z.real, z.imag
            out.append(x)
        page = case["page"]
        k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
        for h in range(case["kv_heads"]):
            for cache, x in ((k_cache, out[1]), (v_cache, s["v"].double())):
                flat = cache[:, h].reshape(-1, case["dim"])
                flat[s["slots"].long()] = x[:, h]
                cache[:, h] = flat.view(-1, page, case["dim"])
        return [out[0], k_cache, v_cache]
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    group, out, row = heads // kv_heads, torch.zeros_like(s["q"], dtype=torch.float64), 0

    def held(cache, table, tokens, h):
        return cache[table.long(), h].reshape(-1, dim)[:tokens].double()

    new, old = _lengths(case)
    for b, (n, c) in enumerate(zip(new, old)):
        at = torch.arange(c, c + n, device="cuda")
        i, j = at.repeat_interleave(group)[:, None], torch.arange(n + c, device="cuda")[None]
        hidden = j > i
        if case["window"]:
            hidden |= i - j >= case["window"]
        if s["bidir"] is not None:
            hidden &= j >= s["bidir"][b]
        for h in range(kv_heads):
            q = s["q"][row:row + n, h * group:(h + 1) * group].double().reshape(n * group, dim)
            a, v = q @ held(s["k_cache"], s["tables"][b], n + c, h).t() / math.sqrt(dim), \
                held(s["v_cache"], s["tables"][b], n + c, h)
            if case["softcap"]:
                a = torch.tanh(a / case["softcap"]) * case["softcap"]
            if s["slopes"] is not None:
                a -= s["slopes"][h * group:(h + 1) * group].double().repeat(n)[:, None] * (i - j)
            a.masked_fill_(hidden, -math.inf)
            if case["shared"]:
                f = q @ held(s["k_cache"], s["prefix_table"], case["shared"], h).t() / math.sqrt(dim)
                if case["softcap"]:
                    f = torch.tanh(f / case["softcap"]) * case["softcap"]
                a = torch.cat((f, a), 1)
                v = torch.cat((held(s["v_cache"], s["prefix_table"], case["shared"], h), v))
            out[row:row + n, h * group:(h + 1) * group] = (torch.softmax(a, 1) @ v).view(n, group, dim)
        row += n
    return out
