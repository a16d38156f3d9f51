"""A decoder block on packed weights, from prompts to single tokens.

Every step of the block runs in this framework's kernels: norms with the residual
stream, packed products, rotary positions with the append to a paged cache,
attention over the cache, and the gated activation.  With --experts the gated
layers are a mixture of experts in 8-bit integers: a router's choice, the experts'
products on the carriers of the activations, and their sum by the router's weights.

    python examples/decoder_block.py            # a small block, checked against FP32
    python examples/decoder_block.py --experts 16 --top 4
    python examples/decoder_block.py --layers 8 --width 4096 --heads 32 --kv-heads 8 --ffn 14336 --tokens 64

It takes several prompts of different lengths in one call, decodes tokens for all of
them together, and then for many continuations of one shared prompt.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_06763_amd as cq  # noqa: E402

EPS = 1e-5
GROUP, BITS = 128, 4


def packed(g, n: int, k: int):
    """A random weight [n, k] in evenly spaced 4-bit levels, and its packed form."""
    w = torch.randn((n, k // GROUP, GROUP), generator=g) * k**-0.5
    scale = w.abs().amax(-1)
    codes = torch.round(w / scale[..., None] * 7.0).to(torch.int8).view(n, k)
    one, zero = np.full(scale.shape, 0x3C00, np.uint16), np.zeros(scale.shape, np.uint16)
    return cq.CQWeight.from_codes(codes.numpy(), scale.numpy(), one, zero, BITS, GROUP)


class Experts:
    """Gated layers of which every token takes `top`, in 8-bit integers with a scale for
    each channel, and their router."""

    def __init__(self, g, width, ffn, experts, top):
        self.ffn, self.experts, self.top = ffn, experts, top
        self.router = packed(g, experts, width)
        self.bias = (0.01 * torch.randn(experts, generator=g)).cuda()
        self.up, self.down = self.weights(g, 2 * ffn, width), self.weights(g, width, ffn)
        self.errors = []

    def weights(self, g, n, k):
        w = torch.randn((self.experts, n, k), generator=g).cuda() * k**-0.5
        scale = w.abs().amax(-1) / 127.0
        return torch.round(w / scale[..., None]).to(torch.int8), scale

    def __call__(self, h, check):
        """h [tokens, width], the normed stream; returns the experts' sum."""
        logits = cq.cq_gemm_model_dtype(self.router, h, y_dtype=torch.float32)
        chosen, weights, plan = cq.cq_route(logits, self.top, scoring="sigmoid", bias=self.bias)
        x8, dx = cq.cq_quantize_act_a8(h)
        pair = cq.cq_gemm_routed_w8(x8, dx, *self.up, plan, fan=self.top)
        h8, dh = cq.cq_gated_a8(*pair.split(self.ffn, dim=1))
        y = cq.cq_combine(cq.cq_gemm_routed_w8(h8, dh, *self.down, plan), weights, chosen, self.experts)
        if check:
            want = self.plain(h.float(), chosen, weights)
            self.errors.append(float((y.float() - want).norm() / want.norm()))
        return y

    def plain(self, x, chosen, weights):
        """The same in FP32 from the choice on."""
        out = torch.zeros_like(x)
        up, down = (w.float() * scale[..., None] for w, scale in (self.up, self.down))
        for j in range(self.top):
            for t, e in enumerate(chosen[:, j].tolist()):
                gate, rest = (up[e] @ x[t]).split(self.ffn)
                out[t] += weights[t, j] * (down[e] @ (torch.nn.functional.silu(gate) * rest))
        return out


class Block:
    """Weights of one decoder block, its pages of the cache, and its forward pass."""

    def __init__(self, width, heads, kv_heads, dim, ffn, pages, page, seed, a8=False, experts=0, top=2):
        g = torch.Generator().manual_seed(seed)
        self.heads, self.kv_heads, self.dim, self.ffn, self.a8 = heads, kv_heads, dim, ffn, a8
        self.qkv = packed(g, (heads + 2 * kv_heads) * dim, width)
        self.o = packed(g, width, heads * dim)
        self.experts = Experts(g, width, ffn, experts, top) if experts else None
        if not experts:
            self.up = packed(g, 2 * ffn, width)
            self.down = packed(g, width, ffn)
        self.norms = [(1.0 + 0.1 * torch.randn(width, generator=g)).to(torch.bfloat16).cuda() for _ in range(2)]
        self.k, self.v = (torch.zeros((pages, kv_heads, page, dim), dtype=torch.bfloat16, device="cuda")
                          for _ in range(2))

    def product(self, w, stream, norm, y=None):
        """The stream plus y, through a norm and a packed product: (product, stream)."""
        if self.a8:
            x8, dx, stream = cq.cq_norm_residual_a8(stream, norm, EPS, y=y)
            return cq.cq_gemm_a8(w, x8, dx, y_dtype=torch.bfloat16), stream
        h, stream = cq.cq_norm_residual(stream, norm, EPS, y=y)
        return cq.cq_gemm_model_dtype(w, h), stream

    def __call__(self, stream, y, rope, step):
        """stream [tokens, width] and the last block's output y; returns the same."""
        qkv, stream = self.product(self.qkv, stream, self.norms[0], y)
        t = qkv.shape[0]
        qkv = qkv.view(t, -1, self.dim)
        q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], dim=1)
        q = cq.cq_rope_append(q, k, v, *rope, step["positions"], step["slots"], self.k, self.v)
        if "prefix_table" in step:
            a = cq.cq_attn_shared_prefix(q, self.k, self.v, step["prefix_table"], step["prefix_len"], step["tables"],
                                         step["lens"], step["max_kv"])
        else:
            a = cq.cq_attn_paged(q, self.k, self.v, step["tables"], step["lens"], step["max_kv"],
                                 q_starts=step["starts"], max_q=step["max_q"])
        a = cq.cq_gemm_model_dtype(self.o, a.view(t, -1))
        if self.experts:
            h, stream = cq.cq_norm_residual(stream, self.norms[1], EPS, y=a)
            return stream, self.experts(h, step["check"])
        gated, stream = self.product(self.up, stream, self.norms[1], a)
        return stream, cq.cq_gemm_model_dtype(self.down, cq.cq_gated(*gated.split(self.ffn, dim=1)))


class Pages:
    """Which pages each sequence holds; host bookkeeping only."""

    def __init__(self, pages, page, width):
        self.free, self.page, self.width, self.held = list(range(pages)), page, width, {}

    def step(self, new, prefix=None):
        """Room for new[s] tokens of every sequence s; the arguments of one step.
        prefix: a sequence whose tokens all others begin with."""
        ids, front = list(new), len(self.held[prefix][1]) if prefix is not None else 0
        positions, slots = [], []
        for s in ids:
            table, tokens = self.held.setdefault(s, ([], []))
            for _ in range(new[s]):
                if len(tokens) % self.page == 0:
                    table.append(self.free.pop())
                positions.append(front + len(tokens))
                tokens.append(table[-1] * self.page + len(tokens) % self.page)
                slots.append(tokens[-1])
        tables = np.zeros((len(ids), self.width), np.int32)
        for i, s in enumerate(ids):
            tables[i, :len(self.held[s][0])] = self.held[s][0]
        lens = [len(self.held[s][1]) for s in ids]
        count = [new[s] for s in ids]

        def device(a):
            return torch.from_numpy(np.asarray(a, np.int32)).cuda()

        out = {"positions": device(positions), "slots": device(slots), "tables": device(tables), "lens": device(lens),
               "max_kv": max(lens), "max_q": max(count),
               "starts": device(np.cumsum([0] + count)) if max(count) > 1 else None}
        if prefix is not None:
            out["prefix_table"], out["prefix_len"] = device(self.held[prefix][0]), front
        return out


def rope_tables(rows, dim):
    angle = torch.arange(rows)[:, None] * 10000.0 ** (-torch.arange(0, dim, 2) / dim)
    return angle.cos().cuda(), angle.sin().cuda()


def forward(blocks, x, rope, step):
    stream, y = x, None
    for b in blocks:
        stream, y = b(stream, y, rope, step)
    return stream.float() + y.float()


# ---------------------------------------------------------------- the same in FP32, without a cache


def plain_forward(blocks, x, rope, segments):
    """x [tokens, width]: sequences of the given lengths, whole; FP32 throughout."""
    x, cos, sin = x.float(), *rope
    for b in blocks:
        weights = [cq.cq_decode_ref(w, want_codes=False)[1] for w in (b.qkv, b.o, b.up, b.down)]

        def norm(v, w):
            return v * torch.rsqrt((v * v).mean(1, keepdim=True) + EPS) * w.float()

        qkv = (norm(x, b.norms[0]) @ weights[0].t()).view(len(x), -1, b.dim)
        out, row = [], 0
        for n in segments:
            q, k, v = (t.transpose(0, 1) for t in qkv[row:row + n].split([b.heads, b.kv_heads, b.kv_heads], dim=1))
            half, c, s = b.dim // 2, cos[:n], sin[:n]
            q, k = (torch.cat((t[..., :half] * c - t[..., half:] * s, t[..., half:] * c + t[..., :half] * s), -1)
                    for t in (q, k))
            k, v = (t.repeat_interleave(b.heads // b.kv_heads, 0) for t in (k, v))
            a = (q @ k.transpose(1, 2)) * b.dim**-0.5
            a = torch.softmax(a + torch.full((n, n), -torch.inf, device=x.device).triu(1), -1) @ v
            out.append(a.transpose(0, 1).reshape(n, -1))
            row += n
        x = x + torch.cat(out) @ weights[1].t()
        gate, up = (norm(x, b.norms[1]) @ weights[2].t()).split(b.ffn, dim=1)
        x = x + (torch.nn.functional.silu(gate) * up) @ weights[3].t()
    return x


def serve(layers=2, width=1024, heads=8, kv_heads=2, dim=128, ffn=2816, prompts=(37, 5, 130), tokens=4, samples=6,
          page=16, a8=False, check=True, experts=0, top=2):
    """Prompts, then `tokens` tokens of each; then the same for `samples` continuations
    of the last prompt.  Returns the relative errors against FP32 (check), or times: of
    each sequence, or of each call of the experts, given their choice, which a sequence's
    small errors may turn."""
    longest = max(prompts) + tokens + 1
    pages = sum(-(-(n + tokens) // page) for n in prompts) + samples * -(-tokens // page)
    blocks = [Block(width, heads, kv_heads, dim, ffn, pages, page, seed, a8, experts, top) for seed in range(layers)]
    rope, book = rope_tables(longest, dim), Pages(pages, page, -(-longest // page))
    g = torch.Generator().manual_seed(99)
    seq = {s: torch.randn((n + tokens, width), generator=g).to(torch.bfloat16).cuda() for s, n in enumerate(prompts)}
    more = torch.randn((samples, tokens, width), generator=g).to(torch.bfloat16).cuda()
    got, times = {s: [] for s in seq}, []

    def run(x, new, prefix=None):
        step = book.step(new, prefix)
        step["check"] = check
        torch.cuda.synchronize()
        begin = time.perf_counter()
        y = forward(blocks, x, rope, step)
        torch.cuda.synchronize()
        times.append(time.perf_counter() - begin)
        return y

    y = run(torch.cat([seq[s][:n] for s, n in enumerate(prompts)]), dict(enumerate(prompts)))
    for s, part in enumerate(y.split(list(prompts))):
        got[s].append(part)
    tail, base = [], len(prompts) - 1
    for i in range(tokens):  # the last prompt stays as it is: its continuations follow below
        y = run(torch.stack([seq[s][n + i] for s, n in enumerate(prompts[:-1])]), {s: 1 for s in range(base)})
        for s in range(base):
            got[s].append(y[s:s + 1])
    for i in range(tokens):
        tail.append(run(more[:, i].contiguous(), {("sample", j): 1 for j in range(samples)}, prefix=base))
    if not check:
        return times
    if experts:
        return [e for b in blocks for e in b.experts.errors]
    errors = []

    def compare(a, b):
        errors.append(float((a - b).norm() / b.norm()))

    whole = [seq[s] for s in range(base)] + [seq[base][:prompts[base]]]
    want = plain_forward(blocks, torch.cat(whole), rope, [len(w) for w in whole])
    for s, part in enumerate(want.split([len(w) for w in whole])):
        compare(torch.cat(got[s]), part)
    for j in range(samples):
        x = torch.cat((seq[base][:prompts[base]], more[j]))
        compare(torch.stack([t[j] for t in tail]), plain_forward(blocks, x, rope, [len(x)])[-tokens:])
    return errors


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("layers", 2), ("width", 1024), ("heads", 8), ("kv-heads", 2), ("ffn", 2816), ("tokens", 4),
                        ("samples", 6), ("experts", 0), ("top", 2)):
        p.add_argument(f"--{name}", type=int, default=value)
    p.add_argument("--a8", action="store_true", help="products of the normed stream over Dynamic-A8")
    a = p.parse_args()
    sizes = {k: v for k, v in vars(a).items()}
    if a.width <= 1024:
        errors = serve(**sizes)
        print("relative error against FP32, each", "call of the experts:" if a.experts else "sequence:", " ".join(f"{e:.4f}" for e in errors))
    else:
        times = serve(**sizes, prompts=(900, 2000, 1100), check=False)
        n = a.tokens
        print(f"4000 prompt tokens {times[0] * 1e3:.2f} ms; a token of 2 sequences {min(times[1:1 + n]) * 1e3:.3f} ms; "
              f"of {a.samples} continuations {min(times[1 + n:]) * 1e3:.3f} ms")


if __name__ == "__main__":
    main()
