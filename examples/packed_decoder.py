"""A decoder layer on packed lanes: attention over a bounded cache, and a layer of experts.

    python examples/packed_decoder.py [--width 512 --heads 8 --kv-heads 2 --experts 8 --topk 2 --tokens 200 --bits 4 --type bf16]

Sequences with prompts of different lengths decode together, a token each a step. The projections are 4-bit weights
(samd.matvec4), keys and values go into a paged cache of 4- or 8-bit lanes (samd.cache_append), attention reads it and
counts the tokens' weights (samd.paged_attention), and a sequence that has filled its pages is cut down to the tokens that
got the most (samd.cache_evict) into the other half of its pages. The feed-forward part is a layer of experts with 4-bit
weights (samd.moe_layer4). Beside it the same layer runs on its own keys and values in 64 bits, without the cache's lanes.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1809_10572_gb300 import samd  # noqa: E402

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
GROUP = 32


class Weights:
    """A 4-bit matrix (packed signed lanes, scales for 32 inputs), and the values it stands for."""

    def __init__(self, rows: int, cols: int, dtype, gen):
        w = torch.randn((rows, cols // GROUP, GROUP), device="cuda", generator=gen) / cols ** 0.5
        self.scales = (w.abs().amax(-1) / 7).clamp(min=torch.finfo(dtype).tiny).to(dtype)
        q = (w / self.scales.float().unsqueeze(-1)).round().clamp(-8, 7)
        self.lanes = samd.pack(q.view(rows, cols).to(torch.int8), samd.fmt(4, True)).view(rows, -1)
        self.values = (q.double() * self.scales.double().unsqueeze(-1)).view(rows, cols)

    def __call__(self, x):
        return samd.matvec4(x, self.lanes, self.scales, GROUP, samd.fmt(4, True))


class Layer:
    def __init__(self, a, dtype, gen):
        self.a, self.dtype, self.dim = a, dtype, a.width // a.heads
        kv = a.kv_heads * self.dim
        self.q, self.k, self.v = (Weights(n, a.width, dtype, gen) for n in (a.width, kv, kv))
        self.o = Weights(a.width, a.width, dtype, gen)
        hidden = a.width
        self.gate, self.up = (Weights(a.experts * hidden, a.width, dtype, gen) for _ in range(2))
        self.down = Weights(a.experts * a.width, hidden, dtype, gen)
        self.router = (torch.randn((a.experts, a.width), device="cuda", generator=gen) / a.width ** 0.5).to(dtype)
        # two sets of pages for every sequence: one in use, one to cut down into
        pages = a.budget // a.page
        self.cache = samd.cache_empty(2 * a.sequences * pages, a.page, a.kv_heads, self.dim, a.bits, dtype)
        tables = torch.randperm(2 * a.sequences * pages, device="cuda", generator=gen).to(torch.int32)
        self.table, self.spare = tables.view(2, a.sequences, pages).unbind(0)
        self.scores = torch.zeros((a.sequences, a.kv_heads, a.budget), device="cuda")

    def heads(self, x, n):
        return x.view(x.shape[0], n, self.dim)

    def keys_and_values(self, x):
        return self.heads(self.k(x), self.a.kv_heads), self.heads(self.v(x), self.a.kv_heads)

    def prompt(self, x, lengths, starts):
        samd.cache_append(self.cache, *self.keys_and_values(x), self.table, lengths, starts)

    def step(self, x, lengths):
        """One token of every sequence; lengths counts it. Returns the layer's output, and the attention's."""
        samd.cache_append(self.cache, *self.keys_and_values(x), self.table, lengths)
        att = samd.paged_attention(self.heads(self.q(x), self.a.heads), self.cache, self.table, lengths, scores=self.scores)
        h = x + self.o(att.view(x.shape[0], -1))
        y = samd.moe_layer4(h, self.router, self.a.topk, *((w.lanes, w.scales) for w in (self.gate, self.up, self.down)), GROUP,
                            samd.fmt(4, True))
        return h + y, att

    def cut(self, lengths):
        """Cuts the sequences down. Returns the kept tokens' places and the new lengths."""
        kept, lengths, scores = samd.cache_evict(self.cache, self.table, lengths, self.scores, self.spare, self.a.keep, self.a.recent)
        self.scores.zero_()
        self.scores[..., :self.a.keep] = scores
        self.table, self.spare = self.spare, self.table
        return kept, lengths


def main(argv=None) -> dict:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("width", 512), ("heads", 8), ("kv-heads", 2), ("experts", 8), ("topk", 2), ("sequences", 4), ("tokens", 200),
                          ("page", 16), ("budget", 128), ("keep", 64), ("recent", 16), ("bits", 4)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--type", choices=sorted(TYPES), default="bf16")
    a = ap.parse_args(argv)
    dtype = TYPES[a.type]
    gen = torch.Generator(device="cuda").manual_seed(1)
    layer = Layer(a, dtype, gen)
    new = [a.budget // 2 // (1 + i) for i in range(a.sequences)]  # prompts of different lengths
    lengths = torch.tensor(new, dtype=torch.int32, device="cuda")
    starts = torch.tensor([sum(new[:i]) for i in range(a.sequences + 1)], dtype=torch.int32, device="cuda")
    x = torch.randn((sum(new), a.width), device="cuda", generator=gen).to(dtype)
    layer.prompt(x, lengths, starts)
    # beside it: each key head's own list of keys and values, as they were before they became lanes
    k, v = layer.keys_and_values(x)
    book = [[[t[starts[b]:starts[b + 1], h].double() for t in (k, v)] for h in range(a.kv_heads)] for b in range(a.sequences)]
    x = torch.randn((a.sequences, a.width), device="cuda", generator=gen).to(dtype)
    worst, cuts = 0.0, 0
    for _ in range(a.tokens):
        lengths = lengths + 1
        k, v = layer.keys_and_values(x)
        q = layer.heads(layer.q(x), a.heads).double()
        y, att = layer.step(x, lengths)
        want = torch.empty(att.shape, dtype=torch.float64, device="cuda")
        group = a.heads // a.kv_heads
        for b in range(a.sequences):
            for h in range(a.kv_heads):
                rows = book[b][h] = [torch.cat((old, t[b, h].double()[None])) for old, t in zip(book[b][h], (k, v))]
                p = torch.softmax(q[b, h * group:(h + 1) * group] @ rows[0].t() * layer.dim ** -0.5, -1)
                want[b, h * group:(h + 1) * group] = p @ rows[1]
        worst = max(worst, float((att.double() - want).norm() / want.norm()))
        # the next token: this one's output, at the size that a norm would give it
        x = (y.float() / y.float().square().mean(-1, keepdim=True).sqrt()).to(dtype)
        if int(lengths.max()) == a.budget:
            kept, lengths = layer.cut(lengths)
            cuts += 1
            for b in range(a.sequences):
                n = int(lengths[b])
                for h in range(a.kv_heads):
                    book[b][h] = [t[kept[b, h, :n].long()] for t in book[b][h]]
    finite = bool(torch.isfinite(x).all())
    print(f"{a.tokens} tokens of {a.sequences} sequences, cut down {cuts} times; attention over {a.bits}-bit lanes is "
          f"{100 * worst:.1f}% from that over the values at most")
    return {"worst": worst, "cuts": cuts, "finite": finite, "lengths": lengths.tolist(), "status": samd.samd_device_status()}


if __name__ == "__main__":
    main()
