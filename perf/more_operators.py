"""Decoding with a language model's layer on packed lanes, as measurable cases.

The key-value cache in 4- or 8-bit lanes, in pages: writing tokens into it and
reading them back (samd.cache_append / cache_read), attention of one new token
for each sequence (samd.paged_attention), evicting the tokens that got the
least weight (samd.cache_evict). And the sparse form of the gated block: a whole
layer of experts with 4-bit weights for a few tokens (samd.moe_layer4).

With `own` false a case runs in its plain form, elementary torch operations in
32 bits; with `own` true it runs through the library's public binding.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
BLOCK = 32  # elements of a cached row that share a scale


# ---- the cases -----------------------------------------------------------------


def listed():
    return [
        # a decoding step's new tokens into the cache and back: the smallest call, latency counts
        dict(name="append_16", kind="append", seqs=16, most=2048, new=1, heads=8, dim=128, bits=8, page=16, type="bf16"),
        # prompts of ragged lengths behind what their sequences hold already
        dict(name="append_prompts", kind="append", seqs=7, most=9000, new=3001, heads=8, dim=128, bits=4, page=64,
             type="f16"),
        # one short sequence, as many key heads as query heads
        dict(name="att_1x100", kind="attention", seqs=1, most=100, q_heads=8, heads=8, dim=64, bits=8, page=16,
             scores=False, type="bf16"),
        # a batch of ragged lengths, four query heads to a key head
        dict(name="att_16x8192", kind="attention", seqs=16, most=8192, q_heads=32, heads=8, dim=128, bits=8, page=16,
             scores=False, type="bf16"),
        # one very long sequence: its length has to be split
        dict(name="att_1x131072", kind="attention", seqs=1, most=131072, q_heads=64, heads=8, dim=128, bits=4, page=64,
             scores=False, type="f16"),
        # many sequences, empty ones among them, an odd head size
        dict(name="att_53x4001", kind="attention", seqs=53, most=4001, q_heads=12, heads=12, dim=96, bits=8, page=32,
             scores=False, type="f16"),
        # the step that also counts the weights, for evicting
        dict(name="att_scores_8x16000", kind="attention", seqs=8, most=16000, q_heads=28, heads=4, dim=128, bits=4,
             page=16, scores=True, type="bf16"),
        # a small cache cut down
        dict(name="evict_2x600", kind="evict", seqs=2, most=600, keep=256, recent=64, heads=4, dim=64, bits=8, page=16,
             type="bf16"),
        # and a large one, of ragged lengths
        dict(name="evict_16x8192", kind="evict", seqs=16, most=8192, keep=2048, recent=200, heads=8, dim=128, bits=8,
             page=32, type="f16"),
        # one token through a small layer of experts
        dict(name="moe_1x1024x512", kind="moe", M=1, K=1024, F=512, E=32, topk=4, G=32, zeros=False, act="silu",
             type="bf16"),
        # and a large one
        dict(name="moe_1x4096x8192", kind="moe", M=1, K=4096, F=8192, E=8, topk=2, G=128, zeros=False, act="silu",
             type="bf16"),
        # a batch that reaches most of many experts, weights with zero points
        dict(name="moe_13x2048x1408", kind="moe", M=13, K=2048, F=1408, E=64, topk=6, G=64, zeros=True, act="gelu",
             type="f16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attention", "attention", "evict", "moe", "moe"])
    c = dict(kind=kind)
    if kind == "moe":
        while True:
            c |= dict(M=_log(rng, 1, 32), K=32 * _log(rng, 8, 128), F=32 * _log(rng, 8, 256), E=_log(rng, 4, 128))
            c |= dict(topk=rng.randint(1, min(8, c["E"])), G=rng.choice([32, 64, 128]), zeros=rng.random() < 0.3)
            c |= dict(act=rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu"]), type=rng.choice(["bf16", "f16"]))
            if c["E"] * c["K"] * c["F"] <= 1 << 28 and work(c)["bytes"] < 1.5e8:
                return c
    while True:
        heads = rng.choice([1, 2, 4, 5, 8, 12])
        c |= dict(seqs=_log(rng, 1, 100), most=_log(rng, 1, 100000), heads=heads,
                  dim=rng.choice([64, 128, 128, 32 * rng.randint(1, 8)]), bits=rng.choice([4, 8]),
                  page=rng.choice([16, 16, 32, 64, 128]), type=rng.choice(["bf16", "f16"]))
        if kind == "append":
            c["new"] = 1 if rng.random() < 0.5 else _log(rng, 1, c["most"])
        elif kind == "attention":
            c |= dict(q_heads=heads * rng.choice([1, 1, 2, 4, 7, 8, 12]), scores=rng.random() < 0.3)
        else:
            c["keep"] = _log(rng, 1, c["most"])
            c["recent"] = rng.randint(0, c["keep"])
        if work(c)["bytes"] < 1.5e8 and c["seqs"] * c["most"] * heads * c["dim"] < 3e8:
            return c


def _lengths(c):
    """Ragged lengths of the sequences: the first is the longest, every eleventh is empty (a padded batch)."""
    n = [max(1, int(c["most"] * ((i * 0.618033988749895) % 1.0))) for i in range(c["seqs"])]
    return [c["most"]] + [0 if i % 11 == 7 else n[i] for i in range(1, c["seqs"])]


def _new(c):
    """How many of each sequence's tokens are new: at most `new`, spread as the lengths are."""
    part = [int(c["new"] * ((0.5 + i * 0.7548776662466927) % 1.0)) for i in range(c["seqs"])]
    return [min(n, 1 if c["new"] == 1 else max(1, part[i])) for i, n in enumerate(_lengths(c))]


def work(c):
    if c["kind"] == "moe":
        M, K, F = c["M"], c["K"], c["F"]
        experts = c["E"] * (1 - (1 - c["topk"] / c["E"]) ** M)  # that at least one token reaches
        per = 3 if c["zeros"] else 2
        row = lambda n: n // 2 + -(-n // c["G"]) * per  # noqa: E731
        weights = experts * (2 * F * row(K) + K * row(F))
        return {"bytes": weights + 2 * c["E"] * K + 4 * M * K, "flops": 6 * M * c["topk"] * K * F + 2 * M * c["E"] * K}
    row = c["dim"] * c["bits"] // 8 + c["dim"] // BLOCK * 2  # a cached key or value
    tokens = sum(_lengths(c))
    if c["kind"] == "append":  # rows in, into the cache, out of it and back
        return {"bytes": 2 * c["heads"] * sum(_new(c)) * (4 * c["dim"] + 2 * row), "flops": 0}
    if c["kind"] == "attention":
        b = 2 * c["heads"] * tokens * row + 4 * c["seqs"] * c["q_heads"] * c["dim"]
        return {"bytes": b + (8 * c["heads"] * tokens if c["scores"] else 0),
                "flops": 4 * c["q_heads"] * tokens * c["dim"]}
    kept = sum(min(n, c["keep"]) for n in _lengths(c))
    return {"bytes": c["heads"] * (4 * tokens + kept * (4 * row + 8)), "flops": 0}


# ---- inputs --------------------------------------------------------------------


def _gen(seed, k):
    return torch.Generator(device=DEV).manual_seed((int(seed) * 1000003 + 7919 * k) & 0x7FFFFFFF)


def _tokens(seed, k, shape, t):
    """Activations: normal values, with a few channels that are much larger, as trained models have them."""
    x = torch.randn(shape, device=DEV, generator=_gen(seed, k))
    big = torch.rand(shape[-1], device=DEV, generator=_gen(seed, k + 1)) < 0.01
    return (x * (1 + 15 * big)).to(t)


def _lanes4(seed, k, rows, width, zeros):
    """4-bit lanes of normally distributed weights, packed as samd_pack writes them."""
    v = torch.empty((rows, width), dtype=torch.half, device=DEV).normal_(0, 2.6, generator=_gen(seed, k))
    q = v.round_().clamp_(-8, 7).add_(8 if zeros else 0).to(torch.int8).view(rows, width // 2, 2) & 15
    return (q[:, :, 0] | (q[:, :, 1] << 4)).view(torch.int32).reshape(rows, width // 8)


def _weights4(seed, k, c, rows, width):
    """E matrices one behind the other: lanes, scales, zero points."""
    n, groups = c["E"] * rows, -(-width // c["G"])
    s = (0.5 + torch.rand((n, groups), device=DEV, generator=_gen(seed, k + 1))).mul_(0.4 / math.sqrt(width))
    z = torch.randint(5, 11, (n, groups), dtype=torch.uint8, device=DEV, generator=_gen(seed, k + 2))
    return {"q": _lanes4(seed, k, n, width, c["zeros"]), "s": s.to(TYPES[c["type"]]), "z": z if c["zeros"] else None}


def _cache(seed, c, pages):
    """Pages of cached rows: lanes of normally distributed values, scales that differ between blocks."""
    words, shape = c["dim"] * c["bits"] // 32, (pages, c["heads"], c["page"])
    out = {}
    for i, name in enumerate(("k", "v")):
        if c["bits"] == 4:
            lanes = _lanes4(seed, 40 + 10 * i, math.prod(shape), c["dim"], False)
        else:
            lanes = torch.empty((math.prod(shape), c["dim"]), dtype=torch.half, device=DEV)
            lanes = lanes.normal_(0, 42, generator=_gen(seed, 40 + 10 * i)).round_().clamp_(-127, 127).to(torch.int8)
            lanes = lanes.view(torch.int32)
        s = torch.rand((*shape, c["dim"] // BLOCK), device=DEV, generator=_gen(seed, 41 + 10 * i))
        out[name] = lanes.view(*shape, words)
        out[name + "s"] = s.add_(0.5).mul_(1 / (42 if c["bits"] == 8 else 2.6)).to(TYPES[c["type"]])
    return out


def prepare(c, seed):
    t = TYPES[c["type"]]
    s = {"c": c}
    if c["kind"] == "moe":
        M, K, F = c["M"], c["K"], c["F"]
        s["x"] = _tokens(seed, 0, (M, K), t)
        s["router"] = torch.randn((c["E"], K), device=DEV, generator=_gen(seed, 5)).mul_(1 / math.sqrt(K)).to(t)
        s["gate"], s["up"] = _weights4(seed, 10, c, F, K), _weights4(seed, 20, c, F, K)
        s["down"] = _weights4(seed, 30, c, K, F)
        return s
    # the sequences' pages, anywhere in the cache, and for evicting as many as are wanted behind them
    n = _lengths(c)
    width = max(1, -(-c["most"] // c["page"]))
    more = -(-c["keep"] // c["page"]) if c["kind"] == "evict" else 0
    pages = c["seqs"] * (width + more)
    order = torch.randperm(pages, device=DEV, generator=_gen(seed, 1)).to(torch.int32)
    s["table"] = order[:c["seqs"] * width].view(c["seqs"], width)
    s["lengths"] = torch.tensor(n, dtype=torch.int32, device=DEV)
    s["cache"] = _cache(seed, c, pages)
    if c["kind"] == "append":
        rows = _new(c)
        s["starts"] = torch.tensor([sum(rows[:i]) for i in range(c["seqs"] + 1)], dtype=torch.int32, device=DEV)
        s["k"], s["v"] = (_tokens(seed, 10 * i, (sum(rows), c["heads"], c["dim"]), t) for i in (2, 3))
    elif c["kind"] == "attention":
        s["q"] = _tokens(seed, 20, (c["seqs"], c["q_heads"], c["dim"]), t)
        s["scores"] = torch.rand((c["seqs"], c["heads"], c["most"]), device=DEV, generator=_gen(seed, 2)) \
            if c["scores"] else None
    else:
        s["dst"] = order[c["seqs"] * width:].view(c["seqs"], more)
        # weights that some tokens gather most of, and many that never got any
        w = torch.rand((c["seqs"], c["heads"], c["most"]), device=DEV, generator=_gen(seed, 2))
        s["scores"] = torch.exp(8 * w).mul_(0.01) * (w > 0.2)
    return s


# ---- one pass ------------------------------------------------------------------


def _plain_values(lanes, scales, bits):
    """Of rows of packed signed lanes, in 32 bits."""
    v = lanes.unsqueeze(-1) >> torch.arange(0, 32, bits, dtype=torch.int32, device=DEV)
    half = 1 << (bits - 1)
    v = ((v & (2 * half - 1)) ^ half) - half
    rows = v.shape[:-2]
    return (v.reshape(*rows, -1, BLOCK).float() * scales.float().unsqueeze(-1)).view(*rows, -1)


def _plain_append(s):
    """What the cache holds of the rows."""
    c, t = s["c"], TYPES[s["c"]["type"]]
    most = 127 if c["bits"] == 8 else 7
    x = torch.stack((s["k"], s["v"])).float()
    x = x.view(*x.shape[:-1], -1, BLOCK)
    scale = (x.abs().amax(-1, keepdim=True) / most).to(t).float()
    lanes = torch.where(scale > 0, (x / scale).round().clamp(-most, most), torch.zeros_like(x))
    k, v = (lanes * scale).view(2, *s["k"].shape).to(t)
    return {"k": k, "v": v}


def _plain_attention(s):
    c, t = s["c"], TYPES[s["c"]["type"]]
    pages = s["table"].long()
    q = s["q"].float().view(c["seqs"], c["heads"], -1, c["dim"])
    span = pages.shape[1] * c["page"]

    def rows(name):  # (sequence, head, token, element)
        x = _plain_values(s["cache"][name][pages], s["cache"][name + "s"][pages], c["bits"])
        return x.transpose(1, 2).reshape(c["seqs"], c["heads"], span, c["dim"])

    logits = q @ rows("k").transpose(2, 3) * (1 / math.sqrt(c["dim"]))
    there = (torch.arange(span, device=DEV) < s["lengths"].unsqueeze(1))[:, None, None]
    logits = torch.where(there, logits, torch.full_like(logits, -3e38))
    p = torch.exp(logits - logits.amax(-1, keepdim=True)) * there
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-30)
    out = (p @ rows("v")).view(c["seqs"], c["q_heads"], c["dim"]).to(t)
    if not c["scores"]:
        return out
    s["scores"] += p.sum(2)[:, :, :c["most"]]
    return {"out": out, "scores": s["scores"]}


def _plain_evict(s):
    c, cache, keep = s["c"], s["cache"], s["c"]["keep"]
    at = torch.arange(c["most"], device=DEV)
    n = s["lengths"][:, None, None]
    rank = torch.where(at >= n - c["recent"], torch.full_like(s["scores"], math.inf), s["scores"])
    rank = torch.where(at < n, rank, torch.full_like(rank, -math.inf))
    first = rank.sort(dim=-1, descending=True, stable=True).indices[..., :keep]
    first = torch.where(torch.arange(keep, device=DEV) < n, first, c["most"]).sort(dim=-1).values
    there = first < c["most"]
    at = torch.where(there, first, 0)
    seq = torch.arange(c["seqs"], device=DEV)[:, None, None]
    head = torch.arange(c["heads"], device=DEV)[None, :, None]
    src, to = s["table"].long()[seq, at // c["page"]], torch.arange(keep, device=DEV)
    dst = s["dst"].long()[seq, to // c["page"]]
    cache["k"][dst, head, to % c["page"]] = torch.where(there.unsqueeze(-1), cache["k"][src, head, at % c["page"]],
                                                        cache["k"][dst, head, to % c["page"]])
    cache["v"][dst, head, to % c["page"]] = torch.where(there.unsqueeze(-1), cache["v"][src, head, at % c["page"]],
                                                        cache["v"][dst, head, to % c["page"]])
    cache["ks"][dst, head, to % c["page"]] = torch.where(there.unsqueeze(-1), cache["ks"][src, head, at % c["page"]],
                                                         cache["ks"][dst, head, to % c["page"]])
    cache["vs"][dst, head, to % c["page"]] = torch.where(there.unsqueeze(-1), cache["vs"][src, head, at % c["page"]],
                                                         cache["vs"][dst, head, to % c["page"]])
    return {"kept": torch.where(there, first, -1).int(), "lengths": s["lengths"].clamp(max=keep),
            "scores": torch.where(there, s["scores"].gather(2, at), 0.0), "cache": cache}


def _plain_weights(w, c, rows):
    """(q - z) * s of every weight, in 32 bits: (expert, row, input)."""
    q = (w["q"].unsqueeze(-1) >> torch.arange(0, 32, 4, dtype=torch.int32, device=DEV)) & 15
    q = q.view(w["q"].shape[0], -1).float()
    groups = torch.arange(q.shape[1], device=DEV) // c["G"]
    if w["z"] is None:
        q = q - 16 * (q >= 8).float()
    else:
        q = q - w["z"].float()[:, groups]
    return (q * w["s"].float()[:, groups]).view(c["E"], rows, -1)


def _plain_act(g, act):
    if act == "silu":
        return g / (1 + torch.exp(-g))
    if act == "gelu":
        return g * (0.5 * (1 + torch.erf(g * math.sqrt(0.5))))
    if act == "gelu_tanh":
        return g * (0.5 * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g * g * g))))
    return g * (g > 0).float()


def _plain_moe(s):
    """Every expert for every token; those that a token did not choose count nothing."""
    c, x = s["c"], s["x"].float()
    logits = s["x"].double() @ s["router"].double().t()  # which expert is the larger is decided in 64 bits
    top = logits.sort(dim=-1, descending=True, stable=True)
    w = torch.exp(top.values[:, :c["topk"]] - top.values[:, :1])
    share = torch.zeros_like(logits).scatter_(1, top.indices[:, :c["topk"]], w / w.sum(-1, keepdim=True)).float()
    g = x @ _plain_weights(s["gate"], c, c["F"]).transpose(1, 2)  # (expert, token, hidden column)
    u = x @ _plain_weights(s["up"], c, c["F"]).transpose(1, 2)
    h = _plain_act(g, c["act"]) * u * share.t().unsqueeze(-1)
    return (h @ _plain_weights(s["down"], c, c["K"]).transpose(1, 2)).sum(0).to(TYPES[c["type"]])


def _plain(s):
    return {"append": _plain_append, "attention": _plain_attention, "evict": _plain_evict,
            "moe": _plain_moe}[s["c"]["kind"]](s)


def _library(s):
    from paper_1809_10572_gb300 import samd

    c = s["c"]
    if c["kind"] == "moe":
        gate, up, down = ((w["q"], w["s"], w["z"]) for w in (s["gate"], s["up"], s["down"]))
        return samd.moe_layer4(s["x"], s["router"], c["topk"], gate, up, down, c["G"], samd.fmt(4, not c["zeros"]),
                               c["act"])
    b = s["cache"]
    cache = samd.PagedCache(b["k"], b["ks"], b["v"], b["vs"])
    if c["kind"] == "append":
        samd.cache_append(cache, s["k"], s["v"], s["table"], s["lengths"], s["starts"])
        k, v = samd.cache_read(cache, s["k"].shape[0], s["table"], s["lengths"], s["starts"])
        return {"k": k, "v": v}
    if c["kind"] == "attention":
        out = samd.paged_attention(s["q"], cache, s["table"], s["lengths"], scores=s["scores"])
        return {"out": out, "scores": s["scores"]} if c["scores"] else out
    kept, lengths, scores = samd.cache_evict(cache, s["table"], s["lengths"], s["scores"], s["dst"], c["keep"],
                                             c["recent"])
    return {"kept": kept, "lengths": lengths, "scores": scores, "cache": b}


def run(state):
    return _library(state) if own else _plain(state)


# ---- the same from the definitions, in 64 bits ----------------------------------


def _exact_bytes(lanes, bits):
    """Lanes as whole numbers: a byte holds one of eight bits or two of four, the lower one first."""
    b = lanes.contiguous().view(torch.int8)
    if bits == 8:
        return b.double()
    lo = torch.remainder(b.int(), 16)
    return torch.stack((lo - 16 * (lo > 7), (b.int() - lo) // 16), -1).flatten(-2).double()


def _exact_append(s):
    c, t = s["c"], TYPES[s["c"]["type"]]
    top, out = 2 ** (c["bits"] - 1) - 1, {}
    for name in ("k", "v"):
        x = s[name].double().unflatten(-1, (-1, BLOCK))
        scale = (x.abs().max(-1, keepdim=True).values / top).to(t).double()
        ratio = torch.nan_to_num(x / scale, nan=0.0)
        out[name] = (torch.round(ratio).clamp(-top, top) * scale).flatten(-2)
    return out


def _exact_attention(s):
    c, cache = s["c"], s["cache"]
    group, out = c["q_heads"] // c["heads"], torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    scores = s["scores"].double() if c["scores"] else None
    for b, n in enumerate(_lengths(c)):
        if n == 0:
            continue
        token = torch.arange(n, device=DEV)
        page, slot = s["table"][b, token // c["page"]].long(), token % c["page"]

        def rows(name):  # (token, head, element)
            x = _exact_bytes(cache[name][page, :, slot], c["bits"])
            return x * cache[name + "s"][page, :, slot].double().repeat_interleave(BLOCK, -1)

        q = s["q"][b].double().view(c["heads"], group, c["dim"])
        p = torch.softmax(torch.einsum("hgd,thd->hgt", q, rows("k")) / c["dim"] ** 0.5, -1)
        out[b] = torch.einsum("hgt,thd->hgd", p, rows("v")).reshape(c["q_heads"], c["dim"])
        if scores is not None:
            scores[b, :, :n] += p.sum(1)
    return out if scores is None else {"out": out, "scores": scores}


def _exact_evict(s):
    """Each head's kept tokens by a sort over (weight, place)."""
    c, keep = s["c"], s["c"]["keep"]
    scores = torch.zeros((c["seqs"], c["heads"], keep), dtype=torch.float64, device=DEV)
    kept = torch.full(scores.shape, -1, dtype=torch.int32, device=DEV)
    cache = {name: v.clone() for name, v in s["cache"].items()}
    for b, n in enumerate(_lengths(c)):
        if n == 0:
            continue
        w = s["scores"][b, :, :n].tolist()
        count, last = min(n, keep), min(c["recent"], n)
        for h in range(c["heads"]):
            old = sorted(range(n - last), key=lambda i: (-w[h][i], i)) if n > keep else list(range(n - last))
            chosen = sorted(old[:count - last] + list(range(n - last, n)))
            at = torch.tensor(chosen, device=DEV)
            to = torch.arange(count, device=DEV)
            kept[b, h, :count] = at.int()
            scores[b, h, :count] = s["scores"][b, h, at].double()
            src, dst = s["table"][b, at // c["page"]].long(), s["dst"][b, to // c["page"]].long()
            for v in cache.values():
                v[dst, h, to % c["page"]] = v[src, h, at % c["page"]]
    return {"kept": kept, "lengths": torch.tensor([min(n, keep) for n in _lengths(c)], dtype=torch.int32), "scores": scores,
            "cache": {name: v.double() if v.is_floating_point() else v for name, v in cache.items()}}


def _exact_weights(w, c, rows, e):
    """Expert e's matrix: the bytes of the packed words hold two lanes each, the lower one first."""
    b = w["q"].view(c["E"], rows, -1)[e].contiguous().view(torch.uint8)
    q = torch.stack((b % 16, b // 16), -1).flatten(-2).double()
    if w["z"] is None:
        q = torch.where(q > 7, q - 16, q)
    else:
        q -= w["z"].view(c["E"], rows, -1)[e].double().repeat_interleave(c["G"], 1)[:, :q.shape[1]]
    return q * w["s"].view(c["E"], rows, -1)[e].double().repeat_interleave(c["G"], 1)[:, :q.shape[1]]


def _exact_act(g, act):
    if act == "silu":
        return g * torch.sigmoid(g)
    if act == "gelu":
        return g * torch.special.ndtr(g)
    if act == "gelu_tanh":  # 0.5 (1 + tanh a) = sigmoid(2 a)
        return g * torch.sigmoid(math.sqrt(8 / math.pi) * (g + 0.044715 * g ** 3))
    return torch.clamp(g, min=0)


def _exact_moe(s):
    """Expert by expert, for the tokens that chose it."""
    c, x = s["c"], s["x"].double()
    logits = torch.einsum("mk,ek->me", x, s["router"].double()).tolist()
    y = torch.zeros_like(x)
    chosen = [sorted(range(c["E"]), key=lambda e: (-row[e], e))[:c["topk"]] for row in logits]
    weight = [torch.softmax(torch.tensor([row[e] for e in idx], dtype=torch.float64), 0) for row, idx in zip(logits, chosen)]
    for e in range(c["E"]):
        who = [(m, float(weight[m][idx.index(e)])) for m, idx in enumerate(chosen) if e in idx]
        if who:
            at, w = torch.tensor([m for m, _ in who], device=DEV), torch.tensor([v for _, v in who], dtype=torch.float64, device=DEV)
            g, u = (x[at] @ _exact_weights(s[name], c, c["F"], e).t() for name in ("gate", "up"))
            y[at] += w[:, None] * ((_exact_act(g, c["act"]) * u) @ _exact_weights(s["down"], c, c["K"], e).t())
    return y


def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] == "evict" and c["seqs"] * c["heads"] * c["most"] > 2_000_000:
        return None
    return {"append": _exact_append, "attention": _exact_attention, "evict": _exact_evict, "moe": _exact_moe}[c["kind"]](s)
