"""The packed cache and its operators in plain 64-bit torch, from their definitions, and the inputs their tests share.
Nothing here calls the library."""
import math

import torch

UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}  # half an ulp at 1
BLOCK = 32


def gen(seed):
    return torch.Generator(device="cpu").manual_seed(seed)


def normal(seed, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen(seed)) * scale).to(device="cuda", dtype=dtype)


def ints(seed, shape, lo, hi, dtype=torch.int64):
    return torch.randint(lo, hi + 1, shape, generator=gen(seed)).to(device="cuda", dtype=dtype)


def pack(lanes, bits):
    """Rows of lanes (..., dim) as 32-bit words (..., dim * bits / 32), the first lane lowest."""
    if bits == 8:
        return lanes.to(torch.int8).contiguous().view(torch.int32)
    n = (lanes.to(torch.int16) & 15).view(*lanes.shape[:-1], -1, 2)
    return (n[..., 0] | n[..., 1] << 4).to(torch.uint8).contiguous().view(torch.int32)


def unpack(words, bits):
    b = words.contiguous().view(torch.int8)
    if bits == 8:
        return b.long()
    lo = b.long() & 15
    return torch.stack((lo - 16 * (lo > 7), (b.long() >> 4)), -1).flatten(-2)


def quantize(x, bits):
    """(lanes, scales) of rows (..., dim) of a 16-bit type."""
    most = 2 ** (bits - 1) - 1
    v = x.double().unflatten(-1, (-1, BLOCK))
    fine = torch.isfinite(v).all(-1)
    top = torch.where(fine, torch.nan_to_num(v).abs().amax(-1), torch.zeros_like(v[..., 0]))
    # (the quotient in fp32 and from there to the type, as the definition rounds it once: a value of 8 or 11 bits by 7 or
    # 127 is never so near to the middle of two of the type's values that the rounding to 24 bits between changes it)
    s = (top.float() / most).to(x.dtype)
    ratio = torch.where((s > 0)[..., None], v / s.double()[..., None], torch.zeros_like(v))
    lanes = torch.where(fine[..., None], torch.round(torch.nan_to_num(ratio)).clamp(-most, most), torch.zeros_like(v))
    return lanes.flatten(-2).long(), torch.where(fine, s, torch.full_like(s, math.nan))


def values(lanes, scales):
    """lane * scale in 64 bits."""
    return lanes.double() * scales.double().repeat_interleave(BLOCK, -1)


def random_rows(seed, shape, dim, bits, t, spread=1.0):
    """Lanes over their whole range, and scales that differ by a power of two or so (2^spread)."""
    most = 2 ** (bits - 1) - 1
    lanes = ints(seed, (*shape, dim), -most - 1, most)
    s = torch.exp2(spread * torch.rand((*shape, dim // BLOCK), generator=gen(seed + 1))) / most
    return lanes, s.to(device="cuda", dtype=t)


def pages_for(seed, seqs, width, more=0):
    """A table of distinct pages in any order, and how many pages there are."""
    n = seqs * width + more
    return torch.randperm(max(n, 1), generator=gen(seed))[:seqs * width].view(seqs, width).to("cuda", torch.int32), max(n, 1)


def gather(paged, table, b, n, page):
    """Rows of the first n tokens of sequence b: (heads, n, ...)."""
    t = torch.arange(n, device="cuda")
    return paged[table[b, t // page].long(), :, t % page].transpose(0, 1)


def attention(q, k, v, scale):
    """One sequence: q (q_heads, dim), k and v (heads, tokens, dim) in 64 bits. (out, weights (q_heads, tokens), logits)."""
    group = q.shape[0] // k.shape[0]
    k, v = k.repeat_interleave(group, 0), v.repeat_interleave(group, 0)
    x = torch.einsum("hd,htd->ht", q.double(), k) * scale
    p = torch.softmax(x, -1)
    return torch.einsum("ht,htd->hd", p, v), p, x


def attention_bound(q, k, v, scale, p, x, want, t):
    """How far out may be from `want`. A logit in units of log2: 33 products of a block of 32 summed in fp32 by two MMAs
    and a scaled addition for each block, 2^-23 of the magnitudes each at most, so 48 * 2^-23 of all magnitudes; the
    difference to the reference, 2^-24 of what it is taken from; ex2 2^-22. A weight's error counts in the sum of weights
    too. A weight times its scale is rounded to fp16 (2^-11); those below 2^-30 of the largest to 2^-31 of it. Sums over n
    tokens: an MMA for 16 of them, 2^-23 each."""
    group = q.shape[0] // k.shape[0]
    mags = torch.einsum("hd,htd->ht", q.double().abs(), k.abs().repeat_interleave(group, 0)).amax(-1) * abs(scale) * 1.4427
    span = (x.abs().amax(-1) * 1.4427 + 110)
    delta = (0.6932 * (48 * 2.0 ** -23 * mags + span * 2.0 ** -23) + 2.0 ** -21)[:, None]
    n = k.shape[1]
    va = v.abs().repeat_interleave(group, 0)
    total = torch.einsum("ht,htd->hd", p, va)
    worst = (p[..., None] * va).amax((1, 2))[:, None] if n * va.shape[-1] * p.shape[0] < 1 << 24 else \
        (p * va.amax(-1)).amax(-1)[:, None]
    bound = (2.0 ** -11 + 2 * delta + (n / 16 + 64) * 2.0 ** -23) * total + n * 2.0 ** -31 * 128 * worst
    return UNIT[t] * (want.abs() + bound) + bound + 2.0 ** -25 * (t is torch.float16), delta
