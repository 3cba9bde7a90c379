"""The gated block's operators in plain 64-bit torch, from their definitions, and
the inputs that their tests share. Nothing here calls the library."""
import math

import torch

UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}  # half an ulp at 1
TINY = 2.0 ** -25  # half of fp16's smallest step


def ints(seed, shape, lo, hi, dtype=torch.float64, device="cuda"):
    g = torch.Generator(device="cpu").manual_seed(seed)
    return torch.randint(lo, hi + 1, shape, generator=g).to(device=device, dtype=dtype)


def normal(seed, shape, dtype, scale=1.0, device="cuda"):
    g = torch.Generator(device="cpu").manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(device=device, dtype=dtype)


def wide(t, extra=8, fill=float("nan")):
    """The same matrix inside wider rows (16-byte units apart) filled with `fill`."""
    rows, cols = t.shape
    ld = -(-cols // 8) * 8 + extra
    out = torch.full((rows, ld), fill, dtype=t.dtype, device=t.device)
    out[:, :cols] = t
    return out[:, :cols]


def pack4(q, word_bits=32):
    """Rows of lane values (-8 .. 15) as samd_pack lays them out."""
    rows, K = q.shape
    L = word_bits // 4
    words = -(-K // L)
    p = torch.zeros((rows, words * L), dtype=torch.int64, device=q.device)
    p[:, :K] = q.long() & 15
    p = p.view(rows, words * L // 2, 2)
    b = (p[:, :, 0] | p[:, :, 1] << 4).to(torch.uint8)
    return b.view(torch.int32 if word_bits == 32 else torch.int64).view(rows, words)


def weights4(q, scales, zeros, group):
    """scale * (q - zero) in 64 bits."""
    K = q.shape[1]
    v = q.double()
    if zeros is not None:
        v = v - (zeros.double() % 16).repeat_interleave(group, 1)[:, :K]
    return v * scales.double().repeat_interleave(group, 1)[:, :K]


def act(g, name):
    if name == "silu":
        return g * torch.sigmoid(g)
    if name == "gelu":
        return g * torch.special.ndtr(g)
    if name == "gelu_tanh":
        return 0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))
    return torch.clamp(g, min=0)


def act_grad(g, name):
    if name == "silu":
        s = torch.sigmoid(g)
        return s * (1 + g * (1 - s))
    if name == "gelu":
        return torch.special.ndtr(g) + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        th = torch.tanh(c * (g + 0.044715 * g ** 3))
        return 0.5 * (1 + th) + 0.5 * g * (1 - th * th) * c * (1 + 3 * 0.044715 * g * g)
    return (g > 0).double()


def block8(x, keep=False):
    """(codes, exponents, values) of the 8-bit form of a matrix; values in 64 bits, NaN where the block is. keep: a
    positive value's code is at least 1 (what the forward pass keeps of a ReLU's argument)."""
    rows, inner = x.shape
    n = -(-inner // 32)
    v = torch.zeros((rows, n * 32), dtype=torch.float64, device=x.device)
    v[:, :inner] = x.double()
    v = v.view(rows, n, 32)
    bad = ~torch.isfinite(v).all(-1, keepdim=True)
    fine = torch.where(bad, torch.zeros_like(v), v)
    # the exponent of the largest magnitude as fp32 holds it (all inputs are fp32 or narrower)
    bits = fine.abs().amax(-1, keepdim=True).float().view(torch.int32)
    e = ((bits >> 23) - 6).clamp(min=0)
    step = ((e.long() + (1023 - 127)) << 52).view(torch.float64)  # 2^(e - 127); a library's pow may be an ulp off
    codes = torch.round(fine / step).clamp(-127, 127)
    if keep:
        codes = torch.where((fine > 0) & (codes == 0), torch.ones_like(codes), codes)
    values = torch.where(bad, torch.full_like(v, float("nan")), codes * step)
    e = torch.where(bad, torch.full_like(e, 255), e)
    return (codes.view(rows, n * 32)[:, :inner].to(torch.int8), e.view(rows, n).to(torch.uint8),
            values.view(rows, n * 32)[:, :inner])


def pack8(codes):
    """Rows of int8 codes as 32-bit words of four lanes."""
    rows, inner = codes.shape
    words = -(-inner // 4)
    p = torch.zeros((rows, words * 4), dtype=torch.int8, device=codes.device)
    p[:, :inner] = codes
    return p.view(torch.int32).view(rows, words)
