"""The gated feed-forward block as a user of this library trains and serves it, as measurable cases.

Serving: matrix-vector products over 4-bit packed weights with group scales
(samd.matvec4), and the block's gate and up projections with the activation and
the product (samd.gated_matvec4). Training: activations kept in 8 bits
(samd.block8_quantize / block8_dequantize), the block's forward pass
(samd.gated_ffn_forward) and its backward pass from 8-bit checkpoints
(samd.gated_ffn_backward).

With `own` false a case runs in its plain form, elementary torch operations in
32 bits; with `own` true it runs through the library's public binding.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BLOCK = 32  # elements that share an exponent in an 8-bit checkpoint


# ---- the cases -----------------------------------------------------------------


def listed():
    return [
        # one token through a small projection: the smallest call, latency counts
        dict(name="mv_1x1024x1024", kind="matvec", M=1, N=1024, K=1024, G=32, zeros=False, type="bf16"),
        # one token through a square projection, unsigned lanes with zero points
        dict(name="mv_1x4096x4096", kind="matvec", M=1, N=4096, K=4096, G=128, zeros=True, type="f16"),
        # one token through an output head: more weights than L2 holds
        dict(name="mv_1x65536x4096", kind="matvec", M=1, N=65536, K=4096, G=64, zeros=False, type="bf16"),
        # a batch of tokens, sizes that are multiples of nothing (rows of 716 bytes, a last group of 24)
        dict(name="mv_13x4100x1432", kind="matvec", M=13, N=4100, K=1432, G=32, zeros=True, type="bf16"),
        # the block's two projections for one token
        dict(name="gmv_1x8192x2048", kind="gated_matvec", M=1, N=8192, K=2048, G=64, zeros=False, act="silu",
             type="bf16"),
        # and for a few tokens at odd sizes
        dict(name="gmv_3x5461x2000", kind="gated_matvec", M=3, N=5461, K=2000, G=128, zeros=True, act="gelu",
             type="f16"),
        # activations of a layer into their 8-bit form and back
        dict(name="ck_8192x4096", kind="ckpt", M=8192, K=4096, type="bf16"),
        # rows that end inside a block and inside a word
        dict(name="ck_777x1001", kind="ckpt", M=777, K=1001, type="f32"),
        # a short prompt through the block, no checkpoints
        dict(name="fwd_64x1024x2816", kind="forward", M=64, K=1024, F=2816, act="gelu_tanh", type="f16"),
        # a long one
        dict(name="fwd_4096x4096x8192", kind="forward", M=4096, K=4096, F=8192, act="silu", type="bf16"),
        # a training step of the block: checkpoint, forward, backward; ragged sizes
        dict(name="step_777x1000x2736", kind="step", M=777, K=1000, F=2736, act="silu", type="bf16"),
        # and a full one
        dict(name="step_8192x4096x8192", kind="step", M=8192, K=4096, F=8192, act="silu", type="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["matvec", "matvec", "gated_matvec", "ckpt", "forward", "step"])
    t = rng.choice(["bf16", "bf16", "f16"])
    act = rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu"])
    if kind in ("matvec", "gated_matvec"):
        while True:
            c = dict(kind=kind, M=_log(rng, 1, 32), N=_log(rng, 64, 65536), K=_log(rng, 64, 16384),
                     G=rng.choice([32, 64, 128]), zeros=rng.random() < 0.5, type=t)
            if rng.random() < 0.5:  # widths of layers are mostly multiples of 128
                c["N"], c["K"] = -(-c["N"] // 128) * 128, -(-c["K"] // 128) * 128
            if kind == "gated_matvec":
                c["act"] = act
            if c["N"] * c["K"] <= (1 << 28) // (2 if kind == "gated_matvec" else 1):
                return c
    if kind == "ckpt":
        while True:
            c = dict(kind=kind, M=_log(rng, 1, 16384), K=_log(rng, 64, 16384), type=rng.choice([t, "f32"]))
            if rng.random() < 0.5:
                c["K"] = -(-c["K"] // 128) * 128
            if c["M"] * c["K"] <= 1 << 25:
                return c
    while True:
        c = dict(kind=kind, M=_log(rng, 1, 8192), K=_log(rng, 128, 4096), F=_log(rng, 256, 8192), act=act, type=t)
        m = 128 if rng.random() < 0.5 else 8  # rows of whole 16-byte units
        c["K"], c["F"] = -(-c["K"] // m) * m, -(-c["F"] // m) * m
        return c


def work(c):
    M, K = c["M"], c["K"]
    e = 4 if c["type"] == "f32" else 2
    if c["kind"] in ("matvec", "gated_matvec"):
        two = 2 if c["kind"] == "gated_matvec" else 1
        weights = c["N"] * (-(-K // 8) * 4 + -(-K // c["G"]) * (3 if c["zeros"] else 2))
        return {"bytes": two * weights + M * (K + c["N"]) * e, "flops": 2 * two * M * c["N"] * K}
    if c["kind"] == "ckpt":  # the values in, codes and exponents out and in again, the values back
        return {"bytes": 2 * M * K * e + 2 * M * (-(-K // 4) * 4 + -(-K // BLOCK)), "flops": 0}
    F = c["F"]
    if c["kind"] == "forward":
        return {"bytes": e * (M * K + 2 * K * F + M * F), "flops": 4 * M * K * F}
    return {"bytes": e * (2 * M * K + 4 * K * F + 2 * M * F), "flops": 12 * M * K * F}


# ---- inputs --------------------------------------------------------------------


def _gen(seed, k):
    return torch.Generator(device=DEV).manual_seed((int(seed) * 1000003 + 7919 * k) & 0x7FFFFFFF)


def _normal(seed, k, shape, scale, t):
    return torch.randn(shape, device=DEV, generator=_gen(seed, k)).mul_(scale).to(t)


def _tokens(seed, k, rows, width, t):
    """Activations: normal values, with a few channels that are much larger, as trained models have them."""
    x = torch.randn((rows, width), device=DEV, generator=_gen(seed, k))
    big = torch.rand(width, device=DEV, generator=_gen(seed, k + 1)) < 0.01
    return (x * (1 + 15 * big)).to(t)


def _weights4(seed, k, c):
    """4-bit lanes of normally distributed weights, packed as samd_pack writes them, their scales and zero points."""
    N, K, t = c["N"], c["K"], TYPES[c["type"]]
    groups, words = -(-K // c["G"]), -(-K // 8)
    v = torch.empty((N, K), dtype=torch.half, device=DEV).normal_(0, 2.6, generator=_gen(seed, k))
    mid = 8 if c["zeros"] else 0
    q = v.round_().clamp_(-8, 7).add_(mid).to(torch.int8)
    q = torch.nn.functional.pad(q, (0, words * 8 - K)).view(N, words * 4, 2) & 15
    packed = (q[:, :, 0] | (q[:, :, 1] << 4)).view(torch.int32).reshape(N, words)
    scales = (0.5 + torch.rand((N, groups), device=DEV, generator=_gen(seed, k + 1))).mul_(0.4 / math.sqrt(K)).to(t)
    zeros = torch.randint(5, 11, (N, groups), dtype=torch.uint8, device=DEV, generator=_gen(seed, k + 2))
    return {"q": packed, "s": scales, "z": zeros if c["zeros"] else None}


def prepare(c, seed):
    t, M, K = TYPES[c["type"]], c["M"], c["K"]
    s = {"c": c, "x": _tokens(seed, 0, M, K, t)}
    if c["kind"] == "matvec":
        s["w"] = _weights4(seed, 10, c)
    elif c["kind"] == "gated_matvec":
        s["wg"], s["wu"] = _weights4(seed, 10, c), _weights4(seed, 20, c)
    elif c["kind"] in ("forward", "step"):
        s["wg"] = _normal(seed, 10, (c["F"], K), 1 / math.sqrt(K), t)
        s["wu"] = _normal(seed, 20, (c["F"], K), 1 / math.sqrt(K), t)
        if c["kind"] == "step":
            s["dh"] = _normal(seed, 30, (M, c["F"]), 0.02, t)
    return s


# ---- one pass ------------------------------------------------------------------


def _plain_weights(w, c):
    """(q - z) * s of every weight, in 32 bits."""
    N, K, G = c["N"], c["K"], c["G"]
    q = (w["q"].unsqueeze(-1) >> torch.arange(0, 32, 4, dtype=torch.int32, device=DEV)) & 15
    q = q.view(N, -1)[:, :K].float()
    groups = torch.arange(K, device=DEV) // G
    if w["z"] is None:
        q = q - 16 * (q >= 8).float()
    else:
        q = q - w["z"].float()[:, groups]
    return q * w["s"].float()[:, groups]


def _plain_act(g, act):
    if act == "silu":
        return g / (1 + torch.exp(-g))
    if act == "gelu":
        return g * (0.5 * (1 + torch.erf(g * math.sqrt(0.5))))
    if act == "gelu_tanh":
        return g * (0.5 * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g * g * g))))
    return g * (g > 0).float()


def _plain_act_grad(g, act):
    if act == "silu":
        s = 1 / (1 + torch.exp(-g))
        return s * (1 + g * (1 - s))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(g * math.sqrt(0.5))) + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    if act == "gelu_tanh":
        a = math.sqrt(2 / math.pi)
        th = torch.tanh(a * (g + 0.044715 * g * g * g))
        return 0.5 * (1 + th) + 0.5 * g * (1 - th * th) * (a * (1 + 3 * 0.044715 * g * g))
    return (g > 0).float()


def _plain_block8(x, act=None):
    """What an 8-bit checkpoint holds of x: blocks of 32 along a row with one power of two, codes of -127 .. 127.
    Under a ReLU a positive value's code is at least 1: its derivative there is not lost to rounding."""
    rows, width = x.shape
    b = torch.nn.functional.pad(x.float(), (0, -width % BLOCK)).view(rows, -1, BLOCK)
    top = torch.frexp(b.abs().amax(-1, keepdim=True)).exponent - 1  # floor(log2)
    step = ((top + (127 - 6)).clamp(min=1) << 23).view(torch.float32)  # 2^(top - 6), by its bits: exact
    codes = (b / step).round().clamp(-127, 127)
    if act == "relu":
        codes = torch.maximum(codes, (b > 0).float() + -127 * (b <= 0).float())
    return (codes * step).view(rows, -1)[:, :width]


def _plain(s):
    c = s["c"]
    t, x = TYPES[c["type"]], s["x"].float()
    if c["kind"] == "matvec":
        return (x @ _plain_weights(s["w"], c).t()).to(t)
    if c["kind"] == "gated_matvec":
        g, u = x @ _plain_weights(s["wg"], c).t(), x @ _plain_weights(s["wu"], c).t()
        return (_plain_act(g, c["act"]) * u).to(t)
    if c["kind"] == "ckpt":
        return _plain_block8(x).to(t)
    wg, wu = s["wg"].float(), s["wu"].float()
    g, u = x @ wg.t(), x @ wu.t()
    h = (_plain_act(g, c["act"]) * u).to(t)
    if c["kind"] == "forward":
        return h
    x8, g, u, dh = _plain_block8(x), _plain_block8(g, c["act"]), _plain_block8(u), s["dh"].float()
    dg, du = dh * u * _plain_act_grad(g, c["act"]), dh * _plain_act(g, c["act"])
    return {"h": h, "dx": (dg @ wg + du @ wu).to(t), "dwg": (dg.t() @ x8).to(t), "dwu": (du.t() @ x8).to(t)}


def _library(s):
    from paper_1809_10572_gb300 import samd

    c, x = s["c"], s["x"]
    if c["kind"] in ("matvec", "gated_matvec"):
        f = samd.fmt(4, not c["zeros"])
        if c["kind"] == "matvec":
            w = s["w"]
            return samd.matvec4(x, w["q"], w["s"], c["G"], f, zeros=w["z"])
        g, u = s["wg"], s["wu"]
        return samd.gated_matvec4(x, g["q"], g["s"], u["q"], u["s"], c["G"], f, c["act"], zeros_g=g["z"],
                                  zeros_u=u["z"])
    if c["kind"] == "ckpt":
        return samd.block8_dequantize(samd.block8_quantize(x), x.dtype)
    if c["kind"] == "forward":
        return samd.gated_ffn_forward(x, s["wg"], s["wu"], c["act"])
    x8 = samd.block8_quantize(x)
    h, g8, u8 = samd.gated_ffn_forward(x, s["wg"], s["wu"], c["act"], checkpoints=True)
    dx, dwg, dwu = samd.gated_ffn_backward(s["dh"], x8, g8, u8, s["wg"], s["wu"], c["act"])
    return {"h": h, "dx": dx, "dwg": dwg, "dwu": dwu}


def run(state):
    return _library(state) if own else _plain(state)


# ---- the same from the definitions, in 64 bits ----------------------------------


def _exact_weights(w, c):
    """The bytes of the packed words hold two lanes each, the lower one first; a table gives a lane's value."""
    N, K, G = c["N"], c["K"], c["G"]
    b = w["q"].contiguous().view(torch.uint8)
    signed = w["z"] is None
    table = torch.tensor([v - 16 if signed and v > 7 else v for v in range(16)], dtype=torch.float64, device=DEV)
    q = torch.stack((table[(b % 16).long()], table[(b // 16).long()]), -1).reshape(N, -1)[:, :K]
    if not signed:
        q -= w["z"].double().repeat_interleave(G, 1)[:, :K]
    return q.mul_(w["s"].double().repeat_interleave(G, 1)[:, :K])


def _exact_act(g, act):
    """An activation's value and its derivative."""
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s + g * s * (1 - s)
    if act == "gelu":
        p = torch.special.ndtr(g)
        return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":  # 0.5 (1 + tanh a) = sigmoid(2 a)
        s = torch.sigmoid(math.sqrt(8 / math.pi) * (g + 0.044715 * g ** 3))
        return g * s, s + g * s * (1 - s) * math.sqrt(8 / math.pi) * (1 + 0.134145 * g ** 2)
    return torch.clamp(g, min=0), (g > 0).double()


def _exact_block8(x, relu=False):
    rows, width = x.shape
    out = torch.zeros((rows, -(-width // BLOCK) * BLOCK), dtype=torch.float64, device=DEV)
    out[:, :width] = x
    b = out.view(rows, -1, BLOCK)
    top = b.abs().max(-1, keepdim=True).values.clamp_min(2.0 ** -120)
    step = (top.view(torch.int64) >> 52 << 52).view(torch.float64) / 64  # the power of two below, six down
    codes = torch.round(b / step).clamp(-127, 127)
    b.copy_(torch.where((b > 0) & (codes < 1) & relu, torch.ones_like(b), codes) * step)
    return out[:, :width]


def exact(c, seed):
    s = prepare(c, seed)
    x = s["x"].double()
    if c["kind"] == "matvec":
        return x @ _exact_weights(s["w"], c).t()
    if c["kind"] == "gated_matvec":
        return _exact_act(x @ _exact_weights(s["wg"], c).t(), c["act"])[0] * (x @ _exact_weights(s["wu"], c).t())
    if c["kind"] == "ckpt":
        return _exact_block8(x)
    wg, wu = s["wg"].double(), s["wu"].double()
    g, u = x @ wg.t(), x @ wu.t()
    h = _exact_act(g, c["act"])[0] * u
    if c["kind"] == "forward":
        return h
    g, u = _exact_block8(g, c["act"] == "relu"), _exact_block8(u)
    a, da = _exact_act(g, c["act"])
    dg, du, x8 = s["dh"].double() * u * da, s["dh"].double() * a, _exact_block8(x)
    return {"h": h, "dx": dg @ wg + du @ wu, "dwg": dg.t() @ x8, "dwu": du.t() @ x8}
