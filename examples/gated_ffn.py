"""A gated feed-forward block, trained with its activations kept in 8 bits and then served from 4-bit weights.

    python examples/gated_ffn.py [--width 512 --hidden 1408 --tokens 1024 --steps 120 --type bf16]

A student block y = (act(x Wg^T) * (x Wu^T)) Wd^T learns the outputs of a fixed teacher. A training step keeps x and
the two projections as 8-bit forms (33 bits for four elements instead of 64) and takes all gradients of the gated part
from them; the down projection is a plain product. Afterwards the weights are rounded to 4-bit lanes with a scale for
every 32 inputs, packed as the library packs lanes, and single tokens go through the packed block.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1809_10572_gb300 import samd  # noqa: E402

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def pack_weights(w: torch.Tensor, group: int):
    """(packed signed 4-bit lanes, scales) of a weight matrix (N, K), scaled by each group's largest magnitude."""
    N, K = w.shape
    pad = torch.nn.functional.pad(w.float(), (0, -K % group)).view(N, -1, group)
    # a group of zeros has a scale too: of the type's smallest step, where that is above 1e-8 (which fp16 rounds to zero)
    least = max(1e-8, torch.finfo(w.dtype).smallest_normal * torch.finfo(w.dtype).eps)
    scales = (pad.abs().amax(-1) / 7).clamp(min=least).to(w.dtype)
    q = (pad / scales.float().unsqueeze(-1)).round().clamp(-8, 7).view(N, -1)[:, :K].to(torch.int8)
    return samd.pack(q, samd.fmt(4, True)).view(N, -1), scales


class TrainedBlock:
    """The block's fp32 master weights, a step of gradient descent on them, and its packed form."""

    def __init__(self, width: int, hidden: int, dtype, act: str, seed: int):
        g = torch.Generator(device="cuda").manual_seed(seed)
        def draw(rows, cols):
            return torch.randn((rows, cols), device="cuda", generator=g) / cols ** 0.5
        self.wg, self.wu, self.wd = draw(hidden, width), draw(hidden, width), draw(width, hidden)
        self.dtype, self.act = dtype, act

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        h = samd.gated_ffn_forward(x, self.wg.to(self.dtype), self.wu.to(self.dtype), self.act)
        return h @ self.wd.to(self.dtype).t()

    def step(self, x: torch.Tensor, target: torch.Tensor, rate: float) -> float:
        wg, wu, wd = (w.to(self.dtype) for w in (self.wg, self.wu, self.wd))
        # forward; what stays for the backward pass: x, g and u in 8 bits
        x8 = samd.block8_quantize(x)
        h, g8, u8 = samd.gated_ffn_forward(x, wg, wu, self.act, checkpoints=True)
        y = h @ wd.t()
        del h
        err = y.float() - target.float()
        loss = float(err.square().mean())
        dy = (err * (2 / err.shape[1])).to(self.dtype)
        # backward: h is formed again from the checkpoints for the down projection's gradient
        dh = dy @ wd
        _, dwg, dwu, h = samd.gated_ffn_backward(dh, x8, g8, u8, wg, wu, self.act, need_dx=False, need_h=True)
        dwd = dy.t() @ h
        for w, d in ((self.wg, dwg), (self.wu, dwu), (self.wd, dwd)):
            w.sub_(d.float() * (rate / x.shape[0]))
        return loss

    def packed(self, group: int = 32) -> "PackedBlock":
        return PackedBlock([pack_weights(w.to(self.dtype), group) for w in (self.wg, self.wu, self.wd)], group, self.act)


class PackedBlock:
    """The block on 4-bit weights, for a few tokens at a time."""

    def __init__(self, weights, group: int, act: str):
        (self.g, self.u, self.d), self.group, self.act, self.f = weights, group, act, samd.fmt(4, True)

    def __call__(self, x: torch.Tensor) -> torch.Tensor:
        h = samd.gated_matvec4(x, *self.g, *self.u, self.group, self.f, self.act)
        return samd.matvec4(h, *self.d, self.group, self.f)

    def bytes(self) -> int:
        return sum(t.numel() * t.element_size() for w in (self.g, self.u, self.d) for t in w)


def main(argv=None) -> dict:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--hidden", type=int, default=1408)
    ap.add_argument("--tokens", type=int, default=1024)
    ap.add_argument("--steps", type=int, default=120)
    ap.add_argument("--rate", type=float, default=2.0)
    ap.add_argument("--type", choices=sorted(TYPES), default="bf16")
    ap.add_argument("--act", choices=sorted(samd.ACTS), default="silu")
    a = ap.parse_args(argv)
    dtype = TYPES[a.type]
    teacher, student = (TrainedBlock(a.width, a.hidden, dtype, a.act, s) for s in (1, 2))
    gen = torch.Generator(device="cuda").manual_seed(3)
    losses = []
    for _ in range(a.steps):
        x = torch.randn((a.tokens, a.width), device="cuda", generator=gen).to(dtype)
        losses.append(student.step(x, teacher.forward(x), a.rate))
    served = student.packed()
    worst = 0.0
    for _ in range(4):  # one token at a time, as a decoder sends them
        x = torch.randn((1, a.width), device="cuda", generator=gen).to(dtype)
        full, low = student.forward(x).float(), served(x).float()
        worst = max(worst, float((low - full).norm() / full.norm()))
    plain = 3 * a.width * a.hidden * 2
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f} in {a.steps} steps; 4-bit weights {served.bytes()} bytes of {plain}, "
          f"a token's output {100 * worst:.1f}% from the 16-bit one at most")
    return {"losses": losses, "serving_error": worst, "bytes": served.bytes(), "status": samd.samd_device_status()}


if __name__ == "__main__":
    main()
