"""How the gated block's example rounds weights to 4-bit lanes and scales, on the host (its packing replaced)."""
import importlib.util
import os

import pytest
import torch

from paper_1809_10572_gb300 import samd

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture()
def rounded(monkeypatch):
    """pack_weights with the lanes' values in the place of packed words."""
    spec = importlib.util.spec_from_file_location("gated_ffn_example_cpu", os.path.join(ROOT, "examples", "gated_ffn.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    monkeypatch.setattr(samd, "pack", lambda q, f: q)
    return mod.pack_weights


@pytest.mark.parametrize("t", [torch.float16, torch.bfloat16])
def test_groups_of_zeros_and_of_tiny_weights(rounded, t):
    torch.manual_seed(0)
    w = torch.randn((4, 96)).to(t)
    w[0, :32] = 0  # as pruned or padded weights have them
    w[1, 32:64] *= 2.0 ** -22  # scales that fp16 holds with few bits
    w[2] = 0
    w[3, 64:] = torch.finfo(t).smallest_normal * torch.finfo(t).eps  # the type's smallest step
    q, scales = rounded(w, 32)
    assert torch.isfinite(scales).all() and (scales > 0).all()
    stands = q.double() * scales.double().repeat_interleave(32, 1)
    assert not q[0, :32].any() and not q[2].any()
    # half a step for rounding, and what a scale of few bits clamps: half of fp16's smallest step on each of 7
    floor = max(1e-8, float(torch.finfo(t).smallest_normal * torch.finfo(t).eps))
    amax = w.double().abs().view(4, 3, 32).amax(-1)
    bound = (0.5 * scales.double() + torch.clamp(amax - 7 * scales.double(), min=0) + 1e-3 * amax).repeat_interleave(32, 1)
    assert ((stands - w.double()).abs() <= bound).all()
    assert (scales.double() >= 0.5 * floor).all()
