"""The gated block and the 8-bit forms where element offsets pass 2^31: the ends of the tensors against their
definitions, bit for bit on integers."""
import pytest
import torch

import ffn_ref as ref
from gpu_util import assert_status_clean
from paper_1809_10572_gb300 import samd

pytestmark = [pytest.mark.gpu, pytest.mark.slow]


def test_more_than_two_to_the_31_hidden_values(samd_lib):
    M, K, F, t = 70000, 64, 32768, torch.bfloat16
    assert M * F > 1 << 31
    gen = torch.Generator(device="cuda").manual_seed(1)

    def draw(shape, lo, hi):
        return torch.randint(lo, hi + 1, shape, device="cuda", generator=gen, dtype=torch.int8).to(t)

    x, wg, wu = draw((M, K), -1, 1), draw((F, K), -1, 1), draw((F, K), -1, 1)
    h, g8, u8 = samd.gated_ffn_forward(x, wg, wu, "relu", checkpoints=True)
    dh = draw((M, F), -1, 1)
    x8 = samd.block8_quantize(x)
    dx, dwg, dwu, again = samd.gated_ffn_backward(dh, x8, g8, u8, wg, wu, "relu", need_h=True)
    X, G, U = x.double(), wg.double(), wu.double()
    for rows in (slice(0, 40), slice(M // 2, M // 2 + 40), slice(M - 40, M)):
        g, u = X[rows] @ G.t(), X[rows] @ U.t()  # at most 64: their 8-bit forms are exact
        want = (torch.clamp(g, min=0) * u).to(t)
        assert torch.equal(h[rows], want) and torch.equal(again[rows], want)
        assert torch.equal(g8.lanes[rows], ref.pack8(ref.block8(g, True)[0]))
        assert torch.equal(u8.exps[rows], ref.block8(u)[1])
        D = dh[rows].double()
        # dg and du are at most 64, exact in bf16
        assert torch.equal(dx[rows], ((D * u * (g > 0)) @ G + (D * torch.clamp(g, min=0)) @ U).to(t))
    for cols in (slice(0, 40), slice(F - 40, F)):
        g, u, D = X @ G[cols].t(), X @ U[cols].t(), dh[:, cols].double()
        assert torch.equal(dwg[cols], ((D * u * (g > 0)).t() @ X).to(t))  # sums of at most 64 * 70000 < 2^24
        assert torch.equal(dwu[cols], ((D * torch.clamp(g, min=0)).t() @ X).to(t))
    assert_status_clean()


def test_more_than_two_to_the_31_rows(samd_lib):
    """Rows of one element: as many steps as rows, and word and block offsets past 2^31."""
    rows = (1 << 31) + 77
    x = torch.ones((rows, 1), dtype=torch.bfloat16, device="cuda")
    x[-3:] = torch.tensor([[3.0], [-5.0], [0.25]], device="cuda")
    x[:2] = torch.tensor([[-7.0], [0.0]], device="cuda")
    b = samd.block8_quantize(x)
    y = samd.block8_dequantize(b, torch.bfloat16)
    assert torch.equal(x, y)
    assert b.exps[-3:].view(-1).tolist() == [128 - 6, 129 - 6, 125 - 6] and int(b.lanes[-2].item()) & 255 == 256 - 80
