"""samd_moe4 with channels far above the others, against its definition in 64 bits within a bound that knows only the
products of the integers; and matrices past 2^31 bytes."""
import pytest
import torch

import ffn_ref as ref
from paper_1809_10572_gb300 import samd
from test_gpu_moe4 import choose, make, plain

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def bound(x, ids, weights, wg, wu, wd, act, t):
    """A sum of n products of lanes and inputs, 16 in an MMA, whose additions are 2^-22 of the partial sums' magnitudes off
    at most, and a scaled addition for each group (32 inputs or more, 2^-24): n / 16 + 8 times 2^-21 of all magnitudes.
    h is rounded once; act as in the gated products' test."""
    out = torch.zeros((x.shape[0], wd.shape[1]), dtype=torch.float64, device="cuda")
    K, F = x.shape[1], wg.shape[1]
    for m in range(x.shape[0]):
        a = x[m].double()
        for j, e in enumerate(ids[m].tolist()):
            g, u = wg[e] @ a, wu[e] @ a
            dg, du = ((K / 16 + 8) * 2.0 ** -21 * (w[e].abs() @ a.abs()) for w in (wg, wu))
            w = weights[m, j].double().abs()
            h = w * (ref.act(g, act) * u).abs()
            dh = w * (1.2 * dg * (u.abs() + du) + ref.act(g, act).abs() * du) + 2.0 ** -16 * h
            dh = dh + ref.UNIT[t] * (h + dh) + ref.TINY
            out[m] += wd[e].abs() @ dh + (F / 16 + 8) * 2.0 ** -21 * (wd[e].abs() @ (h + dh))
    return out


def without(w, columns, rows, G, f):
    """The matrix with the weights of some columns 0: their lanes at the zero point."""
    lanes, scales, zeros = w
    K = scales.shape[1] * G
    b = lanes.view(torch.uint8).view(rows, -1)
    q = torch.stack((b & 15, b >> 4), -1).flatten(1).long()
    at = torch.zeros_like(q) if zeros is None else zeros.long().repeat_interleave(G, 1)[:, :K]
    q[:, columns] = at[:, columns]
    return (ref.pack4(q), scales, zeros), ref.weights4(torch.where(q > 7, q - 16, q) if f.is_signed else q, scales, zeros, G)


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("zeros", [None, False, True])
@pytest.mark.parametrize("G", [32, 64, 128, 256])
@pytest.mark.parametrize("M,K,F,E,topk", [(1, 512, 256, 4, 2), (9, 256, 512, 3, 2), (40, 256, 768, 40, 4)])
def test_channels_far_above_the_others(samd_lib, M, K, F, E, topk, G, zeros, t):
    """Some inputs, and some hidden columns, are 1000 to 10000 times the others, and meet weights of zero: the outputs are
    those of the other channels, with their precision."""
    f, g, u, d, *_ = make(5, E, K, F, G, zeros, t)
    big = torch.tensor([3, 40, K // 2 + 5, K - 1], device="cuda")
    (g, wg), (u, wu) = (without(w, big, E * F, G, f) for w in (g, u))
    wg, wu = wg.view(E, F, K), wu.view(E, F, K)
    # hidden columns: their rows of up carry larger scales
    far = torch.tensor([7, F // 2 + 9, F - 2], device="cuda")
    s = u[1].view(E, F, -1).clone()
    s[:, far] *= 512.0
    wu = wu.clone()
    wu[:, far] *= 512.0
    u = (u[0], s.view(E * F, -1), u[2])
    d, wd = without(d, far, E * K, G, f)
    wd = wd.view(E, K, F)
    x = ref.normal(6, (M, K), t, 0.25)
    ids, w = choose(8, M, E, topk)
    for factor in (1000, 10000):
        x[:, big] = (torch.tensor([1.0, -0.7, 0.3, 0.9], device="cuda") * factor).to(t)
        got = samd.moe4(x, ids, w, g, u, d, G, f, "silu")
        want = plain(x, ids, w, wg, wu, wd, "silu")
        lim = bound(x, ids, w, wg, wu, wd, "silu", t)
        err = (got.double() - want).abs()
        assert torch.isfinite(want.to(t)).all() and (err <= ref.UNIT[t] * (want.abs() + lim) + lim + ref.TINY).all()
        assert float(err.norm()) <= ref.UNIT[t] * float(want.norm())


@pytest.mark.slow
def test_matrices_past_two_to_the_31_bytes(samd_lib):
    """The last experts of matrices of 4.3 GB each."""
    E, K, F, G, topk, t = 512, 4096, 4096, 128, 3, BF16
    g = torch.Generator(device="cuda").manual_seed(3)

    def rows(n, k):
        return (torch.randint(-(1 << 31), (1 << 31) - 1, (n, k // 8), dtype=torch.int32, device="cuda", generator=g),
                (torch.rand((n, k // G), device="cuda", generator=g) + 0.5).mul_(0.01).to(t))

    mats = gate, up, down = rows(E * F, K), rows(E * F, K), rows(E * K, F)
    assert gate[0].numel() * 4 > 1 << 31
    x = ref.normal(4, (2, K), t)
    ids = torch.tensor([[511, 0, 260], [255, 510, 511]], dtype=torch.int32, device="cuda")
    w = torch.tensor([[0.5, 0.25, 0.25], [0.125, 0.5, 0.375]], device="cuda")
    got = samd.moe4(x, ids, w, gate, up, down, G, samd.fmt(4, True), "silu")
    want = torch.zeros((2, K), dtype=torch.float64, device="cuda")
    lim = torch.zeros_like(want)
    for m in range(2):
        for j, e in enumerate(ids[m].tolist()):
            own = []
            for (lanes, scales), n, k in zip(mats, (F, F, K), (K, K, F)):
                b = lanes.view(E, n, -1)[e].contiguous().view(torch.uint8).view(n, -1)
                q = torch.stack((b & 15, b >> 4), -1).flatten(1).long()
                own.append(ref.weights4(torch.where(q > 7, q - 16, q), scales.view(E, n, -1)[e], None, G)[None])
            one = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
            a = x[m:m + 1], one, w[m:m + 1, j:j + 1], *own, "silu"
            want[m] += plain(*a)[0]
            lim[m] += bound(*a, t)[0]
    assert ((got.double() - want).abs() <= ref.UNIT[t] * (want.abs() + lim) + lim + ref.TINY).all()
