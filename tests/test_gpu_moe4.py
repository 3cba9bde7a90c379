"""samd_moe_route and samd_moe4 against their definitions in 64 bits: exact on integers, within derived bounds else."""
import math

import pytest
import torch

import ffn_ref as ref
from gpu_util import assert_status_clean
from paper_1809_10572_gb300 import samd

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16
# what is added to a lane in the MMA's operand, and a zero point: the largest factor of an input in a group's sum
OFFSET = {BF16: 143, F16: 1039}


def matrix(seed, rows, K, G, zeros, t, span=None, word_bits=32):
    """((lanes, scales, zeros), 64-bit weights). span: lanes within that of the zero point, scales powers of two."""
    groups = -(-K // G)
    z = ref.ints(seed + 1, (rows, groups), 3, 12, torch.uint8) if zeros else None
    if span is None:
        q = ref.ints(seed, (rows, K), 0, 15) if zeros is not None else ref.ints(seed, (rows, K), -8, 7)
        s = (ref.normal(seed + 2, (rows, groups), torch.float64, 0.02).abs() + 0.001).to(t)
    else:
        q = ref.ints(seed, (rows, K), -span, span)
        if zeros:
            q = (q + z.double().repeat_interleave(G, 1)[:, :K]).clamp(0, 15)
        elif zeros is not None:
            q = q.abs()
        s = (2.0 ** ref.ints(seed + 2, (rows, groups), -1, 1)).to(t)
    return (ref.pack4(q, word_bits), s, z), ref.weights4(q, s, z, G)


def make(seed, E, K, F, G, zeros, t, span=None, word_bits=32):
    """zeros: True, False (unsigned lanes without zero points), or None (signed lanes)."""
    out = [matrix(seed + 10 * i, E * r, k, G, zeros, t, span, word_bits) for i, (r, k) in enumerate(((F, K), (F, K), (K, F)))]
    (g, wg), (u, wu), (d, wd) = out
    f = samd.fmt(4, zeros is None, 0, word_bits)
    return f, g, u, d, wg.view(E, F, K), wu.view(E, F, K), wd.view(E, K, F)


def plain(x, ids, weights, wg, wu, wd, act, rounded=None):
    """The layer in 64 bits; rounded: h as the kernel rounds it, where it is exact before."""
    y = torch.zeros((x.shape[0], wd.shape[1]), dtype=torch.float64, device="cuda")
    for m in range(x.shape[0]):
        for j, e in enumerate(ids[m].tolist()):
            if 0 <= e < wg.shape[0]:
                h = weights[m, j].double() * (ref.act(wg[e] @ x[m].double(), act) * (wu[e] @ x[m].double()))
                y[m] += wd[e] @ (h.to(rounded).double() if rounded else h)
    return y


def bound(x, ids, weights, wg, wu, wd, sg, su, sd, act, G, t):
    """A group's sum: an MMA for 16 of its inputs and one of the offsets, each within four roundings of 2^-23 of its
    largest partial sum, at most (offset + 15) times the inputs' magnitudes; then a scaled addition a group (2^-24 each,
    at most K / 32 + 8 in a row). h: rounded once; act as in the gated products' test. The tokens' sums: once more."""
    K, F = x.shape[1], wg.shape[1]
    out = torch.zeros((x.shape[0], wd.shape[1]), dtype=torch.float64, device="cuda")

    def sums(w, s, v, n):  # (rows, n) weights, (rows, groups) scales, magnitudes (n,)
        groups = s.shape[1]
        per = torch.zeros(groups * G, dtype=torch.float64, device="cuda")
        per[:n] = v
        per = per.view(groups, G).sum(1)
        mma = 4 * 2.0 ** -23 * (min(G, 128) / 8) * (OFFSET[t] + 15)
        return mma * (s.double() @ per) + (n / 32 + 8) * 2.0 ** -24 * (w.abs() @ v)

    for m in range(x.shape[0]):
        a = x[m].double()
        for j, e in enumerate(ids[m].tolist()):
            if not 0 <= e < wg.shape[0]:
                continue
            g, u = wg[e] @ a, wu[e] @ a
            dg, du = (sums(w[e], s.view(wg.shape[0], F, -1)[e], a.abs(), K) for w, s in ((wg, sg), (wu, su)))
            w = weights[m, j].double().abs()
            h = w * (ref.act(g, act) * u).abs()
            dh = w * (1.2 * dg * (u.abs() + du) + ref.act(g, act).abs() * du) + 2.0 ** -16 * h
            dh = dh + ref.UNIT[t] * (h + dh) + ref.TINY
            out[m] += wd[e].abs() @ dh + sums(wd[e], sd.view(wg.shape[0], K, -1)[e], h + dh, F)
    return out


def choose(seed, M, E, topk):
    ids = torch.stack([torch.randperm(E, generator=torch.Generator().manual_seed(seed + m))[:topk] for m in range(M)])
    w = torch.rand((M, topk), generator=torch.Generator().manual_seed(seed))
    return ids.to("cuda", torch.int32), (w / w.sum(1, keepdim=True)).cuda()


SHAPES = [(1, 64, 32, 1, 1, 32), (1, 2048, 256, 8, 2, 64), (2, 32, 64, 4, 4, 32), (3, 256, 96, 5, 3, 128), (1, 544, 1056, 16, 8, 64),
          (9, 288, 160, 3, 2, 32), (13, 1024, 352, 64, 6, 64), (33, 96, 64, 2, 2, 256), (64, 128, 128, 8, 4, 32),
          (70, 64, 96, 4, 2, 64), (40, 64, 32, 40, 32, 32), (5, 2080, 2336, 6, 2, 32), (2, 4096, 64, 2, 1, 8192),
          (40, 96, 768, 40, 4, 32), (18, 1056, 928, 64, 4, 64)]  # the last two: tiles that are a warp's


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("zeros", [None, False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_normal_data(samd_lib, shape, zeros, t):
    M, K, F, E, topk, G = shape
    f, g, u, d, wg, wu, wd = make(1, E, K, F, G, zeros, t)
    x = ref.normal(2, (M, K), t)
    ids, w = choose(3, M, E, topk)
    got = samd.moe4(x, ids, w, g, u, d, G, f, "silu")
    want = plain(x, ids, w, wg, wu, wd, "silu")
    lim = bound(x, ids, w, wg, wu, wd, g[1], u[1], d[1], "silu", G, t)
    assert ((got.double() - want).abs() <= ref.UNIT[t] * (want.abs() + lim) + lim + ref.TINY).all()
    # as a whole: two roundings, of h and of y, of at most UNIT / sqrt(3) root mean square each, and sums far below them
    assert float((got.double() - want).norm()) <= ref.UNIT[t] * float(want.norm())
    assert_status_clean()


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("zeros", [None, False, True])
@pytest.mark.parametrize("word_bits", [32, 64])
@pytest.mark.parametrize("shape", [(1, 64, 32, 2, 1, 32), (3, 288, 160, 7, 3, 64), (20, 2048, 96, 4, 2, 128), (66, 96, 256, 5, 4, 32), (40, 96, 768, 40, 4, 64)], ids=str)
def test_integers_are_exact(samd_lib, shape, word_bits, zeros, t):
    """One input of a token is 1 or -1, lanes lie within 2 of the zero point, scales are 1/2 .. 2: g and u are at most 4 in
    halves, h (weights of 1/2) at most 8 in eighths, exact in both types; a group's sum of offsets and lanes is at most
    128 * 1039 * 64 < 2^24 eighths, so every partial sum is exact in fp32."""
    M, K, F, E, topk, G = shape
    f, g, u, d, wg, wu, wd = make(11, E, K, F, G, zeros, t, span=2, word_bits=word_bits)
    x = torch.zeros((M, K), device="cuda")
    at = ref.ints(12, (M,), 0, K - 1, torch.int64)
    x[torch.arange(M, device="cuda"), at] = ref.ints(13, (M,), 0, 1).float() * 2 - 1
    ids, _ = choose(14, M, E, topk)
    w = torch.full((M, topk), 0.5, device="cuda")
    want = plain(x, ids, w, wg, wu, wd, "relu", rounded=t)
    got = samd.moe4(x.to(t), ids, w, g, u, d, G, f, "relu")
    assert torch.equal(got, want.to(t))


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("t", [BF16, F16])
def test_activations(samd_lib, act, t):
    M, K, F, E, topk, G = 4, 320, 192, 6, 2, 64
    f, g, u, d, wg, wu, wd = make(21, E, K, F, G, True, t)
    x = ref.normal(22, (M, K), t)
    ids, w = choose(23, M, E, topk)
    got = samd.moe4(x, ids, w, g, u, d, G, f, act)
    want = plain(x, ids, w, wg, wu, wd, act)
    lim = bound(x, ids, w, wg, wu, wd, g[1], u[1], d[1], act, G, t)
    assert ((got.double() - want).abs() <= ref.UNIT[t] * (want.abs() + lim) + lim + ref.TINY).all()
    assert float((got.double() - want).norm()) <= ref.UNIT[t] * float(want.norm())


@pytest.mark.parametrize("t", [BF16, F16])
def test_ids_that_repeat_or_are_none(samd_lib, t):
    """The same expert twice counts twice, an id that is no expert's counts nothing, a token of none gives zeros; all
    tokens may want one expert."""
    M, K, F, E, G = 21, 96, 64, 4, 32
    f, g, u, d, wg, wu, wd = make(31, E, K, F, G, None, t)
    x = ref.normal(32, (M, K), t)
    ids = ref.ints(33, (M, 5), -2, E + 1, torch.int32)
    ids[0] = 2
    ids[1] = -1
    ids[2] = torch.tensor([1 << 30, -(1 << 31), 4, -1, 99], dtype=torch.int32)
    ids[3] = torch.tensor([0, 3, 0, 3, 0], dtype=torch.int32)
    w = torch.rand((M, 5), generator=torch.Generator().manual_seed(34)).cuda()
    for these in (ids, torch.ones_like(ids)):
        got = samd.moe4(x, these, w, g, u, d, G, f, "silu")
        want = plain(x, these, w, wg, wu, wd, "silu")
        lim = bound(x, these, w, wg, wu, wd, g[1], u[1], d[1], "silu", G, t)
        assert ((got.double() - want).abs() <= ref.UNIT[t] * (want.abs() + lim) + lim + ref.TINY).all()
        assert all(torch.equal(got, samd.moe4(x, these, w, g, u, d, G, f, "silu")) for _ in range(4))
    assert not samd.moe4(x, torch.full_like(ids, -1), w, g, u, d, G, f, "silu").any()
    assert not samd.moe4(x, ids, w, g, u, d, G, f, "silu")[1:3].any()


def test_infinities_and_nans_stay_in_their_token(samd_lib):
    M, K, F, E, topk, G, t = 12, 256, 96, 3, 2, 64, BF16
    f, g, u, d, *_ = make(41, E, K, F, G, None, t)
    x = ref.normal(42, (M, K), t)
    ids, w = choose(43, M, E, topk)
    clean = samd.moe4(x, ids, w, g, u, d, G, f)
    bad = x.clone()
    bad[3, 7], bad[8, 200] = math.inf, math.nan
    w2 = w.clone()
    w2[10, 1] = math.nan
    got = samd.moe4(bad, ids, w2, g, u, d, G, f)
    rows = torch.tensor([m not in (3, 8, 10) for m in range(M)], device="cuda")
    assert torch.equal(got[rows], clean[rows]) and torch.isnan(got[~rows]).all()


def test_strides_streams_graphs_and_repeats(samd_lib):
    M, K, F, E, topk, G, t = 6, 512, 320, 9, 3, 32, F16
    f, g, u, d, *_ = make(51, E, K, F, G, True, t)
    router = ref.normal(52, (E, K), t, 0.05)
    x = ref.normal(53, (M, K), t)
    first = samd.moe_layer4(x, router, topk, g, u, d, G, f, "gelu")
    ids, w = samd.moe_route(x, router, topk)
    assert torch.equal(first, samd.moe4(x, ids, w, g, u, d, G, f, "gelu"))
    wide, out = ref.wide(x, 24), torch.full((M, K + 40), 5.0, dtype=t, device="cuda")
    assert torch.equal(samd.moe_layer4(wide, router, topk, g, u, d, G, f, "gelu", out=out[:, 8:K + 8]), first)
    assert (out[:, :8] == 5).all() and (out[:, K + 8:] == 5).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = samd.moe_layer4(x, router, topk, g, u, d, G, f, "gelu", stream=side)
    side.synchronize()
    assert torch.equal(first, y)
    ws = torch.full((M * topk * F * 2 + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    outs, graphs = [torch.zeros_like(first) for _ in range(2)], []
    for i in range(2):  # two graphs, one workspace
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            samd.moe_layer4(x, router, topk, g, u, d, G, f, ("gelu", "silu")[i], out=outs[i], workspace=ws)
        graphs.append(gr)
    for seed in (54, 55):
        x.copy_(ref.normal(seed, (M, K), t))
        for gr in graphs:
            gr.replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(outs[i], samd.moe_layer4(x, router, topk, g, u, d, G, f, ("gelu", "silu")[i]))


def test_empty_calls(samd_lib):
    f, g, u, d, *_ = make(61, 3, 64, 32, 32, None, BF16)
    x = torch.empty((0, 64), dtype=BF16, device="cuda")
    router = torch.zeros((3, 64), dtype=BF16, device="cuda")
    assert samd.moe_layer4(x, router, 2, g, u, d, 32, f).shape == (0, 64)


# ---- routing -------------------------------------------------------------------


def check_route(x, router, topk, normalize, ids, w, exact_logits=True):
    """By sorting; the weights to a few roundings of fp32 (ex2 and the sums)."""
    logits = x.double() @ router.double().t()
    rank = torch.where(torch.isnan(logits), torch.full_like(logits, -math.inf), logits)
    order = sorted_ids(rank, torch.isnan(logits), topk)
    assert torch.equal(ids.long(), order)
    chosen = logits.gather(1, order)
    total = torch.softmax(chosen if normalize else logits, -1)
    want = total if normalize else total.gather(1, order)
    # a logit's fp32 error (K / 32 products in a row, 2^-24 of the magnitudes each) is one of exp's argument
    mags = (x.double().abs() @ router.double().abs().t()).amax(1, keepdim=True)
    lim = 2 * (x.shape[1] / 32 + 16) * 2.0 ** -24 * mags + 2.0 ** -18
    assert ((w.double() - want).abs() <= lim * want + 1e-30).all()


def sorted_ids(rank, nan, topk):
    rows = []
    for r, n in zip(rank.tolist(), nan.tolist()):
        rows.append(sorted(range(len(r)), key=lambda e: (n[e], -r[e], e))[:topk])
    return torch.tensor(rows, dtype=torch.int64, device=rank.device)


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("normalize", [True, False])
@pytest.mark.parametrize("shape", [(1, 32, 1, 1), (1, 4096, 8, 2), (3, 64, 5, 5), (7, 1056, 33, 4), (2, 256, 64, 32), (65, 2048, 128, 8),
                                   (5, 96, 1024, 32), (1, 7168, 256, 8)], ids=str)
def test_route(samd_lib, shape, normalize, t):
    M, K, E, topk = shape
    # integers: logits are exact, many of them equal
    x, router = ref.ints(71, (M, K), -1, 1).to(t), (ref.ints(72, (E, K), -8, 8) * (ref.ints(73, (E, K), 0, 63) == 0)).to(t) / 8
    ids, w = samd.moe_route(x, router, topk, normalize)
    check_route(x, router, topk, normalize, ids, w)
    # values: the chosen are right wherever the first topk + 1 logits (nothing else decides) are further apart than their
    # error
    x, router = ref.normal(74, (M, K), t), ref.normal(75, (E, K), t, 1 / math.sqrt(K))
    ids, w = samd.moe_route(x, router, topk, normalize)
    logits = x.double() @ router.double().t()
    near = logits.sort(-1, descending=True).values[:, :topk + 1]
    gap = (near[:, :-1] - near[:, 1:]).amin(-1) if E > 1 else torch.ones(M, device="cuda")
    ok = gap > 2.0 ** -17
    assert ok.float().mean() > 0.5
    check_route(x[ok], router, topk, normalize, ids[ok], w[ok])


def test_route_of_ties_infinities_and_nans(samd_lib):
    t, K, E = BF16, 64, 40
    router = torch.zeros((E, K), dtype=t, device="cuda")
    x = torch.zeros((4, K), dtype=t, device="cuda")
    x[:, 0] = 1
    router[:, 0] = torch.arange(E, device="cuda") // 10  # four classes of ten equal logits
    router[7, 1], router[33, 1] = math.nan, math.nan
    x[1, 1] = 1.0  # (0 times NaN is one as well: all tokens see two NaN logits)
    ids, w = samd.moe_route(x, router, 12)
    want = [i for i in range(30, 40) if i != 33] + [20, 21, 22]
    assert ids.tolist() == [want] * 4
    torch.testing.assert_close(w.sum(1), torch.ones(4, device="cuda"))
    ids, w = samd.moe_route(x, router, 32)
    assert ids[0, :31].tolist() == want[:9] + list(range(20, 30)) + list(range(10, 20)) + [0, 1]
    router[5, 0], router[6, 0] = -math.inf, math.inf
    ids, _ = samd.moe_route(x, router, 3)
    assert ids.tolist() == [[6, 30, 31]] * 4
