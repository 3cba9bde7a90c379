"""samd_paged_attention on finite values of every range, and on infinities, against its definition in 64 bits."""
import math

import pytest
import torch

import cache_ref as ref
from paper_1809_10572_gb300 import samd

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16
PAGE = 16


def one_sequence(kl, ks, vl, vs, bits, width=0):
    """(cache, table, lengths, key values, value values in pages) of one sequence whose rows are given as (heads, tokens,
    ..); slots behind it have NaN scales. width: entries of the table at least (those behind the sequence name no page);
    with more than 16 of 16 tokens a head is dealt out over CTAs."""
    n = kl.shape[1]

    def paged(x, fill):
        more = x.new_full((x.shape[0], -n % PAGE, x.shape[2]), fill)
        return torch.cat((x, more), 1).unflatten(1, (-1, PAGE)).transpose(0, 1).contiguous()

    kl, ks, vl, vs = paged(kl, 3), paged(ks, math.nan), paged(vl, 3), paged(vs, math.nan)
    table = torch.full((1, max(width, kl.shape[0])), -1, dtype=torch.int32, device="cuda")
    table[0, :kl.shape[0]] = torch.arange(kl.shape[0])
    cache = samd.PagedCache(ref.pack(kl, bits), ks, ref.pack(vl, bits), vs)
    return cache, table, torch.tensor([n], dtype=torch.int32, device="cuda"), ref.values(kl, ks), ref.values(vl, vs)


def check(got, q, n, k, v, scale, t, scores=None, before=None, own=False):
    """Of one sequence; own: every output against its own block's magnitudes, so that what lies in other elements of the
    rows does not count. A weight below 2^-126 of the largest is 0 in fp32: n times that of the largest value at most."""
    kb, vb = (x.transpose(0, 1).flatten(1, 2)[:, :n] for x in (k, v))
    want, p, x = ref.attention(q[0], kb, vb, scale)
    width = ref.BLOCK if own else vb.shape[2]
    for at in range(0, vb.shape[2], width):
        part = slice(at, at + width)
        vp = vb[:, :, part].contiguous()
        bound, delta = ref.attention_bound(q[0], kb, vp, scale, p, x, want[:, part], t)
        bound = bound + n * 2.0 ** -126 * vp.abs().max()
        err = (got[0, :, part].double() - want[:, part]).abs()
        assert (err <= bound).all(), (at, float((err / bound).max()))
    if scores is not None:
        group = q.shape[1] // kb.shape[0]
        w = p.view(kb.shape[0], group, n)
        total = before[0, :, :n].double() + w.sum(1)
        # a weight's error twice (its own, the sum's), the sums over n and over the group, one addition to the old
        lim = (w * (2 * delta.view(-1, group, 1) + (n / 16 + 64 + group) * 2.0 ** -23)).sum(1) + group * 2.0 ** -126
        assert ((scores[0, :, :n].double() - total).abs() <= lim + 2.0 ** -24 * (total + lim)).all()
        assert torch.equal(scores[0, :, n:], before[0, :, n:])


def rising(steps, heads, dim, bits, t, rise):
    """Keys and a scale that make the logits `rise` times `steps` (0 .. 1, a token each) for a query of 1 in element 0."""
    most = 2 ** (bits - 1) - 1
    kl = torch.zeros((heads, len(steps), dim), dtype=torch.int64, device="cuda")
    kl[:, :, 0] = torch.round(most * steps).long()
    return kl, torch.ones((heads, len(steps), dim // 32), dtype=t, device="cuda"), rise / most


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("rise", [15, 22, 40, 88, 100, 180])
@pytest.mark.parametrize("zero", ["all", "front", "all but the last", "odd"])
def test_rows_of_zero_values(samd_lib, zero, rise, bits, t):
    """Values that are zero in whole rows, while the logits rise along the sequence by `rise` in all: such tokens weigh as
    much as others, and the sum of weights stays finite."""
    heads, dim, n = 2, 64, 333
    kl, ks, scale = rising(torch.linspace(0, 1, n, device="cuda"), heads, dim, bits, t, rise)
    vl, vs = ref.random_rows(3, (heads, n), dim, bits, t)
    at = torch.arange(n, device="cuda")
    gone = {"all": at >= 0, "front": at < 300, "all but the last": at < n - 1, "odd": at % 2 == 1}[zero]
    vl[:, gone], vs[:, gone] = 0, 0.0
    cache, table, lens, k, v = one_sequence(kl, ks, vl, vs, bits)
    q = torch.zeros((1, 6, dim), dtype=t, device="cuda")
    q[0, :, 0] = torch.tensor([1, 0.75, 0.5, 0.25, -1, 0.125])
    scores = torch.rand((1, heads, n + 3), generator=ref.gen(4)).cuda()
    before = scores.clone()
    got = samd.paged_attention(q, cache, table, lens, scale=scale, scores=scores)
    check(got, q, n, k, v, scale, t, scores, before)
    assert torch.equal(got, samd.paged_attention(q, cache, table, lens, scale=scale))


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("width", [0, 20])
@pytest.mark.parametrize("last", [31.0, 60.0])
@pytest.mark.parametrize("runs", [1, 4])
def test_zero_values_before_the_first_that_are_not(samd_lib, runs, last, width, t):
    """Logits in units of log2: tokens with zero values at 0, as many at 31.5, then some with values: every partial sum of
    weights is far within fp32 for any reference near the largest logit."""
    dim, n = 64, 48 * runs
    run = torch.arange(n, device="cuda") // (16 * runs)
    kl, ks, scale = rising(torch.tensor([0.0, 31.5, last], device="cuda")[run] * 2 / 127, 1, dim, 8, t, 127 / 2 * math.log(2))
    vl = torch.ones((1, n, dim), dtype=torch.int64, device="cuda")
    vs = torch.ones((1, n, 2), dtype=t, device="cuda")
    vl[:, run < 2], vs[:, run < 2] = 0, 0.0
    cache, table, lens, k, v = one_sequence(kl, ks, vl, vs, 8, width)
    q = torch.zeros((1, 1, dim), dtype=t, device="cuda")
    q[..., 0] = 1
    scores = torch.zeros((1, 1, n), device="cuda")
    got = samd.paged_attention(q, cache, table, lens, scale=scale, scores=scores)
    check(got, q, n, k, v, scale, t, scores, torch.zeros_like(scores))


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("value", [math.inf, -math.inf])
@pytest.mark.parametrize("n,width", [(1, 0), (1, 20), (40, 0), (40, 20), (700, 0)])
def test_an_infinity_in_q_gives_nans(samd_lib, n, width, value, bits, t):
    """Also where the keys' lanes at its element have one sign, so that all products are infinities of one sign."""
    heads, dim = 2, 64
    kl, ks = ref.random_rows(11, (heads, n), dim, bits, t)
    vl, vs = ref.random_rows(13, (heads, n), dim, bits, t)
    q = ref.normal(15, (1, 4, dim), t)
    for lane in (-3, 3):
        kl[:, :, 5] = lane
        cache, table, lens, *_ = one_sequence(kl, ks, vl, vs, bits, width)
        clean, hit = q.clone(), q.clone()
        hit[0, 1, 5] = value
        scores = torch.zeros((2, 1, heads, n), device="cuda")
        a = samd.paged_attention(clean, cache, table, lens, scores=scores[0])
        b = samd.paged_attention(hit, cache, table, lens, scores=scores[1])
        assert torch.isnan(b[0, 1]).all() and torch.isnan(scores[1, 0, 0]).all()
        assert torch.equal(a[0, [0, 2, 3]], b[0, [0, 2, 3]]) and torch.equal(scores[0, 0, 1], scores[1, 0, 1])
        assert torch.isfinite(a).all() and torch.isfinite(scores[0]).all()


@pytest.mark.parametrize("scale", [3e38, -3.4e38])
def test_scales_next_to_the_largest_float(samd_lib, scale):
    """log2(e) times them is past fp32; with a small q the logits are ordinary numbers."""
    heads, dim, n, t = 2, 64, 300, BF16
    kl, ks = ref.random_rows(21, (heads, n), dim, 8, t)
    vl, vs = ref.random_rows(23, (heads, n), dim, 8, t)
    cache, table, lens, k, v = one_sequence(kl, ks, vl, vs, 8)
    q = ref.normal(25, (1, 4, dim), torch.float64).mul_(2.0 ** -126).to(t)
    got = samd.paged_attention(q, cache, table, lens, scale=scale)
    check(got, q, n, k, v, torch.tensor(scale).float().item(), t)


def test_values_of_tiny_scales_before_large_ones(samd_lib):
    """Scales of 2^-110 in front: their weights are summed as those of zero rows are."""
    heads, dim, n, t = 2, 64, 333, BF16
    for rise in (22, 40, 100):
        kl, ks, scale = rising(torch.linspace(0, 1, n, device="cuda"), heads, dim, 8, t, rise)
        vl, vs = ref.random_rows(5, (heads, n), dim, 8, t)
        vs[:, :300] = 2.0 ** -110
        cache, table, lens, k, v = one_sequence(kl, ks, vl, vs, 8)
        q = torch.zeros((1, 4, dim), dtype=t, device="cuda")
        q[..., 0] = torch.tensor([1, 0.5, -1, 0.125])
        scores = torch.zeros((1, heads, n), device="cuda")
        got = samd.paged_attention(q, cache, table, lens, scale=scale, scores=scores)
        check(got, q, n, k, v, scale, t, scores, torch.zeros_like(scores))


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dim", [32, 64, 96, 128, 160, 192, 224, 256])
def test_blocks_of_any_size_beside_each_other(samd_lib, dim, bits, t):
    """Blocks of 32 elements with scales of their own: the same ratio in all tokens, growing along the sequence, falling,
    and any in any token, some of them zero. An output depends on its own block's values alone."""
    heads, n, nb = 2, 700, dim // 32
    lo, hi = (-100, 100) if t is BF16 else (-24, 8)
    kl, ks = ref.random_rows(31, (heads, n), dim, bits, t)
    vl, _ = ref.random_rows(33, (heads, n), dim, bits, t)
    q = ref.normal(35, (1, 6, dim), t, 2.0)
    i, blk = torch.arange(n, device="cuda")[:, None], torch.arange(nb, device="cuda")[None]
    span = hi - lo
    exps = {"own ratio": hi - (blk * 29) % (span + 1) + 0 * i, "rising": lo + (i * span // n + blk * 7) % (span + 1),
            "falling": hi - (i * span // n + blk * 7) % (span + 1), "tiny": lo + 0 * (i + blk),
            "any": ref.ints(37, (n, nb), lo, hi)}
    for name, e in exps.items():
        vs = torch.exp2(e.double()).expand(heads, n, nb).clone()
        if name == "any":
            vs *= ref.ints(39, (heads, n, nb), 0, 9) > 0
        cache, table, lens, k, v = one_sequence(kl, ks, vl, vs.to(t), bits)
        for factor in (1.0, 8.0):
            scale = factor * dim ** -0.5
            check(samd.paged_attention(q, cache, table, lens, scale=scale), q, n, k, v, scale, t, own=True)
        # the same tokens in one CTA
        cache, table, lens, k, v = one_sequence(*(x[:, :200] for x in (kl, ks, vl, vs.to(t))), bits)
        check(samd.paged_attention(q, cache, table, lens, scale=dim ** -0.5), q, 200, k, v, dim ** -0.5, t, own=True)


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("n,width", [(33, 0), (33, 20), (200, 20), (333, 0), (700, 0)])
def test_equal_logits_of_any_size(samd_lib, n, width, t):
    """The same key for all tokens, logits up to 2^40: whatever a logit's rounding is, it is the same for all, and all
    weigh 1 / n. (A weight times its scale is rounded by 2^-11; sums as everywhere.)"""
    heads, dim = 2, 64
    vl, vs = ref.random_rows(41, (heads, n), dim, 8, t)
    kl = torch.zeros((heads, n, dim), dtype=torch.int64, device="cuda")
    kl[..., 0], kl[..., 33] = 127, -100
    cache, table, lens, k, v = one_sequence(kl, torch.ones_like(vs), vl, vs, 8, width)
    vb = v.transpose(0, 1).flatten(1, 2)[:, :n].repeat_interleave(2, 0)
    want = vb.mean(1)
    lim = (2.0 ** -11 + (n / 16 + 64) * 2.0 ** -23) * vb.abs().mean(1)
    for size in (1.0, 2.0 ** 15, -2.0 ** 12):
        for scale in (0.125, 2.0 ** 17, 2.0 ** 18 / 3):
            q = torch.zeros((1, 4, dim), dtype=t, device="cuda")
            q[0, :, 0] = torch.tensor([1, -1, 0.75, 0.01]) * size
            scores = torch.zeros((1, heads, n), device="cuda")
            got = samd.paged_attention(q, cache, table, lens, scale=scale, scores=scores)
            assert ((got[0].double() - want).abs() <= ref.UNIT[t] * (want.abs() + lim) + lim).all(), (size, scale)
            assert ((scores.double() - 2 / n).abs() <= 2 / n * (n / 16 + 66) * 2.0 ** -23).all(), (size, scale)


@pytest.mark.slow
def test_counted_weights_past_two_to_the_31(samd_lib):
    """A workspace whose logits take 2.4 GB, the last sequence's at its end."""
    heads, dim, n, t, seqs, pages = 8, 32, 3000, F16, 9, 65536
    rows = [x for s in (51, 53) for x in ref.random_rows(s, (heads, n), dim, 4, t)]
    cache, one, _, k, v = one_sequence(*rows, 4)
    table = torch.full((seqs, pages), -1, dtype=torch.int32, device="cuda")
    table[0, :one.shape[1]] = table[-1, :one.shape[1]] = one[0]
    lens = torch.tensor([100] + [0] * (seqs - 2) + [n], dtype=torch.int32, device="cuda")
    assert samd.samd_paged_attention_workspace_size(cache._desc, samd._cache_seqs(table, lens), heads, True) > 1 << 31
    q = ref.normal(55, (seqs, heads, dim), t, 2.0)
    scores = torch.zeros((seqs, heads, n), device="cuda")
    got = samd.paged_attention(q, cache, table, lens, scores=scores)
    for b, m in ((0, 100), (seqs - 1, n)):
        check(got[b:b + 1], q[b:b + 1], m, k, v, dim ** -0.5, t, scores[b:b + 1], torch.zeros_like(scores[:1]))
    assert not got[1:-1].any() and not scores[1:-1].any()
