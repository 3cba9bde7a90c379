"""samd_paged_attention against its definition in 64 bits: exact where every rounding is, within derived bounds else."""
import math

import pytest
import torch

import cache_ref as ref
from gpu_util import assert_status_clean
from paper_1809_10572_gb300 import samd

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def make(seed, lengths, heads, dim, bits, page, t, spread=1.0, capacity=None):
    """(cache, table, lengths, key values, value values (pages, heads, page, dim) in 64 bits). Slots of no token hold
    lanes and scales that would be seen: NaN scales."""
    width = -(-(capacity or max(max(lengths), 1)) // page)
    table, pages = ref.pages_for(seed, len(lengths), width)
    shape = (pages, heads, page)
    kl, ks = ref.random_rows(seed + 1, shape, dim, bits, t, spread)
    vl, vs = ref.random_rows(seed + 3, shape, dim, bits, t, spread)
    used = torch.zeros((pages, page), dtype=torch.bool, device="cuda")
    for b, n in enumerate(lengths):
        i = torch.arange(n, device="cuda")
        used[table[b, i // page].long(), i % page] = True
    for s in (ks, vs):
        s.masked_fill_(~used[:, None, :, None], math.nan)
    cache = samd.PagedCache(ref.pack(kl, bits), ks, ref.pack(vl, bits), vs)
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    return cache, table, lens, ref.values(kl, ks), ref.values(vl, vs)


def check(got, q, table, lengths, k, v, page, scale, t, scores=None, before=None):
    for b, n in enumerate(lengths):
        if n == 0:
            assert not got[b].any()
            assert scores is None or torch.equal(scores[b], before[b])
            continue
        kb, vb = ref.gather(k, table, b, n, page), ref.gather(v, table, b, n, page)
        want, p, x = ref.attention(q[b], kb, vb, scale)
        bound, delta = ref.attention_bound(q[b], kb, vb, scale, p, x, want, t)
        err = (got[b].double() - want).abs()
        assert (err <= bound).all(), (b, n, float((err / bound).max()))
        if scores is not None:
            group = q.shape[1] // kb.shape[0]
            w = p.view(kb.shape[0], group, n)
            add = w.sum(1)
            # a weight's error twice (its own, the sum's), the sum over n and over the group, one addition to the old
            lim = (w * (2 * delta.view(-1, group, 1) + (n / 16 + 64 + group) * 2.0 ** -23)).sum(1)
            total = before[b, :, :n].double() + add
            assert ((scores[b, :, :n].double() - total).abs() <= lim + 2.0 ** -24 * (total + lim) + 1e-37).all()
            assert torch.equal(scores[b, :, n:], before[b, :, n:])


LENGTHS = [[1], [0], [2, 0, 15], [16, 17, 31], [100], [255, 256, 0, 3], [257, 1, 0, 0, 64], [1000, 33, 0, 700, 16, 1],
           [5000], [0, 0, 0, 2049]]


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
def test_lengths(samd_lib, lengths, bits, t):
    heads, group, dim, page = 2, 4, 128, 16
    cache, table, lens, k, v = make(1, lengths, heads, dim, bits, page, t)
    q = ref.normal(9, (len(lengths), heads * group, dim), t)
    got = samd.paged_attention(q, cache, table, lens)
    check(got, q, table, lengths, k, v, page, dim ** -0.5, t)
    assert_status_clean()


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dim", [32, 64, 96, 128, 160, 192, 224, 256])
def test_head_sizes(samd_lib, dim, bits, t):
    lengths = [300, 0, 19, 513]
    for heads, group, page in ((1, 1, 16), (3, 5, 64)):
        cache, table, lens, k, v = make(dim, lengths, heads, dim, bits, page, t, spread=4.0)
        q = ref.normal(dim + 1, (4, heads * group, dim), t)
        got = samd.paged_attention(q, cache, table, lens)
        check(got, q, table, lengths, k, v, page, dim ** -0.5, t)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("heads,group", [(1, 1), (8, 1), (2, 2), (3, 7), (2, 8), (2, 9), (1, 16), (2, 17), (1, 71), (1, 256)])
def test_head_layouts(samd_lib, heads, group, bits):
    lengths = [77, 400, 0]
    cache, table, lens, k, v = make(5, lengths, heads, 64, bits, 32, BF16)
    q = ref.normal(6, (3, heads * group, 64), BF16)
    scores = torch.rand((3, heads, 401), generator=ref.gen(7)).cuda()
    before = scores.clone()
    got = samd.paged_attention(q, cache, table, lens, scores=scores)
    check(got, q, table, lengths, k, v, 32, 64 ** -0.5, BF16, scores, before)


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("page", [16, 32, 128, 1024])
def test_scores(samd_lib, page, t):
    """Weights are added to what was there, at the tokens that are, twice the same."""
    for lengths in ([200, 0, 1, 90], [1500, 0, 16, 17, 333]):
        cache, table, lens, k, v = make(21, lengths, 4, 128, 4, page, t)
        q = ref.normal(22, (len(lengths), 28, 128), t, 2.0)
        scores = torch.rand((len(lengths), 4, 1500), generator=ref.gen(23)).cuda()
        before = scores.clone()
        again = scores.clone()
        got = samd.paged_attention(q, cache, table, lens, scale=0.1, scores=scores)
        check(got, q, table, lengths, k, v, page, 0.1, t, scores, before)
        assert torch.equal(got, samd.paged_attention(q, cache, table, lens, scale=0.1, scores=again))
        assert torch.equal(scores, again)
        assert torch.equal(got, samd.paged_attention(q, cache, table, lens, scale=0.1))


def test_scores_narrower_than_the_pages(samd_lib):
    cache, table, lens, k, v = make(25, [40, 300], 2, 64, 8, 16, F16)
    q = ref.normal(26, (2, 4, 64), F16)
    scores = torch.zeros((2, 2, 301), device="cuda")
    narrow = torch.full((2 * 2 * 100 + 50,), 9.0, device="cuda")
    narrow[:400] = 0
    samd.paged_attention(q, cache, table, lens, scores=scores)
    samd.paged_attention(q, cache, table, lens, scores=narrow[:400].view(2, 2, 100))
    assert torch.equal(narrow[:400].view(2, 2, 100), scores[:, :, :100]) and (narrow[400:] == 9.0).all()


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("n", [1, 16, 64, 256, 512, 4096])
def test_a_mean_is_exact(samd_lib, n, bits, t):
    """q = 0: all weights are 1 / n, a power of two, and with scales of 1/4 .. 2 every sum is exact in fp32 (integers of
    at most 4096 * 128 in quarters): one rounding is left. Also with q's of other magnitudes and orthogonal keys."""
    heads, dim, page = 2, 64, 16
    lanes = 2 ** (bits - 1)
    table, pages = ref.pages_for(31, 1, n // page + 1)
    shape = (pages, heads, page)
    kl, vl = (ref.ints(s, (*shape, dim), -lanes, lanes - 1) for s in (32, 33))
    vs = torch.exp2(ref.ints(34, (*shape, dim // 32), -2, 1).double()).to(t)
    ks = torch.ones_like(vs)
    cache = samd.PagedCache(ref.pack(kl, bits), ks, ref.pack(vl, bits), vs)
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    got = samd.paged_attention(torch.zeros((1, 6, dim), dtype=t, device="cuda"), cache, table, lens)
    mean = ref.gather(ref.values(vl, vs), table, 0, n, page).mean(1)
    assert torch.equal(got[0].view(2, 3, dim), mean[:, None].expand(2, 3, dim).to(t))


@pytest.mark.parametrize("t", [BF16, F16])
def test_one_token_takes_all(samd_lib, t):
    """A key that matches q by far: the others' weights are below 2^-100, and out is that token's value."""
    heads, dim, page, n = 3, 128, 32, 700
    table, pages = ref.pages_for(41, 1, 22)
    shape = (pages, heads, page)
    kl, _ = ref.random_rows(42, shape, dim, 8, t)
    vl, vs = ref.random_rows(43, shape, dim, 8, t, 6.0)
    ks = torch.ones_like(vs)
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    for hit in (0, 15, 16, 350, 699):
        k = kl.clone()
        q = torch.sign(ref.normal(hit, (1, heads, dim), torch.float64))
        k[table[0, hit // page].long(), :, hit % page] = (127 * q[0]).long()
        cache = samd.PagedCache(ref.pack(k, 8), ks, ref.pack(vl, 8), vs)
        got = samd.paged_attention(q.to(t), cache, table, lens, scale=1.0)
        want = ref.gather(ref.values(vl, vs), table, 0, n, page)[:, hit]
        # the weight times the scale is rounded to fp16, and out once more
        assert ((got[0].double() - want).abs() <= (ref.UNIT[t] + 2.0 ** -11 * 1.01) * want.abs()).all()


@pytest.mark.parametrize("t", [BF16, F16])
def test_scales_of_any_size(samd_lib, t):
    """Values whose scales differ by many powers of two, among them tokens of no weight with the largest scales, and
    zero scales; queries of many magnitudes."""
    heads, dim, page, n = 2, 64, 16, 333
    lengths = [n]
    lo, hi = (-60, 60) if t is BF16 else (-10, 5)
    table, pages = ref.pages_for(51, 1, 21)
    shape = (pages, heads, page)
    kl, ks = ref.random_rows(52, shape, dim, 8, t)
    vl, _ = ref.random_rows(53, shape, dim, 8, t)
    vs = torch.exp2(ref.ints(54, (*shape, dim // 32), lo, hi).double())
    vs *= ref.ints(55, tuple(vs.shape), 0, 9) > 0
    vs = vs.to(t)
    cache = samd.PagedCache(ref.pack(kl, 8), ks, ref.pack(vl, 8), vs)
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    k, v = ref.values(kl, ks), ref.values(vl, vs)
    for size in (1e-30, 1e-3, 1.0, 20.0, 1e15) if t is BF16 else (1e-6, 1e-3, 1.0, 20.0, 4e3):
        q = ref.normal(56, (1, 4, dim), torch.float64).mul_(size).to(t)
        scale = 1.0 if size <= 20 else 20.0 / size
        check(samd.paged_attention(q, cache, table, lens, scale=scale), q, table, lengths, k, v, page, scale, t)
    check(samd.paged_attention(q, cache, table, lens, scale=-scale), q, table, lengths, k, v, page, -scale, t)
    check(samd.paged_attention(q, cache, table, lens, scale=0.0), q, table, lengths, k, v, page, 0.0, t)


def test_pages_that_are_none_hold_no_tokens(samd_lib):
    """Tokens of a page that the table does not name are left out; a sequence with none left gives zeros."""
    lengths, page = [100, 40, 600], 16
    cache, table, lens, k, v = make(61, lengths, 2, 64, 8, page, BF16)
    table = table.clone()
    gone = {0: [0, 3, 6], 1: [0, 1, 2], 2: list(range(0, 37, 2))}
    bad = [-1, 1 << 30, cache.k_lanes.shape[0], -(1 << 31)]
    good = table.clone()
    for b, pages in gone.items():
        for i, p in enumerate(pages):
            table[b, p] = bad[i % 4]
    q = ref.normal(62, (3, 4, 64), BF16)
    scores = torch.zeros((3, 2, 608), device="cuda")
    got = samd.paged_attention(q, cache, table, lens, scores=scores)
    for b, n in enumerate(lengths):
        keep = torch.tensor([t for t in range(n) if t // page not in gone[b]], dtype=torch.int64, device="cuda")
        if len(keep) == 0:
            assert not got[b].any() and not scores[b].any()
            continue
        kb, vb = (ref.gather(x, good, b, n, page)[:, keep] for x in (k, v))
        want, p, x = ref.attention(q[b], kb, vb, 0.125)
        bound, delta = ref.attention_bound(q[b], kb, vb, 0.125, p, x, want, BF16)
        assert ((got[b].double() - want).abs() <= bound).all()
        w = p.view(2, 2, -1).sum(1)
        assert ((scores[b][:, keep].double() - w).abs() <= 3 * float(delta.max()) * w + 1e-30).all()
        other = torch.ones(608, dtype=torch.bool, device="cuda")
        other[keep] = False
        assert not scores[b][:, other].any()


def test_lengths_past_the_pages_and_below_zero(samd_lib):
    cache, table, lens, k, v = make(65, [320, 320, 320], 2, 64, 8, 16, BF16)
    q = ref.normal(66, (3, 2, 64), BF16)
    far = torch.tensor([(1 << 31) - 1, 320, -5], dtype=torch.int32, device="cuda")
    got, plain = samd.paged_attention(q, cache, table, far), samd.paged_attention(q, cache, table, lens)
    check(got, q, table, [320, 320, 0], k, v, 16, 0.125, BF16)
    assert torch.isfinite(plain).all()
    no_pages = samd.paged_attention(q, cache, table[:, :0], lens)
    assert no_pages.shape == q.shape and not no_pages.any()


def test_infinities_and_nans_stay_in_their_head(samd_lib):
    lengths = [50, 700]
    cache, table, lens, k, v = make(71, lengths, 3, 64, 8, 16, BF16)
    q = ref.normal(72, (2, 6, 64), BF16)
    clean = samd.paged_attention(q, cache, table, lens)
    for where, value in (("q", math.nan), ("q", math.inf), ("k", math.nan), ("v", math.nan), ("v", math.inf)):
        q2 = q.clone()
        c2 = samd.PagedCache(*(x.clone() for x in (cache.k_lanes, cache.k_scales, cache.v_lanes, cache.v_scales)))
        hit = torch.zeros((2, 6), dtype=torch.bool, device="cuda")
        if where == "q":
            q2[1, 3, 5] = value
            hit[1, 3] = True
        else:
            (c2.k_scales if where == "k" else c2.v_scales)[table[1, 2].long(), 1, 7] = value
            hit[1, 2:4] = True
        got = samd.paged_attention(q2, c2, table, lens)
        assert torch.equal(got[~hit], clean[~hit])
        assert not torch.isfinite(got[hit]).all(-1).any()


def test_shared_pages_and_the_same_sequence_twice(samd_lib):
    """Sequences that share a prefix's pages; the result of one does not depend on where its pages lie."""
    cache, table, lens, k, v = make(75, [333, 333], 2, 128, 4, 16, F16)
    table = table.clone()
    table[1, :20] = table[0, :20]
    lens[1] = 320
    q = ref.normal(76, (2, 8, 128), F16)
    check(samd.paged_attention(q, cache, table, lens), q, table, [333, 320], k, v, 16, 128 ** -0.5, F16)
    twice = samd.paged_attention(torch.cat((q[:1], q[:1])), cache, table[:1].repeat(2, 1), lens[:1].repeat(2))
    check(twice, torch.cat((q[:1], q[:1])), table[:1].repeat(2, 1), [333, 333], k, v, 16, 128 ** -0.5, F16)


def test_strides_streams_graphs_and_repeats(samd_lib):
    """q and out as parts of wider rows; a side stream; two captured graphs that share a workspace and are replayed in
    turn with other lengths; the same call twice gives the same bits."""
    heads, group, dim, page = 2, 4, 64, 16
    lengths = [900, 0, 37, 444]
    cache, table, lens, k, v = make(81, lengths, heads, dim, 8, page, BF16, capacity=1024)
    n = heads * group * dim
    wide = ref.normal(82, (4, 3 * n), BF16)
    q = wide[:, n:2 * n].view(4, heads * group, dim)
    first = samd.paged_attention(q, cache, table, lens)
    check(first, q, table, lengths, k, v, page, 0.125, BF16)
    assert all(torch.equal(first, samd.paged_attention(q, cache, table, lens)) for _ in range(5))
    out = torch.full((4, n + 16), 3.0, dtype=BF16, device="cuda")
    samd.paged_attention(q, cache, table, lens, out=out[:, 8:n + 8].view(4, heads * group, dim))
    assert torch.equal(out[:, 8:n + 8].reshape(first.shape), first) and (out[:, :8] == 3).all() and (out[:, n + 8:] == 3).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = samd.paged_attention(q, cache, table, lens, stream=side)
    side.synchronize()
    assert torch.equal(first, y)
    cd = cache._desc
    s = samd._cache_seqs(table, lens)
    ws = torch.full((samd.samd_paged_attention_workspace_size(cd, s, heads * group, True),), 0xAB, dtype=torch.uint8, device="cuda")
    outs, graphs = [torch.zeros_like(first) for _ in range(2)], []
    scores = torch.zeros((4, heads, 1024), device="cuda")
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            samd.paged_attention(q, cache, table, lens, out=outs[i], workspace=ws, scores=scores if i else None)
        graphs.append(g)
    for new in ([900, 0, 37, 444], [1, 20, 37, 100], [0, 0, 0, 0], [899, 0, 30, 17]):
        new = [min(a, b) for a, b in zip(new, lengths)]
        lens.copy_(torch.tensor(new, dtype=torch.int32))
        scores.zero_()
        for o in outs:
            o.fill_(7.0)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for o in outs:
            check(o, q, table, new, k, v, page, 0.125, BF16, scores, torch.zeros_like(scores))
        assert torch.equal(outs[0], outs[1])
    assert_status_clean()


def test_a_cache_without_pages(samd_lib):
    cache = samd.cache_empty(0, 16, 2, 64, 8, BF16)
    table, lens = torch.zeros((3, 40), dtype=torch.int32, device="cuda"), torch.tensor([0, 5, 600], dtype=torch.int32, device="cuda")
    q, k = ref.normal(92, (3, 4, 64), BF16), ref.normal(93, (3, 2, 64), BF16)
    scores = torch.ones((3, 2, 640), device="cuda")
    assert not samd.paged_attention(q, cache, table, lens, scores=scores).any() and (scores == 1).all()
    samd.cache_append(cache, k, k, table, lens)
    assert not samd.cache_read(cache, 3, table, lens)[0].any()


@pytest.mark.parametrize("lengths", [[1] * 40, [3] * 7 + [0] * 30, [20, 1, 1, 1, 1000, 1], [17] * 300], ids=lambda n: f"{len(n)}x{n[0]}")
def test_short_sequences_in_long_tables(samd_lib, lengths):
    """Fewer steps than a CTA's warps for a head, in tables with room for many."""
    cache, table, lens, k, v = make(95, lengths, 3, 64, 8, 16, F16, capacity=1500)
    q = ref.normal(96, (len(lengths), 6, 64), F16)
    scores = torch.zeros((len(lengths), 3, 1500), device="cuda")
    got = samd.paged_attention(q, cache, table, lens, scores=scores)
    check(got, q, table, lengths, k, v, 16, 0.125, F16, scores, torch.zeros_like(scores))


def test_empty_calls(samd_lib):
    cache, table, lens, k, v = make(91, [5], 2, 64, 8, 16, BF16)
    q = torch.empty((0, 4, 64), dtype=BF16, device="cuda")
    assert samd.paged_attention(q, cache, table[:0], lens[:0]).shape == (0, 4, 64)


@pytest.mark.slow
@pytest.mark.parametrize("bits", [4, 8])
def test_long_sequences_past_two_to_the_31(samd_lib, bits):
    """One sequence of 300000 tokens, and offsets past 2^31 bytes: pages at both ends of a cache of 2.4 GB."""
    heads, dim, page, n, t = 2, 256, 64, 300000, BF16
    width = -(-n // page)
    pages = (1 << 31) // (heads * page * dim * bits // 8) + 600
    table = torch.cat((torch.arange(width // 2), torch.arange(pages - (width - width // 2), pages)))[None].to("cuda", torch.int32)
    g = torch.Generator(device="cuda").manual_seed(3)
    words = dim * bits // 32
    lanes = [torch.randint(-(1 << 31), (1 << 31) - 1, (pages, heads, page, words), dtype=torch.int32, device="cuda", generator=g) for _ in range(2)]
    scales = [(torch.rand((pages, heads, page, dim // 32), device="cuda", generator=g) + 0.5).mul_(0.01).to(t) for _ in range(2)]
    cache = samd.PagedCache(lanes[0], scales[0], lanes[1], scales[1])
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    q = ref.normal(4, (1, 10, dim), t)
    got = samd.paged_attention(q, cache, table, lens)
    for h in range(heads):
        kv = []
        for x, s in zip(lanes, scales):
            x, s = x[table[0].long(), h].flatten(0, 1)[:n], s[table[0].long(), h].flatten(0, 1)[:n]
            kv.append(ref.values(ref.unpack(x, bits), s)[None])
        want, p, x = ref.attention(q[0, 5 * h:5 * h + 5], *kv, 1 / 16)
        bound, _ = ref.attention_bound(q[0, 5 * h:5 * h + 5], *kv, 1 / 16, p, x, want, t)
        assert ((got[0, 5 * h:5 * h + 5].double() - want).abs() <= bound).all()
