"""samd_cache_evict against a sort of the scores: places, lengths, scores and rows, all bit for bit. And the cache's
operators together, as a decoder uses them."""
import math

import pytest
import torch

import cache_ref as ref
from gpu_util import assert_status_clean
from paper_1809_10572_gb300 import samd

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def chosen(row, n, keep, recent):
    """The kept places of one head: row is its scores as Python floats."""
    if n <= keep:
        return list(range(n))
    old = n - recent
    low = -math.inf
    order = sorted(range(old), key=lambda i: (row[i] != row[i], -(row[i] if row[i] == row[i] else low), i))
    return sorted(order[:keep - recent] + list(range(old, n)))


def setup(seed, lengths, heads, dim, bits, page, t, keep, capacity):
    width, more = -(-capacity // page), -(-keep // page)
    seqs = len(lengths)
    order, pages = ref.pages_for(seed, seqs, width + more)
    table, dst = order[:, :width].contiguous(), order[:, width:].contiguous()
    shape = (pages, heads, page)
    words = dim * bits // 32
    g = torch.Generator(device="cuda").manual_seed(seed)

    def lanes():
        return torch.randint(-(1 << 31), (1 << 31) - 1, (*shape, words), dtype=torch.int32, device="cuda", generator=g)

    def scales():
        return torch.rand((*shape, dim // 32), device="cuda", generator=g).to(t)

    return samd.PagedCache(lanes(), scales(), lanes(), scales()), table, dst, torch.tensor(lengths, dtype=torch.int32, device="cuda")


def check(cache, table, dst, lens, scores, keep, recent, **kw):
    lengths, page = lens.tolist(), cache.page
    before = [x.clone() for x in (cache.k_lanes, cache.k_scales, cache.v_lanes, cache.v_scales)]
    want = [x.clone() for x in before]
    kept, new, got = samd.cache_evict(cache, table, lens, scores, dst, keep, recent, **kw)
    assert kept.shape == got.shape == (len(lengths), cache.heads, keep)
    assert new.tolist() == [min(max(n, 0), keep) for n in lengths]
    wide = torch.zeros((*scores.shape[:2], max(max(lengths), 1)), device="cuda")
    wide[..., :min(wide.shape[2], scores.shape[2])] = scores[..., :wide.shape[2]]
    rows = wide.tolist()
    want_kept = torch.full_like(kept, -1)
    want_scores = torch.zeros_like(got)
    for b, n in enumerate(lengths):
        for h in range(cache.heads):
            at = torch.tensor(chosen(rows[b][h], max(n, 0), keep, recent), dtype=torch.int64, device="cuda")
            to = torch.arange(len(at), device="cuda")
            want_kept[b, h, :len(at)] = at.int()
            want_scores[b, h, :len(at)] = wide[b, h, at]
            src, d = table[b, at // page].long(), dst[b, to // page].long()
            for w, x in zip(want, before):
                w[d, h, to % page] = x[src, h, at % page]
    assert torch.equal(kept, want_kept)
    assert torch.equal(torch.nan_to_num(got, nan=-1.5), torch.nan_to_num(want_scores, nan=-1.5))
    for x, w in zip((cache.k_lanes, cache.k_scales, cache.v_lanes, cache.v_scales), want):
        assert torch.equal(x, w)
    assert_status_clean()
    return kept, new, got


def some_scores(seed, shape):
    """Heavy-tailed weights, many of them zero, many equal, some below zero, infinite or NaN."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    w = torch.rand(shape, device="cuda", generator=g)
    s = torch.exp(9 * torch.rand(shape, device="cuda", generator=g)) * (w > 0.3)
    s = torch.where(w > 0.8, torch.round(s / 100) * 100, s)
    for i, v in enumerate((-1.0, -0.0, math.inf, -math.inf, math.nan, 1e-42, 3e38)):
        s = torch.where((w > 0.31 + 0.01 * i) & (w < 0.313 + 0.01 * i), torch.full_like(s, v), s)
    return s


@pytest.mark.parametrize("lengths,heads,keep,recent", [
    ([1], 1, 1, 0), ([2], 1, 1, 0), ([2], 1, 1, 1), ([100, 0, 33, 7], 3, 33, 5), ([100, 0, 33, 34], 2, 33, 33),
    ([600, 599], 4, 256, 64), ([513, 512, 511], 1, 512, 0), ([8192, 8193, 100], 2, 2048, 200), ([9000], 2, 8999, 17),
    ([20000, 3], 3, 77, 0), ([50000, 65536], 2, 4096, 4095), ([65537, 1000], 1, 1000, 1), ([150000, 70001], 2, 30000, 999)], ids=str)
def test_places_and_rows(samd_lib, lengths, heads, keep, recent):
    cache, table, dst, lens = setup(1, lengths, heads, 64, 8, 64, BF16, keep, max(lengths))
    check(cache, table, dst, lens, some_scores(2, (len(lengths), heads, max(lengths))), keep, recent)


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dim,page", [(32, 16), (64, 32), (96, 16), (128, 128), (160, 16), (192, 64), (224, 16), (256, 16)])
def test_row_sizes(samd_lib, dim, page, bits, t):
    lengths = [90, 0, 41, 200]
    cache, table, dst, lens = setup(dim, lengths, 2, dim, bits, page, t, 40, 200)
    check(cache, table, dst, lens, some_scores(3, (4, 2, 200)), 40, 8)


@pytest.mark.parametrize("value", [0.0, 1.0, -2.0, math.nan, math.inf])
@pytest.mark.parametrize("n", [1000, 30000, 100000])
def test_all_scores_equal(samd_lib, n, value):
    """Ties go to the earlier token."""
    cache, table, dst, lens = setup(5, [n], 2, 32, 4, 64, BF16, 300, n)
    kept, _, _ = check(cache, table, dst, lens, torch.full((1, 2, n), value, device="cuda"), 300, 100)
    assert kept[0, 0].tolist() == list(range(200)) + list(range(n - 100, n))


def test_scores_narrower_or_wider_than_the_lengths(samd_lib):
    cache, table, dst, lens = setup(7, [500, 300], 2, 64, 8, 16, F16, 100, 512)
    for width in (0, 1, 150, 301, 900):
        check(cache, table, dst, lens, some_scores(8, (2, 2, width)), 100, 10)


def test_lengths_past_the_pages_and_below_zero(samd_lib):
    cache, table, dst, lens = setup(9, [512, 512, 512], 2, 64, 8, 16, BF16, 100, 512)
    s = some_scores(10, (3, 2, 512))
    whole = check(cache, table, dst, lens, s, 100, 10)
    lens[1], lens[2] = (1 << 31) - 1, -7
    kept, new, _ = samd.cache_evict(cache, table, lens, s, dst, 100, 10)
    assert torch.equal(kept[:2], whole[0][:2]) and (kept[2] == -1).all() and new.tolist() == [100, 100, 0]


def test_pages_that_are_none(samd_lib):
    """A row whose old or new page is none of the cache's is not copied; nothing else is touched."""
    cache, table, dst, lens = setup(11, [200], 1, 64, 8, 16, BF16, 64, 200)
    s = some_scores(12, (1, 1, 200))
    good_table, good_dst = table.clone(), dst.clone()
    table[0, 3], table[0, 12], dst[0, 1] = -1, 1 << 30, cache.k_lanes.shape[0]
    before = cache.k_lanes.clone()
    kept, _, _ = samd.cache_evict(cache, table, lens, s, dst, 64, 9)
    want = before.clone()
    for i, at in enumerate(kept[0, 0].tolist()):
        if at // 16 not in (3, 12) and i // 16 != 1:
            want[good_dst[0, i // 16], 0, i % 16] = before[good_table[0, at // 16], 0, at % 16]
    assert torch.equal(cache.k_lanes, want)


def test_streams_graphs_and_repeats(samd_lib):
    cache, table, dst, lens = setup(13, [3000, 9000, 0], 3, 128, 4, 32, BF16, 1024, 9000)
    s = some_scores(14, (3, 3, 9000))
    first = check(cache, table, dst, lens, s, 1024, 100)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(map(torch.nan_to_num, first), map(torch.nan_to_num, samd.cache_evict(cache, table, lens, s, dst, 1024, 100))))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = samd.cache_evict(cache, table, lens, s, dst, 1024, 100, stream=side)
    side.synchronize()
    assert torch.equal(first[0], other[0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        kept, new, scores = samd.cache_evict(cache, table, lens, s, dst, 1024, 100)
    for seed, n in ((15, [500, 8000, 1025]), (16, [3000, 1024, 9000])):
        s.copy_(some_scores(seed, (3, 3, 9000)))
        lens.copy_(torch.tensor(n, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        want = check(cache, table, dst, lens, s, 1024, 100)
        assert torch.equal(kept, want[0]) and torch.equal(new, want[1])


def test_empty_calls(samd_lib):
    cache, table, dst, lens = setup(17, [5], 2, 64, 8, 16, BF16, 3, 16)
    kept, new, s = samd.cache_evict(cache, table[:0], lens[:0], torch.zeros((0, 2, 16), device="cuda"), dst[:0], 3)
    assert kept.shape == s.shape == (0, 2, 3) and new.shape == (0,)


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("bits", [4, 8])
def test_a_decoder_with_a_bounded_cache(samd_lib, bits, t):
    """Prompts, then tokens one by one with attention that counts weights; when a sequence reaches its budget all are cut
    down, and decoding goes on from the kept tokens. A plain list of (key, value, score) rows follows each head."""
    heads, group, dim, page, budget, keep, recent = 2, 3, 64, 16, 80, 48, 8
    prompts = [70, 3, 33]
    seqs = len(prompts)
    width = budget // page
    order, pages = ref.pages_for(21, seqs, 2 * width)
    table, spare = order[:, :width].contiguous(), order[:, width:].contiguous()
    cache = samd.cache_empty(pages, page, heads, dim, bits, t)
    lens = torch.tensor(prompts, dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, 70, 73, 106], dtype=torch.int32, device="cuda")
    k, v = (ref.normal(s, (106, heads, dim), t) for s in (22, 23))
    samd.cache_append(cache, k, v, table, lens, starts)
    scores = torch.zeros((seqs, heads, budget), device="cuda")
    rk, rv = (ref.values(*ref.quantize(x, bits)) for x in (k, v))
    book = [[[rk[starts[b]:starts[b + 1], h], rv[starts[b]:starts[b + 1], h]] for h in range(heads)] for b in range(seqs)]
    evicted = 0
    for step in range(60):
        lens.add_(1)
        k, v, q = (ref.normal(100 + 3 * step + i, (seqs, heads * (group if i == 2 else 1), dim), t) for i in range(3))
        samd.cache_append(cache, k, v, table, lens)
        rk, rv = (ref.values(*ref.quantize(x, bits)) for x in (k, v))
        before = scores.clone()
        out = samd.paged_attention(q, cache, table, lens, scores=scores)
        for b in range(seqs):
            for h in range(heads):
                row = book[b][h]
                row[0], row[1] = torch.cat((row[0], rk[b, h][None])), torch.cat((row[1], rv[b, h][None]))
                mine = q[b, h * group:(h + 1) * group]
                want, p, x = ref.attention(mine, row[0][None], row[1][None], dim ** -0.5)
                bound, delta = ref.attention_bound(mine, row[0][None], row[1][None], dim ** -0.5, p, x, want, t)
                assert ((out[b, h * group:(h + 1) * group].double() - want).abs() <= bound).all()
                n = row[0].shape[0]
                added = (scores[b, h, :n].double() - before[b, h, :n].double())
                assert ((added - p.sum(0)).abs() <= 4 * float(delta.max()) + 1e-5).all()
        if int(lens.max()) == budget:
            kept, lens, new = samd.cache_evict(cache, table, lens, scores, spare, keep, recent)
            for b in range(seqs):
                for h in range(heads):
                    n = book[b][h][0].shape[0]
                    at = chosen(scores[b, h, :n].tolist(), n, keep, recent)
                    assert kept[b, h, :len(at)].tolist() == at
                    book[b][h] = [x[at] for x in book[b][h]]
            scores = torch.zeros_like(scores)
            scores[..., :keep] = new
            table, spare = spare, table
            evicted += 1
    assert evicted == 2
    assert_status_clean()
