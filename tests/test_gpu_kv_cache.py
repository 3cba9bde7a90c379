"""samd_cache_append and samd_cache_read against the definition, bit for bit."""
import math

import pytest
import torch

import cache_ref as ref
from gpu_util import assert_status_clean
from paper_1809_10572_gb300 import samd

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def new_cache(pages, page, heads, dim, bits, t):
    """A cache of patterns that are no valid row's."""
    c = samd.cache_empty(pages, page, heads, dim, bits, t)
    for x in (c.k_lanes, c.v_lanes):
        x.fill_(0x5A5A5A5A)
    for x in (c.k_scales, c.v_scales):
        x.fill_(-123.0)
    return c


def fill(c, k, v, table, lengths, starts):
    """What the cache holds afterwards, by the definition: (k_lanes, k_scales, v_lanes, v_scales)."""
    out = [x.clone() for x in (c.k_lanes, c.k_scales, c.v_lanes, c.v_scales)]
    kl, ks = ref.quantize(k, c.bits)
    vl, vs = ref.quantize(v, c.bits)
    rows = (ref.pack(kl, c.bits), ks, ref.pack(vl, c.bits), vs)
    for b, n in enumerate(lengths.tolist()):
        first, last = starts[b], starts[b + 1]
        for token in range(first, last):
            pos = n - (last - token)
            if pos < 0 or pos >= table.shape[1] * c.page:
                continue
            page = int(table[b, pos // c.page])
            if 0 <= page < c.k_lanes.shape[0]:
                for o, r in zip(out, rows):
                    o[page, :, pos % c.page] = r[token]
    return out


def same(c, want):
    for got, w in zip((c.k_lanes, c.k_scales, c.v_lanes, c.v_scales), want):
        if got.dtype is torch.int32:
            assert torch.equal(got, w)
        else:
            assert torch.equal(torch.isnan(got), torch.isnan(w)) and torch.equal(torch.nan_to_num(got), torch.nan_to_num(w))


def rows(seed, tokens, heads, dim, t):
    """Rows of every magnitude, with zeros and with values that lie half way between two lanes."""
    x = ref.normal(seed, (tokens, heads, dim), torch.float64)
    x *= torch.exp2(ref.ints(seed + 1, (tokens, heads, dim // 32, 1), -6, 6).double()).expand(-1, -1, -1, 32).flatten(-2)
    x[:, :, :32] *= (ref.ints(seed + 2, (tokens, heads, 1), 0, 3) > 0)  # some blocks of zeros
    if dim >= 64:  # 7 or 127 is the largest of a block: its scale is 1, and halves are ties
        x[:, :, 32:64] = ref.ints(seed + 3, (tokens, heads, 32), -14, 14).double() / 2
        x[::2, :, 40] = 7.0
        x[1::2, :, 40] = 127.0
    return x.to(t)


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("heads,dim,page", [(1, 32, 16), (3, 64, 32), (8, 128, 16), (2, 96, 64), (5, 160, 16), (1, 192, 256), (2, 224, 16), (2, 256, 128)])
def test_append_and_read(samd_lib, heads, dim, page, bits, t):
    lengths = torch.tensor([37, 0, 16, 1, 50, 33], dtype=torch.int32, device="cuda")
    new = [37, 0, 3, 1, 17, 1]
    starts = [sum(new[:i]) for i in range(7)]
    table, pages = ref.pages_for(1, 6, -(-50 // page), more=2)
    c = new_cache(pages, page, heads, dim, bits, t)
    k, v = rows(11, starts[-1], heads, dim, t), rows(21, starts[-1], heads, dim, t)
    want = fill(c, k, v, table, lengths, starts)
    s = torch.tensor(starts, dtype=torch.int32, device="cuda")
    samd.cache_append(c, k, v, table, lengths, s)
    same(c, want)
    got = samd.cache_read(c, starts[-1], table, lengths, s)
    for g, x in zip(got, (k, v)):
        lanes, scales = ref.quantize(x, bits)
        assert torch.equal(g, ref.values(lanes, scales).to(t))
    assert_status_clean()


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("bits", [4, 8])
def test_one_token_each_without_starts(samd_lib, bits, t):
    """A decoding step of a padded batch: sequences of length 0 (and below) are left out, and read as zeros."""
    lengths = torch.tensor([1, 0, 16, 17, -3, 48, 49], dtype=torch.int32, device="cuda")
    table, pages = ref.pages_for(2, 7, 3)
    c = new_cache(pages, 16, 2, 64, bits, t)
    k, v = rows(31, 7, 2, 64, t), rows(41, 7, 2, 64, t)
    want = fill(c, k, v, table, lengths, list(range(8)))
    samd.cache_append(c, k, v, table, lengths)
    same(c, want)  # 49 tokens are more than the pages hold: that one is left out too
    gk, gv = samd.cache_read(c, 7, table, lengths)
    for g, x in ((gk, k), (gv, v)):
        q = ref.values(*ref.quantize(x, bits)).to(t)
        q[[1, 4, 6]] = 0
        assert torch.equal(g, q)


def test_rows_of_no_sequence_and_pages_that_are_none(samd_lib):
    lengths = torch.tensor([20, 34], dtype=torch.int32, device="cuda")
    table = torch.tensor([[1, -1, 7], [3, 9999999, 0]], dtype=torch.int32, device="cuda")
    c = new_cache(5, 16, 2, 64, 8, BF16)
    starts = [2, 12, 30]
    k, v = rows(51, 34, 2, 64, BF16), rows(61, 34, 2, 64, BF16)
    want = fill(c, k, v, table, lengths, starts)
    s = torch.tensor(starts, dtype=torch.int32, device="cuda")
    samd.cache_append(c, k, v, table, lengths, s)
    same(c, want)
    gk, gv = (torch.full_like(k, 5.0) for _ in range(2))
    samd.cache_read(c, 34, table, lengths, s, k=gk, v=gv)
    q = ref.values(*ref.quantize(k, 8)).to(BF16)
    q[:2], q[30:] = 5.0, 5.0       # of no sequence: left as they are
    q[8:12] = 0                    # tokens 16 .. 19 of the first lie in page -1
    q[12:28] = 0                   # 16 .. 31 of the second in page 9999999
    assert torch.equal(gk, q)


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("bits", [4, 8])
def test_infinities_nans_and_the_smallest_values(samd_lib, bits, t):
    table, pages = ref.pages_for(3, 1, 1)
    lengths = torch.tensor([6], dtype=torch.int32, device="cuda")
    s = torch.tensor([0, 6], dtype=torch.int32, device="cuda")
    k = ref.normal(71, (6, 1, 64), t)
    k[0, 0, 3], k[1, 0, 40], k[2, 0, 0] = math.inf, math.nan, -math.inf
    big = torch.finfo(t).max
    k[3, 0, :32] = big
    k[3, 0, 5:9] = -big / 2
    tiny = torch.finfo(t).smallest_normal * torch.finfo(t).eps  # the smallest above zero
    k[4, 0, :32] = tiny * torch.arange(32, device="cuda")
    k[4, 0, 32:] = -tiny * 300 * torch.arange(32, device="cuda")
    k[5] = torch.finfo(t).smallest_normal
    v = -k.flip(-1)
    c = new_cache(pages, 16, 1, 64, bits, t)
    want = fill(c, k, v, table, lengths, [0, 6])
    samd.cache_append(c, k, v, table, lengths, s)
    same(c, want)
    g, _ = samd.cache_read(c, 6, table, lengths, s)
    q = ref.values(*ref.quantize(k, bits)).to(t)
    assert torch.equal(torch.isnan(g), torch.isnan(q)) and torch.equal(torch.nan_to_num(g), torch.nan_to_num(q))


def test_strides_streams_and_graphs(samd_lib):
    """Keys and values as parts of one projection's rows; another stream; a captured step replayed with other lengths."""
    heads, dim, t = 3, 64, BF16
    table, pages = ref.pages_for(4, 5, 2)
    lengths = torch.tensor([1, 9, 32, 0, 17], dtype=torch.int32, device="cuda")
    qkv = ref.normal(81, (5, 5 * heads * dim), t)
    k = qkv[:, 2 * heads * dim:3 * heads * dim].view(5, heads, dim)
    v = qkv[:, 4 * heads * dim:].view(5, heads, dim)
    c, d = new_cache(pages, 16, heads, dim, 4, t), new_cache(pages, 16, heads, dim, 4, t)
    want = fill(c, k, v, table, lengths, list(range(6)))
    wide = torch.zeros((5, 7 + 1), dtype=torch.int32, device="cuda")
    wide[:, :2] = table
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    samd.cache_append(c, k, v, wide[:, :2], lengths, stream=side)
    side.synchronize()
    same(c, want)
    out = [torch.zeros((5, 2 * heads * dim), dtype=t, device="cuda") for _ in range(2)]
    views = [o[:, heads * dim:].view(5, heads, dim) for o in out]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        samd.cache_append(d, k, v, table, lengths)
        samd.cache_read(d, 5, table, lengths, k=views[0], v=views[1])
    for step in range(3):
        lengths.add_(1)
        qkv.copy_(ref.normal(90 + step, tuple(qkv.shape), t))
        want = fill(d, k, v, table, lengths, list(range(6)))
        g.replay()
        torch.cuda.synchronize()
        same(d, want)
        q = ref.values(*ref.quantize(v, 4)).to(t)
        q[2] = 0  # its pages are full
        assert torch.equal(views[1], q) and not out[1][:, :heads * dim].any()


def test_empty_calls(samd_lib):
    c = new_cache(1, 16, 2, 64, 8, BF16)
    none = torch.empty((0, 2, 64), dtype=BF16, device="cuda")
    table, lengths = torch.empty((0, 3), dtype=torch.int32, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    samd.cache_append(c, none, none, table, lengths)
    assert samd.cache_read(c, 0, table, lengths)[0].shape == (0, 2, 64)


@pytest.mark.slow
def test_offsets_past_two_to_the_31(samd_lib):
    """A cache of 2.4 GB of lanes: its first and last pages."""
    pages, page, heads, dim, t = 9400, 64, 16, 256, BF16
    c = samd.cache_empty(pages, page, heads, dim, 8, t)
    assert c.k_lanes.numel() * 4 > 1 << 31
    table = torch.tensor([[0, pages - 1]], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([2 * page], dtype=torch.int32, device="cuda")
    s = torch.tensor([0, 2 * page], dtype=torch.int32, device="cuda")
    k, v = (ref.normal(n, (2 * page, heads, dim), t) for n in (5, 6))
    samd.cache_append(c, k, v, table, lengths, s)
    for x, lanes, scales in ((k, c.k_lanes, c.k_scales), (v, c.v_lanes, c.v_scales)):
        ql, qs = ref.quantize(x, 8)
        for i, p in enumerate((0, pages - 1)):
            part = slice(i * page, (i + 1) * page)
            assert torch.equal(lanes[p].transpose(0, 1), ref.pack(ql[part], 8)) and torch.equal(scales[p].transpose(0, 1), qs[part])
    got = samd.cache_read(c, 2 * page, table, lengths, s)
    assert torch.equal(got[0], ref.values(*ref.quantize(k, 8)).to(t))
