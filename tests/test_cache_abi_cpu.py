"""Refusals of the packed cache's entry points, answered on the host before any launch (addresses here are never read), and
the binding's own checks."""
import ctypes

import pytest
import torch

from paper_1809_10572_gb300 import samd

OK, EINVAL, EALIGN, ESHAPE, EUNSUP = range(5)
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return samd.load()


def cache(pages=4, page=16, heads=2, dim=64, fmt=None, type=samd.SAMD_BF16, kl=16, ks=16, vl=16, vs=16):
    return samd.samd_cache(pages, page, heads, dim, fmt or samd.cache_fmt(8), type, kl, ks, vl, vs)


def seqs(seqs=3, max_pages=2, ld=2, table=16, lengths=16):
    return samd.samd_cache_seqs(seqs, max_pages, ld, table, lengths)


BAD_CACHES = [(dict(type=samd.SAMD_F32), EINVAL), (dict(type=9), EINVAL), (dict(fmt=samd.fmt(4, True, 0, 16)), EINVAL),
              (dict(fmt=samd.fmt(8, False)), EUNSUP), (dict(fmt=samd.fmt(6, True)), EUNSUP),
              (dict(fmt=samd.fmt(4, True, 1)), EUNSUP), (dict(fmt=samd.fmt(4, True, 0, 64)), EUNSUP),
              (dict(pages=-1), ESHAPE), (dict(page=0), ESHAPE), (dict(heads=0), ESHAPE), (dict(dim=0), ESHAPE),
              (dict(page=8), EUNSUP), (dict(page=24), EUNSUP), (dict(page=1 << 17), EUNSUP), (dict(dim=48), EUNSUP),
              (dict(dim=288), EUNSUP), (dict(heads=65537), EUNSUP), (dict(heads=1 << 16, page=1 << 15), EUNSUP)]
BAD_SEQS = [(dict(seqs=-1), ESHAPE), (dict(max_pages=-1), ESHAPE), (dict(ld=1), ESHAPE),
            (dict(max_pages=1 << 27, ld=1 << 27), EUNSUP), (dict(seqs=1 << 30), EUNSUP),
            (dict(seqs=1 << 28, max_pages=1 << 26, ld=1 << 26), EUNSUP)]
BAD_ADDRESSES = [(dict(kl=None), {}, EINVAL), (dict(vs=None), {}, EINVAL), (dict(ks=8), {}, EALIGN), (dict(vl=4), {}, EALIGN),
                 ({}, dict(table=None), EINVAL), ({}, dict(lengths=None), EINVAL), ({}, dict(table=6), EALIGN),
                 ({}, dict(lengths=9), EALIGN)]


def check_both(call):
    assert call(null=True) == EINVAL
    for kw, status in BAD_CACHES:
        assert call(cache(**kw)) == status, kw
    for kw, status in BAD_SEQS:
        assert call(s=seqs(**kw)) == status, kw
    for kc, ks, status in BAD_ADDRESSES:
        assert call(cache(**kc), seqs(**ks)) == status, (kc, ks)


@pytest.mark.parametrize("name", ["samd_cache_append", "samd_cache_read"])
def test_rows_refusals(lib, name):
    def call(c=None, s=None, starts=16, tokens=5, k=16, ldk=128, v=16, ldv=128, null=False):
        return getattr(lib, name)(None if null else ctypes.byref(c or cache()), ctypes.byref(s or seqs()), starts, tokens,
                                  k, ldk, v, ldv, None)

    check_both(call)
    for kw in (dict(tokens=-1), dict(ldk=120), dict(ldv=127), dict(starts=None, tokens=4), dict(ldk=1 << 61, tokens=1 << 20)):
        assert call(**kw) == ESHAPE, kw
    assert call(ldk=132) == EALIGN and call(ldv=129) == EALIGN
    assert call(tokens=0, k=None, v=None) == OK and call(s=seqs(seqs=0), tokens=0, k=None, v=None, starts=None) == OK
    for kw in (dict(k=None), dict(v=None)):
        assert call(**kw) == EINVAL
    for kw in (dict(k=8), dict(v=4), dict(starts=2)):
        assert call(**kw) == EALIGN


def test_attention_refusals(lib):
    def call(c=None, s=None, q_heads=4, q=16, ldq=256, scale=1.0, out=16, ldo=256, scores=None, lds=0, ws=16, nb=BIG, null=False):
        return lib.samd_paged_attention(None if null else ctypes.byref(c or cache()), ctypes.byref(s or seqs()), q_heads, q,
                                        ldq, scale, out, ldo, scores, lds, ws, nb, None)

    check_both(call)
    for q_heads in (0, -2, 3, 5):
        assert call(q_heads=q_heads) == ESHAPE
    assert call(q_heads=514, ldq=1 << 20, ldo=1 << 20) == EUNSUP
    for scale in (float("inf"), float("-inf"), float("nan")):
        assert call(scale=scale) == EINVAL
    for kw in (dict(ldq=255), dict(ldo=248), dict(scores=16, lds=-1), dict(ldq=1 << 62), dict(scores=16, lds=1 << 61)):
        assert call(**kw) == ESHAPE, kw
    assert call(ldq=260) == EALIGN and call(ldo=257) == EALIGN
    for kw in (dict(q=None), dict(out=None)):
        assert call(**kw) == EINVAL
    for kw in (dict(q=2), dict(out=8), dict(scores=2, lds=1), dict(ws=8)):
        assert call(**kw) == EALIGN
    assert call(s=seqs(seqs=0), q=None, out=None) == OK
    long = seqs(max_pages=1000, ld=1000)
    need, more = (samd.samd_paged_attention_workspace_size(cache(), long, 4, s) for s in (False, True))
    assert 0 < need < more  # with scores: the logits of every token too
    assert more - need >= 3 * 2 * 1000 * 16 * 8 * 4
    assert call(s=long, nb=need - 1) == ESHAPE and call(s=long, ws=None) == EINVAL
    assert call(s=long, scores=16, lds=10, nb=more - 1) == ESHAPE
    assert samd.samd_paged_attention_workspace_size(cache(dim=48), long, 4, False) == 0
    assert samd.samd_paged_attention_workspace_size(cache(), long, 3, False) == 0
    assert samd.samd_paged_attention_workspace_size(cache(), seqs(), 4, False) == 0  # 32 tokens: nothing is split


def test_evict_refusals(lib):
    def call(c=None, s=None, scores=16, lds=32, keep=20, recent=5, dst=32, ldd=2, kept=16, new=16, out=16, null=False):
        return lib.samd_cache_evict(None if null else ctypes.byref(c or cache()), ctypes.byref(s or seqs()), scores, lds, keep,
                                    recent, dst, ldd, kept, new, out, None)

    check_both(call)
    assert call(recent=-1) == EINVAL and call(recent=21) == EINVAL and call(keep=0, recent=0) == ESHAPE
    assert call(keep=(1 << 30) + 1, ldd=1 << 40) == EUNSUP and call(s=seqs(seqs=1 << 27)) == EUNSUP
    for kw in (dict(lds=-1), dict(lds=1 << 61), dict(ldd=1), dict(keep=33)):
        assert call(**kw) == ESHAPE, kw
    for kw in (dict(scores=None), dict(dst=None), dict(kept=None), dict(new=None), dict(dst=16)):  # 16: the sequences' own
        assert call(**kw) == EINVAL, kw
    for kw in (dict(scores=5), dict(dst=18), dict(kept=7), dict(new=2), dict(out=1)):
        assert call(**kw) == EALIGN, kw
    assert call(s=seqs(seqs=0), scores=None, kept=None) == OK


def meta(*shape, dtype=torch.int32):
    return torch.empty(shape, dtype=dtype, device="meta")


def paged(pages=4, heads=2, page=16, dim=64, bits=8, t=torch.bfloat16):
    """A cache without memory: the binding's checks come before the library's."""
    lanes, scales = meta(pages, heads, page, dim * bits // 32), meta(pages, heads, page, dim // 32, dtype=t)
    return lanes, scales


def test_the_binding_checks_its_tensors(monkeypatch):
    monkeypatch.setattr(samd, "_address", lambda t: 16)
    l, s = paged()
    c = samd.PagedCache(l, s, l, s)
    assert (c.bits, c.dim, c.heads, c.page, c.dtype) == (8, 64, 2, 16, torch.bfloat16)
    assert samd.PagedCache(*paged(bits=4) * 2).bits == 4
    for bad in ((l, s, l.long(), s), (l, s.half(), l, s), (l, s.float(), l, s.float()), (l[..., :8], s, l, s), (l, s, l[:3], s),
                (l[0], s[0], l[0], s[0]), (l.transpose(1, 2), s, l, s), (l, s[..., :1], l, s[..., :1].clone())):
        with pytest.raises(ValueError):
            samd.PagedCache(*bad)
    for kw in (dict(bits=6), dict(dim=48), dict(dim=288), dict(page=8), dict(page=24)):
        with pytest.raises(ValueError):
            samd.cache_empty(**(dict(pages=2, page=16, heads=2, dim=64, bits=8, dtype=torch.half) | kw))
    t = torch.bfloat16
    table, lengths = meta(3, 2), meta(3)
    k = meta(5, 2, 64, dtype=t)
    starts = meta(4)
    for kw in (dict(k=k.half()), dict(k=meta(5, 2, 32, dtype=t)), dict(k=meta(5, 3, 64, dtype=t)), dict(v=meta(4, 2, 64, dtype=t)),
               dict(k=k.transpose(0, 1)), dict(k=meta(5, 2, 128, dtype=t)[..., ::2]), dict(table=table.long()),
               dict(lengths=meta(2)), dict(lengths=lengths.long()), dict(table=meta(2, 3).t()), dict(starts=meta(3)),
               dict(starts=starts.long()), dict(lengths=meta(6)[::2])):
        a = dict(k=k, v=k, table=table, lengths=lengths, starts=starts) | kw
        with pytest.raises(ValueError):
            samd.cache_append(c, **a)
    with pytest.raises(ValueError):
        samd.cache_read(c, 5, table, lengths, starts, k=k.half(), v=k)
    with pytest.raises(ValueError, match="size"):
        samd.cache_read(c, 1 << 32, table, lengths, starts)
    q = meta(3, 4, 64, dtype=t)
    for kw in (dict(q=q.half()), dict(q=meta(3, 3, 64, dtype=t)), dict(q=meta(2, 4, 64, dtype=t)), dict(q=meta(3, 0, 64, dtype=t)),
               dict(q=meta(3, 256, dtype=t)), dict(scores=meta(3, 2, 32)), dict(scores=meta(3, 4, 32, dtype=torch.float32)),
               dict(scores=meta(3, 32, 2, dtype=torch.float32).transpose(1, 2)), dict(out=meta(3, 4, 32, dtype=t)),
               dict(out=q.float())):
        a = dict(q=q, cache=c, table=table, lengths=lengths) | kw
        with pytest.raises(ValueError):
            samd.paged_attention(**a)
    w, dst = meta(3, 2, 32, dtype=torch.float32), meta(3, 2)
    for kw in (dict(keep=0), dict(recent=21), dict(recent=-1), dict(dst_table=meta(3, 1)), dict(dst_table=meta(2, 2)),
               dict(dst_table=dst.long()), dict(scores=w.half()), dict(scores=meta(2, 2, 32, dtype=torch.float32)),
               dict(keep=1 << 31, dst_table=meta(3, 1 << 28))):
        a = dict(cache=c, table=table, lengths=lengths, scores=w, dst_table=dst, keep=20, recent=4) | kw
        with pytest.raises(ValueError):
            samd.cache_evict(**a)
    with pytest.raises(ValueError, match="size"):
        samd._cache_seqs(meta((1 << 32) + 5, 1), meta((1 << 32) + 5))


def test_host_tensors_are_refused():
    lanes, scales = torch.zeros((4, 2, 16, 16), dtype=torch.int32), torch.zeros((4, 2, 16, 2), dtype=torch.half)
    with pytest.raises(ValueError, match="device"):
        samd.PagedCache(lanes, scales, lanes, scales)
