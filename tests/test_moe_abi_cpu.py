"""Refusals of the expert layer's entry points, answered on the host before any launch (addresses here are never read),
and the binding's own checks."""
import ctypes

import pytest
import torch

from paper_1809_10572_gb300 import samd

OK, EINVAL, EALIGN, ESHAPE, EUNSUP = range(5)


@pytest.fixture(scope="module")
def lib():
    return samd.load()


def desc(M=3, K=64, F=96, E=8, topk=2, group=32, ldx=64, ldy=64, type=samd.SAMD_BF16, act=0):
    return samd.samd_moe_desc(M, K, F, E, topk, group, ldx, ldy, type, act)


def w4(lanes=16, scales=16, zeros=None):
    return samd.samd_weights4(lanes, scales, zeros)


COMMON = [(dict(type=samd.SAMD_F32), EINVAL), (dict(type=5), EINVAL), (dict(M=-1), ESHAPE), (dict(K=0), ESHAPE), (dict(E=0), ESHAPE),
          (dict(topk=0), ESHAPE), (dict(ldx=56), ESHAPE), (dict(ldx=68), EALIGN), (dict(K=48), EUNSUP),
          (dict(K=1 << 21, ldx=1 << 21, ldy=1 << 21), EUNSUP), (dict(E=1025), EUNSUP), (dict(E=64, topk=33), EUNSUP),
          (dict(ldx=1 << 61), ESHAPE)]


def test_route_refusals(lib):
    def call(d=None, normalize=1, x=16, router=16, ids=16, weights=16, null=False):
        return lib.samd_moe_route(None if null else ctypes.byref(d or desc()), normalize, x, router, ids, weights, None)

    assert call(null=True) == EINVAL and call(normalize=2) == EINVAL and call(normalize=-1) == EINVAL
    for kw, status in COMMON:
        assert call(desc(**kw)) == status, kw
    assert call(desc(topk=9)) == ESHAPE  # of eight experts
    assert call(desc(M=0), x=None, ids=None) == OK
    for kw in ("x", "router", "ids", "weights"):
        assert call(**{kw: None}) == EINVAL
        assert call(**{kw: 2}) == EALIGN


def test_moe4_refusals(lib):
    def call(d=None, f=None, x=16, ids=16, weights=16, g=None, u=None, dn=None, y=16, ws=16, nb=1 << 40, null=False):
        return lib.samd_moe4(None if null else ctypes.byref(d or desc()), f or samd.fmt(4, True), x, ids, weights, g or w4(),
                             u or w4(), dn or w4(), y, ws, nb, None)

    assert call(null=True) == EINVAL
    for kw, status in COMMON + [(dict(group=16), EINVAL), (dict(group=48), EINVAL), (dict(act=4), EINVAL), (dict(F=0), ESHAPE),
                                (dict(ldy=56), ESHAPE), (dict(ldy=65), EALIGN), (dict(F=40), EUNSUP), (dict(F=1 << 21), EUNSUP)]:
        assert call(desc(**kw)) == status, kw
    assert call(f=samd.fmt(4, True, 0, 16)) == EINVAL
    for f in (samd.fmt(8, True), samd.fmt(4, True, 1)):
        assert call(f=f) == EUNSUP
    assert call(desc(M=0), x=None, y=None, ws=None) == OK
    assert call(desc(M=0, topk=9)) == OK  # some of the ids may be other devices' experts
    for kw in ("x", "ids", "weights", "y", "ws"):
        assert call(**{kw: None}) == EINVAL
        assert call(**{kw: 6}) == EALIGN
    for kw in ("g", "u", "dn"):
        assert call(**{kw: w4(lanes=None)}) == EINVAL and call(**{kw: w4(scales=None)}) == EINVAL
        assert call(**{kw: w4(lanes=8)}) == EALIGN and call(**{kw: w4(zeros=16)}) == EINVAL
        assert call(f=samd.fmt(4, False), **{kw: w4(zeros=16)}) == EINVAL  # of one matrix only
    z = w4(zeros=16)
    assert call(f=samd.fmt(4, False), g=z, u=z, dn=w4(zeros=8)) == EALIGN
    need = samd.samd_moe4_workspace_size(desc())
    assert need == 3 * 2 * 96 * 2 and call(nb=need - 1) == ESHAPE
    assert samd.samd_moe4_workspace_size(desc(M=1000)) == 64 * 2 * 96 * 2  # 64 tokens at a time
    assert samd.samd_moe4_workspace_size(desc(M=1000, E=64, topk=32)) == 32 * 32 * 96 * 2
    assert samd.samd_moe4_workspace_size(desc(K=48)) == 0


def test_the_binding_checks_its_tensors():
    t = torch.bfloat16
    x, router = torch.zeros((3, 64), dtype=t), torch.zeros((8, 64), dtype=t)
    for kw in (dict(router=router.half()), dict(router=router[:, :32]), dict(router=router.t()), dict(topk=0), dict(topk=9),
               dict(x=x.float(), router=router.float()), dict(x=x[0]), dict(ids=torch.zeros((3, 2), dtype=torch.int64)),
               dict(weights=torch.zeros((3, 3)))):
        a = dict(x=x, router=router, topk=2) | kw
        with pytest.raises(ValueError):
            samd.moe_route(**a)
    E, F, K, G = 8, 96, 64, 32
    def m(rows, k):
        return torch.zeros((rows, k // 8), dtype=torch.int32), torch.zeros((rows, k // G), dtype=t)
    gate, up, down = m(E * F, K), m(E * F, K), m(E * K, F)
    ids, w = torch.zeros((3, 2), dtype=torch.int32), torch.zeros((3, 2))
    assert samd._experts4(gate, up, down, K, G, samd.fmt(4, True), t) == (E, F)
    z = torch.zeros((E * F, K // G), dtype=torch.uint8)
    for kw in (dict(x=x.half()), dict(ids=ids.long()), dict(ids=ids[:2]), dict(ids=ids[0]), dict(weights=w.half()), dict(weights=w[:, :1]),
               dict(group=16), dict(gate=(gate[0], gate[1].half())), dict(up=(up[0][:, :4], up[1])), dict(down=m(E * K + 1, F)),
               dict(down=m(32, F)), dict(gate=m(E * F + 1, K)), dict(gate=(*gate, z.int())), dict(gate=(*gate, z[:5])),
               dict(out=torch.zeros((3, 32), dtype=t)), dict(out=torch.zeros((3, 64)))):
        a = dict(x=x, ids=ids, weights=w, gate=gate, up=up, down=down, group=G, f=samd.fmt(4, True)) | kw
        with pytest.raises((ValueError, IndexError)):
            samd.moe4(**a)
    with pytest.raises(ValueError, match="device"):
        samd.moe4(x, ids, w, gate, up, down, G, samd.fmt(4, True))
    with pytest.raises(KeyError):
        samd.moe4(x, ids, w, gate, up, down, G, samd.fmt(4, True), "tanh")
    far = (1 << 32) + 8
    with pytest.raises(ValueError, match="size"):
        samd.moe_route(torch.empty((far, 64), dtype=t, device="meta"), torch.empty((8, 64), dtype=t, device="meta"), 2)
