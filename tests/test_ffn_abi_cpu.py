"""Refusals of the gated block's entry points, answered on the host before any
launch (addresses here are never read), and the binding's own checks."""
import ctypes

import pytest
import torch

from paper_1809_10572_gb300 import samd

OK, EINVAL, EALIGN, ESHAPE, EUNSUP = range(5)


@pytest.fixture(scope="module")
def lib():
    return samd.load()


def mv(M=2, N=8, K=64, group=32, ldx=64, ldy=8, type=samd.SAMD_BF16):
    return samd.samd_matvec_desc(M, N, K, group, ldx, ldy, type)


def w4(lanes=16, scales=16, zeros=None):
    return samd.samd_weights4(lanes, scales, zeros)


def call_mv(lib, d=None, f=None, x=16, w=None, y=16, null=False):
    return lib.samd_matvec4(None if null else ctypes.byref(d or mv()), f or samd.fmt(4, True), x, w or w4(), y, None)


def test_matvec4_refusals(lib):
    assert call_mv(lib, null=True) == EINVAL
    assert call_mv(lib, mv(type=samd.SAMD_F32)) == EINVAL and call_mv(lib, mv(type=7)) == EINVAL
    for group in (0, 16, 48, -32, 33):
        assert call_mv(lib, mv(group=group)) == EINVAL
    assert call_mv(lib, f=samd.fmt(4, True, 0, 16)) == EINVAL
    for f in (samd.fmt(8, True), samd.fmt(3, False), samd.fmt(4, True, 1)):
        assert call_mv(lib, f=f) == EUNSUP
    for d in (mv(M=-1), mv(N=-1), mv(K=0), mv(ldx=63), mv(ldy=7)):
        assert call_mv(lib, d) == ESHAPE
    big = (1 << 30) + 32
    assert call_mv(lib, mv(K=big, ldx=big)) == EUNSUP and call_mv(lib, mv(N=big, ldy=big)) == EUNSUP
    assert call_mv(lib, mv(M=0), x=None, y=None) == OK and call_mv(lib, mv(N=0), x=None, y=None) == OK
    assert call_mv(lib, x=None) == EINVAL and call_mv(lib, y=None) == EINVAL
    assert call_mv(lib, w=w4(lanes=None)) == EINVAL and call_mv(lib, w=w4(scales=None)) == EINVAL
    assert call_mv(lib, w=w4(zeros=16)) == EINVAL  # signed lanes take no zero points
    u = samd.fmt(4, False)
    assert call_mv(lib, x=8) == EALIGN and call_mv(lib, y=24 + 2) == EALIGN
    assert call_mv(lib, w=w4(lanes=4)) == EALIGN and call_mv(lib, w=w4(scales=2)) == EALIGN
    assert call_mv(lib, f=u, w=w4(zeros=1)) == EALIGN


def test_gated_matvec4_refusals(lib):
    def call(act=0, f=None, wg=None, wu=None, d=None):
        return lib.samd_gated_matvec4(ctypes.byref(d or mv()), act, f or samd.fmt(4, True), 16, wg or w4(), wu or w4(), 16, None)

    assert call(act=-1) == EINVAL and call(act=4) == EINVAL
    assert call(wu=w4(lanes=None)) == EINVAL and call(wu=w4(scales=8)) == EALIGN
    u = samd.fmt(4, False)
    assert call(f=u, wg=w4(zeros=16)) == EINVAL and call(f=u, wu=w4(zeros=16)) == EINVAL  # of one matrix only
    assert call(d=mv(K=0)) == ESHAPE and call(d=mv(M=0)) == OK


def test_block8_refusals(lib):
    def b8(lanes=16, exps=16):
        return samd.samd_block8(lanes, exps)

    def q(type=samd.SAMD_BF16, x=16, ld=64, rows=2, inner=64, b=None):
        return lib.samd_block8_quantize(type, x, ld, rows, inner, b or b8(), None)

    def dq(type=samd.SAMD_BF16, y=16, ld=64, rows=2, inner=64, b=None):
        return lib.samd_block8_dequantize(type, b or b8(), rows, inner, y, ld, None)

    for call in (q, dq):
        assert call(type=3) == EINVAL and call(type=-1) == EINVAL
        assert call(rows=-1) == ESHAPE and call(inner=-1) == ESHAPE and call(ld=63) == ESHAPE
        assert call(rows=1 << 40, ld=1 << 40) == ESHAPE
        assert call(rows=0) == OK and call(inner=0) == OK
        assert call(b=b8(lanes=None)) == EINVAL and call(b=b8(exps=None)) == EINVAL
        assert call(b=b8(lanes=8)) == EALIGN and call(b=b8(exps=1)) == EALIGN
    assert q(x=None) == EINVAL and q(x=8) == EALIGN and dq(y=None) == EINVAL and dq(y=8) == EALIGN


def ffn(M=2, K=64, F=40, ldx=64, ldw=64, ldh=40, type=samd.SAMD_F16, act=0):
    return samd.samd_ffn_desc(M, K, F, ldx, ldw, ldh, type, act)


BAD_SHAPES = [(dict(type=samd.SAMD_F32), EINVAL), (dict(act=4), EINVAL), (dict(act=-1), EINVAL), (dict(M=-1), ESHAPE),
              (dict(K=0), ESHAPE), (dict(F=0), ESHAPE), (dict(ldx=56), ESHAPE), (dict(ldw=56), ESHAPE),
              (dict(ldh=32), ESHAPE), (dict(ldx=68), EALIGN), (dict(ldw=65), EALIGN), (dict(ldh=44), EALIGN),
              (dict(ldx=1 << 38), EUNSUP), (dict(M=1 << 30, F=1 << 20, ldh=1 << 20), EUNSUP)]


def test_forward_refusals(lib):
    b, n = samd.samd_block8(16, 16), samd.samd_block8(None, None)

    def call(d, x=16, wg=16, wu=16, h=16, cg=n, cu=n):
        return lib.samd_gated_ffn_forward(ctypes.byref(d), x, wg, wu, h, cg, cu, None)

    assert lib.samd_gated_ffn_forward(None, 16, 16, 16, 16, n, n, None) == EINVAL
    for kw, status in BAD_SHAPES:
        assert call(ffn(**kw)) == status, kw
    assert call(ffn(M=0), x=None) == OK
    d = ffn()
    for kw in ("x", "wg", "wu", "h"):
        assert call(d, **{kw: None}) == EINVAL and call(d, **{kw: 8}) == EALIGN
    # checkpoints: all four pointers or none
    half = samd.samd_block8(16, None)
    for cg, cu in ((b, n), (n, b), (half, b), (b, half), (samd.samd_block8(None, 16), n)):
        assert call(d, cg=cg, cu=cu) == EINVAL
    assert call(d, cg=b, cu=samd.samd_block8(16, 8)) == EALIGN


def test_backward_refusals(lib):
    b, n = samd.samd_block8(16, 16), samd.samd_block8(None, None)

    def call(d, dh=16, cx=b, cg=b, cu=b, wg=16, wu=16, dx=16, dwg=16, dwu=16, h=None, ws=16, nb=1 << 40):
        return lib.samd_gated_ffn_backward(ctypes.byref(d), dh, cx, cg, cu, wg, wu, dx, dwg, dwu, h, ws, nb, None)

    for kw, status in BAD_SHAPES:
        assert call(ffn(**kw)) == status, kw
        assert samd.samd_gated_ffn_backward_workspace_size(ffn(**kw)) == 0
    d = ffn()
    need = samd.samd_gated_ffn_backward_workspace_size(d)
    assert need >= 2 * (2 * 40 * 2 + 64 * 2)
    assert call(d, dx=None, dwg=None, dwu=None) == EINVAL  # no output
    assert call(d, nb=need - 1) == ESHAPE and call(d, ws=None) == EINVAL and call(d, ws=24) == EALIGN
    for kw in (dict(dh=None), dict(cg=n), dict(cu=n), dict(cx=n), dict(wg=None), dict(wu=None)):
        assert call(d, **kw) == EINVAL
    for kw in ("dh", "wg", "wu", "dx", "dwg", "dwu", "h"):
        assert call(d, **{kw: 8}) == EALIGN
    assert call(d, cg=samd.samd_block8(16, 4)) == EALIGN


def test_backward_of_no_tokens(lib):
    """An empty tensor has no address: with M = 0 a dx or an h alone looks like no output, and there is nothing to do."""
    n = samd.samd_block8(None, None)

    def call(d, dx=None, h=None):
        return lib.samd_gated_ffn_backward(ctypes.byref(d), None, n, n, n, None, None, dx, None, None, h, None, 0, None)

    assert call(ffn(M=0)) == OK
    assert call(ffn(M=0), dx=16) == OK and call(ffn(M=0), h=16) == OK
    assert call(ffn(M=0), dx=8) == EALIGN and call(ffn(M=0, K=0)) == ESHAPE


def test_the_binding_checks_its_tensors():
    """Shapes, types and strides that the C side cannot see (raised before the library is called)."""
    x = torch.zeros((2, 64), dtype=torch.bfloat16)
    lanes, s = torch.zeros((8, 8), dtype=torch.int32), torch.zeros((8, 2), dtype=torch.bfloat16)
    z = torch.zeros((8, 2), dtype=torch.uint8)
    f, u = samd.fmt(4, True), samd.fmt(4, False)
    bad = [dict(x=x.float()), dict(x=x[0]), dict(x=x.t()), dict(lanes=lanes.long()), dict(lanes=lanes[:, :7]),
           dict(scales=s.half()), dict(scales=s[:, :1]), dict(group=48), dict(f=u, zeros=z.int()),
           dict(f=u, zeros=z[:, :1]), dict(out=torch.zeros((2, 7), dtype=torch.bfloat16)),
           dict(out=torch.zeros((2, 8), dtype=torch.half))]
    for kw in bad:
        args = dict(x=x, lanes=lanes, scales=s, group=32, f=f, zeros=None, out=None) | kw
        with pytest.raises((ValueError, IndexError)):
            samd.matvec4(args["x"], args["lanes"], args["scales"], args["group"], args["f"], zeros=args["zeros"], out=args["out"])
    with pytest.raises(ValueError):
        samd.block8_quantize(x.double())
    with pytest.raises(ValueError):
        samd.block8_dequantize(samd.Block8(torch.zeros((2, 16), dtype=torch.int32), torch.zeros((2, 3), dtype=torch.uint8), 64), torch.half)
    w = torch.zeros((40, 64), dtype=torch.bfloat16)
    for args in ((x.float(), w, w), (x, w.half(), w), (x, w[:, :63], w), (x, w, w[:39]), (x, w, torch.zeros((40, 72), dtype=torch.bfloat16)[:, :64])):
        with pytest.raises(ValueError):
            samd.gated_ffn_forward(*args)
    with pytest.raises(KeyError):
        samd.gated_ffn_forward(x, w, w, "tanh")
    b, bh = samd.block8_empty(2, 64, "cpu"), samd.block8_empty(2, 40, "cpu")
    dh = torch.zeros((2, 40), dtype=torch.bfloat16)
    for args in ((dh, bh, bh, bh, w, w), (dh, b, b, bh, w, w), (dh.half(), b, bh, bh, w, w)):
        with pytest.raises(ValueError):
            samd.gated_ffn_backward(*args)
    with pytest.raises(ValueError):  # host tensors
        samd.matvec4(x, lanes, s, 32, f)


def test_the_binding_refuses_sizes_past_an_int():
    """The descriptors hold sizes in 32 bits: 2^32 + 5 rows are not 5 (tensors without memory: only shapes are read)."""
    t, far = torch.bfloat16, (1 << 32) + 5

    def empty(*shape, dtype=t):
        return torch.empty(shape, dtype=dtype, device="meta")

    f = samd.fmt(4, True)
    lanes, s = empty(8, 1, dtype=torch.int32), empty(8, 1)
    with pytest.raises(ValueError, match="size"):
        samd.matvec4(empty(far, 8), lanes, s, 32, f)
    with pytest.raises(ValueError, match="size"):
        samd.matvec4(empty(1, 8), empty(far, 1, dtype=torch.int32), empty(far, 1), 32, f)
    with pytest.raises(ValueError, match="size"):
        samd.matvec4(empty(1, far), empty(1, -(-far // 8), dtype=torch.int32), empty(1, -(-far // 32)), 32, f)
    with pytest.raises(ValueError, match="size"):
        samd.gated_matvec4(empty(far, 8), lanes, s, lanes, s, 32, f)
    for M, K, F in ((far, 8, 8), (1, far - 5, 8), (1, 8, far - 5)):
        with pytest.raises(ValueError, match="size"):
            samd.gated_ffn_forward(empty(M, K), empty(F, K), empty(F, K))
        x8, f8 = samd.block8_empty(M, K, "meta"), samd.block8_empty(M, F, "meta")
        with pytest.raises(ValueError, match="size"):
            samd.gated_ffn_backward(empty(M, F), x8, f8, f8, empty(F, K), empty(F, K))
    # what fits is answered by the library's own limit, or by the tensors' kind
    assert samd._matvec_desc(empty((1 << 31) - 1, 8), s, 32, None).M == (1 << 31) - 1
