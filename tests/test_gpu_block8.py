"""The 8-bit form of activations: codes, exponents and values equal to the
definition, bit for bit (every step of it is exact but the one rounding, whose
ties go to even)."""
import pytest
import torch

import ffn_ref as ref
from paper_1809_10572_gb300 import samd

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]


def check(x, b):
    rows, inner = x.shape
    codes, exps, values = ref.block8(x)
    assert torch.equal(b.exps, exps)
    assert torch.equal(b.lanes, ref.pack8(codes))  # canonical: lanes past the row's end are zero
    return values


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("shape", [(1, 1), (1, 31), (3, 32), (2, 33), (5, 64), (7, 100), (1, 255), (4, 256), (3, 257),
                                   (129, 1001), (64, 4096), (2, 5), (1000, 8), (17, 2052)])
def test_matches_the_definition(samd_lib, shape, t):
    x = ref.normal(1, shape, torch.float64) * 2.0 ** ref.ints(2, shape, -12, 6)
    x = x.to(t)
    b = samd.block8_quantize(x)
    values = check(x, b)
    for to in TYPES:
        assert torch.equal(samd.block8_dequantize(b, to), values.to(torch.float32).to(to))
    # what a 16-bit tensor's form stands for needs no rounding in its type
    if t != torch.float32:
        assert torch.equal(samd.block8_dequantize(b, t).double(), values)


@pytest.mark.parametrize("t", TYPES)
def test_ties_clamps_and_extremes(samd_lib, t):
    top = torch.finfo(t).max
    small = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24, torch.float32: 2.0 ** -149}[t]
    x = torch.zeros((8, 32), dtype=torch.float64, device="cuda")
    x[0, :8] = torch.tensor([64.0, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5, 3.5])  # step 1: ties to even
    x[1, :4] = torch.tensor([127.5, -127.5, 127.0, -127.25])  # codes past 127 are clamped
    x[2, :3] = torch.tensor([top, -top, top / 2])
    x[3, :2] = torch.tensor([small, -small])
    x[4, 5] = small * 3
    x[5, :3] = torch.tensor([2.0 ** -126, 2.0 ** -132, -(2.0 ** -126)])  # exponent 1 and below: the clamp of e at 0
    x[6, :3] = torch.tensor([2.0 ** -119, 2.0 ** -120, 2.0 ** -126])
    x[7, :] = -0.0
    x = x.to(t)
    b = samd.block8_quantize(x)
    values = check(x, b)
    assert torch.equal(samd.block8_dequantize(b, torch.float32).double(), values)
    assert torch.equal(samd.block8_dequantize(b, t).double(), values)


@pytest.mark.parametrize("t", TYPES)
def test_infinities_and_nans_make_their_block_nan(samd_lib, t):
    x = ref.normal(3, (6, 130), t)
    x[0, 5], x[1, 40], x[2, 129], x[3, 64], x[3, 65] = (float(v) for v in ("inf", "-inf", "nan", "nan", "inf"))
    b = samd.block8_quantize(x)
    values = check(x, b)
    got = samd.block8_dequantize(b, t)
    assert torch.equal(torch.isnan(got), torch.isnan(values))
    fine = ~torch.isnan(values)
    assert torch.equal(got[fine].double(), values[fine])


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("ld", [100, 101, 104, 112])
def test_strides_and_guards(samd_lib, ld, t):
    base = torch.full((9, ld), float("nan"), dtype=t, device="cuda")
    base[:, :100] = ref.normal(4, (9, 100), t)
    x = base[:, :100]
    b = samd.Block8(torch.full((11, 25), 77, dtype=torch.int32, device="cuda"),
                    torch.full((11, 4), 77, dtype=torch.uint8, device="cuda"), 100)
    inner = samd.Block8(b.lanes[:9], b.exps[:9], 100)
    samd.block8_quantize(x, out=inner)
    values = check(x, inner)
    assert (b.lanes[9:] == 77).all() and (b.exps[9:] == 77).all()
    y = torch.full((11, ld), 5.0, dtype=t, device="cuda")
    samd.block8_dequantize(inner, t, out=y[:9, :100])
    assert torch.equal(y[:9, :100].double(), values.to(torch.float32).to(t).double())
    y[:9, :100] = 5.0
    assert (y == 5.0).all()


def test_lanes_are_the_librarys_own_format(samd_lib):
    x = ref.normal(5, (6, 50), torch.bfloat16)
    b = samd.block8_quantize(x)
    assert torch.equal(samd.unpack(b.lanes, samd.block8_fmt(), 6, 50), ref.block8(x)[0])


def test_empty_and_side_stream(samd_lib):
    x = torch.empty((0, 64), dtype=torch.float32, device="cuda")
    b = samd.block8_quantize(x)
    assert samd.block8_dequantize(b, torch.float32).shape == (0, 64)
    x = torch.empty((3, 0), dtype=torch.float32, device="cuda")
    assert samd.block8_dequantize(samd.block8_quantize(x), torch.float32).shape == (3, 0)
    x = ref.normal(6, (40, 300), torch.float16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    b = samd.block8_quantize(x, stream=side)
    y = samd.block8_dequantize(b, torch.float16, stream=side)
    side.synchronize()
    assert torch.equal(y.double(), ref.block8(x)[2])
