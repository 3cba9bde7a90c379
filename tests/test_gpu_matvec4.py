"""samd_matvec4 and samd_gated_matvec4 against 64-bit products of the lanes'
definitions: bit for bit on integer data (every sum is an integer below 2^24
times a power of two, so fp32 is exact and only the last rounding is left), and
within derived bounds on normal data."""
import pytest
import torch

import ffn_ref as ref
from gpu_util import assert_status_clean
from paper_1809_10572_gb300 import samd

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def make(seed, N, K, G, zeros, t, exact, word_bits=32):
    """(lanes, scales, zeros, 64-bit weights)."""
    groups = -(-K // G)
    q = ref.ints(seed, (N, K), 0, 15) if zeros is not False else ref.ints(seed, (N, K), -8, 7)
    z = ref.ints(seed + 1, (N, groups), 0, 15, torch.uint8) if zeros is True else None
    if exact:
        s = 2.0 ** ref.ints(seed + 2, (N, groups), -1, 1)
    else:
        s = ref.normal(seed + 2, (N, groups), torch.float64, 0.02).abs() + 0.001
    s = s.to(t)
    return ref.pack4(q, word_bits), s, z, ref.weights4(q, s, z, G)


def sum_bound(K):
    """Error of the kernel's fp32 sum over K terms, as a multiple of the sum of magnitudes: two MMAs a group of 32
    (each within four roundings of 2^-23 of its largest partial sum), then a chain of at most K / 256 + 8 scaled
    additions."""
    return 8 * 2.0 ** -23 + (K / 256 + 8) * 2.0 ** -24


SHAPES = [(1, 1, 1, 32), (1, 16, 32, 32), (1, 17, 33, 32), (2, 40, 256, 64), (3, 100, 1432, 32), (5, 129, 1000, 128),
          (8, 64, 2048, 64), (9, 33, 520, 32), (13, 70, 130, 64), (16, 48, 4096, 128), (17, 31, 96, 256), (32, 80, 264, 32),
          (33, 20, 300, 64), (70, 50, 65, 32), (1, 5000, 64, 32), (4, 24, 9000, 1024), (1, 8, 16384, 16384),
          (2, 19, 7, 4096)]


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("zeros", [False, None, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_integers_are_exact(samd_lib, shape, zeros, t):
    # |x| <= 2, |q - z| <= 15, scales of 1/2 .. 2: sums are multiples of 1/2 below 2 * 15 * 2 * 16384 < 2^20
    M, N, K, G = shape
    lanes, s, z, w = make(11, N, K, G, zeros, t, exact=True)
    x = ref.ints(12, (M, K), -2, 2)
    want = x @ w.t()
    f = samd.fmt(4, zeros is False)
    got = samd.matvec4(x.to(t), lanes, s, G, f, zeros=z)
    assert got.shape == (M, N) and torch.equal(got, want.to(t))


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("shape", [(1, 300, 640, 64), (3, 130, 1001, 32), (16, 64, 513, 128), (40, 33, 72, 32)])
def test_strides_word_width_and_guards(samd_lib, shape, t):
    """64-bit words hold the same lanes; rows of x and y any stride apart (odd ones too); nothing outside the
    outputs is written, nothing outside the inputs is used."""
    M, N, K, G = shape
    lanes, s, z, w = make(21, N, K, G, True, t, exact=True, word_bits=64)
    x = ref.ints(22, (M, K), -2, 2)
    want = (x @ w.t()).to(t)
    for ldx, ldy in ((K + 8 - K % 8, N + 3), (K + 1, N), (K + 7, N + 8)):
        xb = torch.full((M, ldx), float("nan"), dtype=t, device="cuda")
        xb[:, :K] = x
        yb = torch.full((M + 2, ldy), 7.0, dtype=t, device="cuda")
        samd.matvec4(xb[:, :K], lanes, s, G, samd.fmt(4, False, 0, 64), zeros=z, out=yb[:M, :N])
        assert torch.equal(yb[:M, :N], want)
        yb[:M, :N] = 7.0
        assert (yb == 7.0).all()


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("shape", [(1, 256, 4096, 128), (2, 64, 1000, 32), (7, 200, 2048, 64), (24, 96, 3000, 32)])
def test_normal_data(samd_lib, shape, t):
    M, N, K, G = shape
    lanes, s, z, w = make(31, N, K, G, True, t, exact=False)
    x = ref.normal(32, (M, K), t)
    want = x.double() @ w.t()
    mag = x.double().abs() @ w.abs().t()
    got = samd.matvec4(x, lanes, s, G, samd.fmt(4, False), zeros=z)
    err = (got.double() - want).abs()
    assert (err <= ref.UNIT[t] * want.abs() + sum_bound(K) * mag * (1 + ref.UNIT[t]) + ref.TINY).all()


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("shape", [(1, 48, 256, 64), (2, 33, 1000, 32), (6, 100, 72, 128), (12, 40, 2048, 64), (35, 30, 520, 32)])
def test_gated(samd_lib, shape, t, act):
    M, N, K, G = shape
    lg, sg, zg, wg = make(41, N, K, G, True, t, exact=False)
    lu, su, zu, wu = make(51, N, K, G, True, t, exact=False)
    x = ref.normal(42, (M, K), t)
    g, u = x.double() @ wg.t(), x.double() @ wu.t()
    dg, du = (sum_bound(K) * (x.double().abs() @ w.abs().t()) for w in (wg, wu))
    a = ref.act(g, act)
    want = a * u
    got = samd.gated_matvec4(x, lg, sg, lu, su, G, samd.fmt(4, False), act, zeros_g=zg, zeros_u=zu)
    err = (got.double() - want).abs()
    # |act'| < 1.2; the activation itself to 2^-16 (exp of a product with log2 e, relative 2^-23 of |g|, |g| < 100)
    bound = ref.UNIT[t] * want.abs() + 1.2 * dg * (u.abs() + du) + a.abs() * du + 2.0 ** -16 * want.abs() + ref.TINY
    assert (err <= bound * (1 + ref.UNIT[t])).all()


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("shape", [(1, 40, 64, 32), (3, 77, 500, 64), (20, 35, 129, 32)])
def test_gated_integers_are_exact(samd_lib, shape, t):
    # |g|, |u| <= 500 * 2 * 8 = 2^13 in halves: products of up to 2^28 in quarters are rounded once in fp32
    # and once to t, so compare with the same two roundings
    M, N, K, G = shape
    lg, sg, _, wg = make(61, N, K, G, False, t, exact=True)
    lu, su, _, wu = make(71, N, K, G, False, t, exact=True)
    x = ref.ints(62, (M, K), -1, 1)
    want = (torch.clamp(x @ wg.t(), min=0).float() * (x @ wu.t()).float()).to(t)
    got = samd.gated_matvec4(x.to(t), lg, sg, lu, su, G, samd.fmt(4, True), "relu")
    assert torch.equal(got, want)


def test_infinities_and_nans_stay_in_their_token(samd_lib):
    lanes, s, _, w = make(81, 50, 200, 64, False, BF16, exact=True)
    x = ref.ints(82, (4, 200), -2, 2)
    w[:, 70] = torch.where(w[:, 70] == 0, w[:, 70] + 0, w[:, 70])
    x[1, 70], x[2, 5] = float("inf"), float("nan")
    got = samd.matvec4(x.to(BF16), lanes, s, 64, samd.fmt(4, True))
    want = x @ w.t()
    for m in (0, 3):
        assert torch.equal(got[m], want[m].to(BF16))
    assert torch.isnan(got[2]).all()
    # infinity times a weight: its sign, or a NaN where the weight is zero
    assert torch.equal(torch.isnan(got[1]), torch.isnan(want[1]))
    fine = ~torch.isnan(want[1])
    assert torch.equal(got[1][fine], want[1][fine].to(BF16))


def test_an_infinite_scale_reaches_its_row_only(samd_lib):
    lanes, s, _, w = make(91, 40, 96, 32, False, F16, exact=True)
    x = ref.ints(92, (2, 96), 1, 2)
    s2 = s.clone()
    s2[7, 2] = float("nan")
    a, b = (samd.matvec4(x.to(F16), lanes, v, 32, samd.fmt(4, True)) for v in (s, s2))
    rows = torch.arange(40, device="cuda") != 7
    assert torch.equal(a[:, rows], b[:, rows]) and torch.isnan(b[:, 7]).all()


def test_empty_calls(samd_lib):
    lanes, s, _, _ = make(95, 8, 64, 32, False, BF16, exact=True)
    x = torch.empty((0, 64), dtype=BF16, device="cuda")
    assert samd.matvec4(x, lanes, s, 32, samd.fmt(4, True)).shape == (0, 8)
    x = torch.empty((2, 64), dtype=BF16, device="cuda")
    assert samd.matvec4(x, lanes[:0], s[:0], 32, samd.fmt(4, True)).shape == (2, 0)


def test_side_stream_graph_and_repeats(samd_lib):
    lanes, s, _, w = make(97, 500, 1024, 64, False, BF16, exact=False)
    x = ref.normal(98, (2, 1024), BF16)
    f = samd.fmt(4, True)
    first = samd.matvec4(x, lanes, s, 64, f)
    assert all(torch.equal(first, samd.matvec4(x, lanes, s, 64, f)) for _ in range(5))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = samd.matvec4(x, lanes, s, 64, f, stream=side)
    side.synchronize()
    assert torch.equal(first, y)
    out = torch.zeros_like(first)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        samd.matvec4(x, lanes, s, 64, f, out=out)
    x.copy_(ref.normal(99, (2, 1024), BF16))
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, samd.matvec4(x, lanes, s, 64, f))


@pytest.mark.slow
def test_weights_past_two_to_the_31_bytes(samd_lib):
    """Rows of lanes whose offsets pass 31 bits: the first and last rows of 2.3 GB of weights."""
    N, K, G = 140000, 32768, 128
    lanes = torch.zeros((N, K // 8), dtype=torch.int32, device="cuda")
    s = torch.ones((N, K // G), dtype=BF16, device="cuda")
    rows = torch.cat((torch.arange(40), torch.arange(N - 40, N))).cuda()
    q = ref.ints(5, (80, K), -8, 7)
    lanes[rows] = ref.pack4(q)
    x = ref.ints(6, (1, K), -1, 1)
    got = samd.matvec4(x.to(BF16), lanes, s, G, samd.fmt(4, True))
    assert torch.equal(got[:, rows], (x @ q.t()).to(BF16))
    assert not got[:, 40:N - 40].any()
    assert_status_clean()
