"""The gated feed-forward block, forward and backward, against its definition in
64 bits: bit for bit on integer data (all sums exact in fp32, so only the stated
roundings are left), within derived bounds on normal data, and the gradients
against differences of the definition."""
import pytest
import torch

import ffn_ref as ref
from gpu_util import assert_status_clean
from paper_1809_10572_gb300 import samd

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16
ACTS = ["silu", "gelu", "gelu_tanh", "relu"]
SHAPES = [(1, 8, 8), (1, 1, 1), (3, 40, 33), (127, 64, 128), (128, 72, 130), (129, 200, 264), (300, 1000, 520),
          (64, 129, 257), (257, 300, 96), (200, 2048, 300), (5, 96, 1500), (640, 264, 700)]


def make(shape, t, exact, seed=1):
    M, K, F = shape
    if exact:
        x, wg, wu = ref.ints(seed, (M, K), -2, 2, t), ref.ints(seed + 1, (F, K), -2, 2, t), ref.ints(seed + 2, (F, K), -2, 2, t)
    else:
        x = ref.normal(seed, (M, K), t)
        wg, wu = ref.normal(seed + 1, (F, K), t, K ** -0.5), ref.normal(seed + 2, (F, K), t, K ** -0.5)
    return ref.wide(x), ref.wide(wg), ref.wide(wu)


def form8(values):
    """A checkpoint of the given values, made by the definition."""
    codes, exps, _ = ref.block8(values)
    return samd.Block8(ref.pack8(codes), exps, values.shape[1])


def relative(got, want):
    return float((got.double() - want).norm() / want.norm())


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward_integers_are_exact(samd_lib, shape, t):
    # |g|, |u| <= 4 K < 2^24; act(g) * u rounds once in fp32 and once to t
    M, K, F = shape
    x, wg, wu = make(shape, t, exact=True)
    g, u = x.double() @ wg.double().t(), x.double() @ wu.double().t()
    want = (torch.clamp(g, min=0).float() * u.float()).to(t)
    h = torch.full((M + 1, -(-F // 8) * 8 + 16), 3.0, dtype=t, device="cuda")
    got, g8, u8 = samd.gated_ffn_forward(x, wg, wu, "relu", checkpoints=True, out=h[:M, :F])
    assert torch.equal(got, want)
    for b, v, keep in ((g8, g, True), (u8, u, False)):
        codes, exps, _ = ref.block8(v, keep)
        assert torch.equal(b.exps, exps) and torch.equal(b.lanes, ref.pack8(codes))
    got.fill_(3.0)
    assert (h == 3.0).all()
    assert torch.equal(samd.gated_ffn_forward(x, wg, wu, "relu"), want)  # the same without checkpoints
    assert_status_clean()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("shape", [(70, 200, 140), (130, 1000, 300), (1, 512, 264)])
def test_forward_normal_data(samd_lib, shape, t, act):
    M, K, F = shape
    x, wg, wu = make(shape, t, exact=False)
    X, G, U = x.double(), wg.double(), wu.double()
    g, u = X @ G.t(), X @ U.t()
    # an MMA adds 16 products to the accumulator within four roundings of 2^-23 of the sum of magnitudes
    dg, du = (4 * (K / 16 + 1) * 2.0 ** -23 * (X.abs() @ w.abs().t()) for w in (G, U))
    a = ref.act(g, act)
    got, g8, u8 = samd.gated_ffn_forward(x, wg, wu, act, checkpoints=True)
    err = (got.double() - a * u).abs()
    bound = ref.UNIT[t] * (a * u).abs() + 1.2 * dg * (u.abs() + du) + a.abs() * du + 2.0 ** -16 * (a * u).abs() + ref.TINY
    assert (err <= bound * (1 + ref.UNIT[t])).all()
    # a checkpoint is at most one step (the clamp at 127 of 128) from the value: 2^-6 of the block's largest magnitude
    for b, v, d in ((g8, g, dg), (u8, u, du)):
        n = -(-F // 32)
        pad = torch.zeros((M, n * 32), dtype=torch.float64, device="cuda")
        pad[:, :F] = v.abs() + d
        top = pad.view(M, n, 32).amax(-1).repeat_interleave(32, 1)[:, :F]
        assert ((samd.block8_dequantize(b, torch.float32).double() - v).abs() <= 2.0 ** -6 * top + d).all()


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("shape", SHAPES)
def test_backward_integers_are_exact(samd_lib, shape, t):
    """dg = dh * u where g > 0, du = dh * g there: integers of at most 2 * 3 and 2 * 12, sums below 2^24; x, g, u
    are integers that their 8-bit forms hold exactly."""
    M, K, F = shape
    x, g, u = ref.ints(1, (M, K), -100, 100), ref.ints(2, (M, F), -12, 12), ref.ints(3, (M, F), -3, 3)
    dh = ref.wide(ref.ints(4, (M, F), -2, 2, t))
    wg, wu = ref.wide(ref.ints(5, (F, K), -3, 3, t)), ref.wide(ref.ints(6, (F, K), -3, 3, t))
    D = dh.double()
    dg, du = D * u * (g > 0), D * torch.clamp(g, min=0)
    dx, dwg, dwu, h = samd.gated_ffn_backward(dh, form8(x), form8(g), form8(u), wg, wu, "relu", need_h=True)
    assert torch.equal(dx, (dg @ wg.double() + du @ wu.double()).to(t))
    assert torch.equal(dwg, (dg.t() @ x).to(t)) and torch.equal(dwu, (du.t() @ x).to(t))
    assert torch.equal(h, (torch.clamp(g, min=0) * u).to(t))
    assert_status_clean()


def test_backward_writes_its_outputs_only(samd_lib):
    M, K, F, t = 130, 100, 140, BF16
    x, g, u = ref.ints(1, (M, K), -9, 9), ref.ints(2, (M, F), -9, 9), ref.ints(3, (M, F), -3, 3)
    dh, wg, wu = ref.wide(ref.ints(4, (M, F), -2, 2, t)), ref.wide(ref.ints(5, (F, K), -3, 3, t)), ref.wide(ref.ints(6, (F, K), -3, 3, t))
    ldx, ldw, ldh = 120, wg.stride(0), dh.stride(0)
    d = samd.samd_ffn_desc(M, K, F, ldx, ldw, ldh, samd.SAMD_BF16, samd.SAMD_RELU_ACT)
    nb = samd.samd_gated_ffn_backward_workspace_size(d)
    D = dh.double()
    dg, du = D * u * (g > 0), D * torch.clamp(g, min=0)
    want = {"dx": dg @ wg.double() + du @ wu.double(), "dwg": dg.t() @ x, "dwu": du.t() @ x, "h": torch.clamp(g, min=0) * u}
    sizes = {"dx": (M, K, ldx), "dwg": (F, K, ldw), "dwu": (F, K, ldw), "h": (M, F, ldh)}
    for wanted in (("dx", "dwg", "dwu", "h"), ("dx",), ("dwg",), ("dwu",), ("h",), ("dwu", "dx")):
        bufs = {k: torch.full((sizes[k][0] + 1, sizes[k][2]), 5.0, dtype=t, device="cuda") for k in wanted}
        ws = torch.full((nb + 64,), 0xA5, dtype=torch.uint8, device="cuda")  # its contents do not matter
        samd.samd_gated_ffn_backward(d, dh, form8(x), form8(g), form8(u), wg, wu,
                                     *(bufs.get(k) for k in ("dx", "dwg", "dwu", "h")), ws, nb)
        for k, b in bufs.items():
            rows, cols, _ = sizes[k]
            assert torch.equal(b[:rows, :cols], want[k].to(t)), k
            b[:rows, :cols] = 5.0
            assert (b == 5.0).all(), k
        assert (ws[nb:] == 0xA5).all()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("shape", [(200, 136, 300), (65, 1000, 72)])
def test_backward_normal_data(samd_lib, shape, t, act):
    """Each product sees one rounding of dg and du and one of its result, each at most UNIT / sqrt(3) of the norm for
    mantissas spread over their range: together below 0.82 UNIT; the rest of UNIT is for fp32."""
    M, K, F = shape
    x8, g8, u8 = (ref.block8(ref.normal(s, sh, torch.float32)) for s, sh in ((1, (M, K)), (2, (M, F)), (3, (M, F))))
    forms = [samd.Block8(ref.pack8(c), e, v.shape[1]) for c, e, v in (x8, g8, u8)]
    x, g, u = x8[2], g8[2], u8[2]
    dh = ref.wide(ref.normal(4, (M, F), t))
    wg, wu = ref.wide(ref.normal(5, (F, K), t, K ** -0.5)), ref.wide(ref.normal(6, (F, K), t, K ** -0.5))
    D = dh.double()
    dg, du = D * u * ref.act_grad(g, act), D * ref.act(g, act)
    dx, dwg, dwu, h = samd.gated_ffn_backward(dh, *forms, wg, wu, act, need_h=True)
    xt = x.to(t).double()  # in fp16 and bf16 alike without rounding, from fp32 values of this size
    assert torch.equal(xt, x)
    assert relative(dx, dg @ wg.double() + du @ wu.double()) <= ref.UNIT[t]
    assert relative(dwg, dg.t() @ x) <= ref.UNIT[t] and relative(dwu, du.t() @ x) <= ref.UNIT[t]
    want = ref.act(g, act) * u
    assert ((h.double() - want).abs() <= (ref.UNIT[t] + 2.0 ** -16) * want.abs() + ref.TINY).all()


@pytest.mark.parametrize("act", ACTS)
def test_gradients_against_differences(samd_lib, act):
    """The whole step (checkpoint, forward, backward) against central differences of the definition in 64 bits, for
    the loss sum(h * dh). The checkpoints cost a relative error of at most 2^-6 / sqrt(3) of a block's largest
    magnitude, about 2.2 deviations: 0.02 a factor, three factors; 0.06 bounds the norm. (A ReLU's derivative is not
    continuous: its checkpoint keeps the sign of g.)"""
    M, K, F, t = 96, 72, 80, F16
    x, wg, wu = make((M, K, F), t, exact=False, seed=7)
    dh = ref.wide(ref.normal(11, (M, F), t))
    h, g8, u8 = samd.gated_ffn_forward(x, wg, wu, act, checkpoints=True)
    dx, dwg, dwu = samd.gated_ffn_backward(dh, samd.block8_quantize(x), g8, u8, wg, wu, act)
    point = [v.double().contiguous() for v in (x, wg, wu)]

    def loss(p):
        return float((ref.act(p[0] @ p[1].t(), act) * (p[0] @ p[2].t()) * dh.double()).sum())

    # along random directions: the gradient's part along one is what a difference sees
    for i, grad in enumerate((dx, dwg, dwu)):
        formula = torch.zeros(8, dtype=torch.float64)
        diff = torch.zeros(8, dtype=torch.float64)
        for j in range(8):
            step = 1e-5 * ref.normal(100 * i + j, point[i].shape, torch.float64)
            p = list(point)
            p[i] = point[i] + step
            up = loss(p)
            p[i] = point[i] - step
            diff[j] = (up - loss(p)) / 2
            formula[j] = float((grad.double() * step).sum())
        assert float((formula - diff).norm() / diff.norm()) < 0.06


@pytest.mark.parametrize("act", ACTS)
def test_activation_derivatives_are_those_of_the_definition(samd_lib, act):
    """act and act' through the backward's elementwise part: du = dh * act(g), dg = dh * act'(g) with u = 1, read off
    as one-token weight gradients with x = 1; and act' against differences of act."""
    g = torch.linspace(-12, 12, 1024, dtype=torch.float64, device="cuda").view(32, 32)
    _, _, g = ref.block8(g)
    g = g.reshape(1, 1024)
    one = torch.ones((1, 1024), device="cuda", dtype=F16)
    w = torch.zeros((1024, 8), dtype=F16, device="cuda")
    x = torch.ones((1, 8), dtype=torch.float64, device="cuda")
    _, dwg, dwu = samd.gated_ffn_backward(one, form8(x), form8(g), form8(one), w, w, act)
    want, want_d = ref.act(g, act)[0], ref.act_grad(g, act)[0]
    for got, ex in ((dwu[:, 0], want), (dwg[:, 0], want_d)):
        # rounded twice to fp16; the tails through exp and erfc keep 2^-14 of 1e-3 and the value
        assert ((got.double() - ex).abs() <= 2.1 * ref.UNIT[F16] * ex.abs() + 2 * ref.TINY + 2.0 ** -14 * 1e-3).all()
    e = 1e-6
    diff = (ref.act(g[0] + e, act) - ref.act(g[0] - e, act)) / (2 * e)
    off = g[0].abs() > 1e-3 if act == "relu" else torch.ones(1024, dtype=torch.bool, device="cuda")
    assert ((diff - want_d).abs()[off] < 1e-8).all()


def test_nan_stays_in_its_token(samd_lib):
    M, K, F = 140, 72, 96
    x, wg, wu = make((M, K, F), BF16, exact=False)
    clean = samd.gated_ffn_forward(x, wg, wu)
    x[130, 5] = float("nan")
    h, g8, u8 = samd.gated_ffn_forward(x, wg, wu, checkpoints=True)
    rows = torch.arange(M, device="cuda") != 130
    assert torch.equal(h[rows], clean[rows]) and torch.isnan(h[130]).all()
    assert (g8.exps[130] == 255).all() and (g8.exps[rows] < 255).all() and not g8.lanes[130].any()
    dh = ref.wide(ref.normal(3, (M, F), BF16))
    dx, dwg, _ = samd.gated_ffn_backward(dh, samd.block8_quantize(x), g8, u8, wg, wu)
    assert torch.isnan(dx[130]).all() and torch.isfinite(dx[rows].float()).all()
    assert torch.isnan(dwg).all()  # a sum over the tokens


def test_no_tokens(samd_lib):
    K, F, t = 24, 40, F16
    _, wg, wu = make((1, K, F), t, exact=False)
    x = torch.empty((0, K), dtype=t, device="cuda")
    h, g8, u8 = samd.gated_ffn_forward(x, wg, wu, checkpoints=True)
    assert h.shape == (0, F)
    dx, dwg, dwu = samd.gated_ffn_backward(torch.empty((0, 40), dtype=t, device="cuda"), samd.block8_quantize(x), g8, u8, wg, wu)
    torch.cuda.synchronize()
    assert dx.shape == (0, K) and not dwg.any() and not dwu.any()


@pytest.mark.parametrize("want", [dict(need_dw=False), dict(need_dx=False, need_dw=False, need_h=True),
                                  dict(need_dw=False, need_h=True), dict(need_h=True)])
def test_no_tokens_and_some_outputs(samd_lib, want):
    K, F, t = 24, 40, BF16
    _, wg, wu = make((1, K, F), t, exact=False)
    empty = torch.empty((0, F), dtype=t, device="cuda")
    b8, f8 = samd.block8_empty(0, K), samd.block8_empty(0, F)
    got = samd.gated_ffn_backward(empty, b8, f8, f8, wg, wu, **want)
    torch.cuda.synchronize()
    assert [g is not None for g in got[:3]] == [want.get("need_dx", True)] + [want.get("need_dw", True)] * 2
    assert all(g.shape == (0, K) for g in got[:1] if g is not None) and all(not g.any() for g in got[1:3] if g is not None)
    if want.get("need_h"):
        assert got[3].shape == (0, F)


def test_streams_graphs_and_repeats(samd_lib):
    shape = (300, 264, 520)
    x, wg, wu = make(shape, BF16, exact=False)
    dh = ref.wide(ref.normal(9, (300, 520), BF16))

    def step(stream=None):
        h, g8, u8 = samd.gated_ffn_forward(x, wg, wu, checkpoints=True, stream=stream)
        x8 = samd.block8_quantize(x, stream=stream)
        return (h,) + samd.gated_ffn_backward(dh, x8, g8, u8, wg, wu, stream=stream)

    first = step()
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, step()))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = step(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = step()
    for v in kept:
        v.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, kept))
    assert_status_clean()


@pytest.mark.slow
def test_many_tiles(samd_lib):
    """More tiles than SMs in every product, so that accumulators and stages go round: bit for bit on integers."""
    M, K, F, t = 2300, 1300, 2600, BF16
    x, wg, wu = make((M, K, F), t, exact=True)
    g, u = x.double() @ wg.double().t(), x.double() @ wu.double().t()
    got, g8, u8 = samd.gated_ffn_forward(x, wg, wu, "relu", checkpoints=True)
    assert torch.equal(got, (torch.clamp(g, min=0).float() * u.float()).to(t))
    assert torch.equal(g8.lanes, ref.pack8(ref.block8(g, True)[0])) and torch.equal(u8.exps, ref.block8(u)[1])
    g, u = ref.ints(2, (M, F), -12, 12), ref.ints(3, (M, F), -3, 3)
    dh = ref.wide(ref.ints(4, (M, F), -2, 2, t))
    D, X = dh.double(), x.double()
    dg, du = D * u * (g > 0), D * torch.clamp(g, min=0)
    dx, dwg, dwu = samd.gated_ffn_backward(dh, form8(X), form8(g), form8(u), wg, wu, "relu")
    assert torch.equal(dx, (dg @ wg.double() + du @ wu.double()).to(t))
    assert torch.equal(dwg, (dg.t() @ X).to(t)) and torch.equal(dwu, (du.t() @ X).to(t))
    assert_status_clean()


@pytest.mark.parametrize("shape", [(700, 1096, 900), (200, 4104, 1300), (1500, 2600, 1200), (3000, 600, 3100), (2600, 3000, 2200)])
def test_gradients_of_x_and_of_the_weights_in_one_launch(samd_lib, shape):
    """Sizes whose dx and weight gradients fill the GPU together, with tiles of each width: bit for bit on integers, all
    outputs, and dx with one weight's gradient."""
    M, K, F = shape
    t = BF16
    x, g, u = ref.ints(1, (M, K), -9, 9), ref.ints(2, (M, F), -9, 9), ref.ints(3, (M, F), -3, 3)
    dh, wg, wu = ref.ints(4, (M, F), -2, 2, t), ref.ints(5, (F, K), -3, 3, t), ref.ints(6, (F, K), -3, 3, t)
    dh, wg, wu = (ref.wide(v) for v in (dh, wg, wu))
    D = dh.double()
    dg, du = D * u * (g > 0), D * torch.clamp(g, min=0)
    want = ((dg @ wg.double() + du @ wu.double()).to(t), (dg.t() @ x).to(t), (du.t() @ x).to(t))
    forms = form8(x), form8(g), form8(u)
    got = samd.gated_ffn_backward(dh, *forms, wg, wu, "relu")
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    d = samd.samd_ffn_desc(M, K, F, K, wg.stride(0), dh.stride(0), samd.SAMD_BF16, samd.SAMD_RELU_ACT)
    ws = torch.empty(samd.samd_gated_ffn_backward_workspace_size(d), dtype=torch.uint8, device="cuda")
    for i in (1, 2):
        dx = torch.full((M + 1, K), 5.0, dtype=t, device="cuda")
        dw = torch.full((F + 1, wg.stride(0)), 5.0, dtype=t, device="cuda")
        samd.samd_gated_ffn_backward(d, dh, *forms, wg, wu, dx, dw if i == 1 else None, dw if i == 2 else None, None, ws)
        assert torch.equal(dx[:M], want[0]) and torch.equal(dw[:F, :K], want[i])
        dx[:M] = 5.0
        dw[:F, :K] = 5.0
        assert (dx == 5.0).all() and (dw == 5.0).all()
    assert_status_clean()
