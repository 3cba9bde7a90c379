"""The example that trains the gated block with 8-bit checkpoints and serves it from 4-bit weights."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("gated_ffn_example", os.path.join(ROOT, "examples", "gated_ffn.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("args", [[], ["--type", "f16", "--width", "200", "--hidden", "424", "--tokens", "300", "--act", "gelu"]])
def test_trains_and_serves(samd_lib, example, args):
    got = example.main(args)
    assert got["status"] == samd_lib.SAMD_OK
    assert all(l == l for l in got["losses"]) and got["losses"][-1] < 0.8 * got["losses"][0]
    # a lane's rounding is uniform over a step of amax / 7: 0.12 of the weights' deviation (amax of 32 normals is about
    # two deviations), in three matrices
    assert got["serving_error"] < 0.3


def test_packed_weights_are_the_librarys_lanes(samd_lib, example):
    """Served outputs equal the product with the weights that the lanes and scales stand for."""
    torch.manual_seed(0)
    w = torch.randn((70, 90), device="cuda").half()
    lanes, scales = example.pack_weights(w, 32)
    q = samd_lib.unpack(lanes, samd_lib.fmt(4, True), 70, 90).double()
    stands = q * scales.double().repeat_interleave(32, 1)[:, :90]
    x = torch.randn((2, 90), device="cuda").half()
    want = x.double() @ stands.t()
    got = samd_lib.matvec4(x, lanes, scales, 32, samd_lib.fmt(4, True))
    assert float((got.double() - want).norm() / want.norm()) < 2.0 ** -11


@pytest.mark.parametrize("t", [torch.float16, torch.bfloat16])
def test_a_group_of_zeros(samd_lib, example, t):
    """Its scale is not zero, its lanes are, and it adds nothing."""
    torch.manual_seed(1)
    w = torch.randn((40, 96), device="cuda").to(t)
    w[3, 32:64] = 0
    w[9] = 0
    lanes, scales = example.pack_weights(w, 32)
    assert (scales > 0).all() and torch.isfinite(scales).all()
    q = samd_lib.unpack(lanes, samd_lib.fmt(4, True), 40, 96).view(40, 96)
    assert not q[3, 32:64].any() and not q[9].any() and q[3, :32].any()
    x = torch.randn((1, 96), device="cuda").to(t)
    got = samd_lib.matvec4(x, lanes, scales, 32, samd_lib.fmt(4, True))
    assert torch.isfinite(got).all() and got[0, 9] == 0
