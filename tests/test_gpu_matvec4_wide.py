"""The matrix-vector products over more rows than the GPU's CTAs take in one turn: every CTA's ring of stages runs on
from tile to tile with all of its warps at work, in each instance by tokens, alignment, scales and zero points. Integer
data, bit for bit (tests/test_gpu_matvec4.py has the reasoning)."""
import pytest
import torch

import ffn_ref as ref
from gpu_util import assert_status_clean
from paper_1809_10572_gb300 import samd

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def weights(seed, N, K, G, zeros, t):
    """(lanes, scales, zeros, 64-bit weights) as samd.matvec4 takes them, with scales of 1/2, 1 or 2."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def ints(shape, lo, hi, dtype):
        return torch.randint(lo, hi + 1, shape, generator=g, device="cuda", dtype=dtype)

    groups = -(-K // G)
    q = ints((N, K), 0, 15, torch.int8) if zeros else ints((N, K), -8, 7, torch.int8)
    z = ints((N, groups), 0, 15, torch.uint8) if zeros else None
    s = (2.0 ** ints((N, groups), -1, 1, torch.int32).double()).to(t)
    return ref.pack4(q), s, z, ref.weights4(q, s, z, G)


# (K, G): blocks of 256 and of 128 inputs; scales on their own size and not (a number of groups that is no multiple of a
# block's); groups past a block; rows that are not whole 16-byte units (K = 4104)
WIDTHS = [(2048, 32), (2048, 64), (2048, 256), (2080, 32), (4128, 64), (4224, 128), (2304, 512), (4104, 32), (4104, 128)]


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("K,G", WIDTHS)
def test_every_instance_over_many_tiles(samd_lib, K, G, zeros, t):
    # |x| <= 2, |q - z| <= 15, scales of at most 2: multiples of 1/2 below 2^18
    N = 20011
    lanes, s, z, w = weights(K + G, N, K, G, zeros, t)
    f = samd.fmt(4, not zeros)
    x = ref.ints(5, (32, K), -2, 2)
    want = (x @ w.t()).to(t)
    for M in (1, 2, 3, 5, 8, 13, 32):
        assert torch.equal(samd.matvec4(x[:M].to(t), lanes, s, G, f, zeros=z), want[:M]), M
    for M in (5, 13, 17):  # rows of x that are not 16-byte aligned
        xb = torch.full((M, K + 1), float("nan"), dtype=t, device="cuda")
        xb[:, :K] = x[:M]
        assert torch.equal(samd.matvec4(xb[:, :K], lanes, s, G, f, zeros=z), want[:M]), M
    assert_status_clean()


@pytest.mark.parametrize("t", [BF16, F16])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("K,G", [(2048, 32), (2080, 32), (2048, 256), (4128, 64), (4104, 128), (1000, 64)])
def test_the_pair_over_many_tiles(samd_lib, K, G, zeros, t):
    # with a ReLU every output is a product of two exact sums, rounded to fp32 and then to t
    N = 10007
    lg, sg, zg, wg = weights(2 * K + G, N, K, G, zeros, t)
    lu, su, zu, wu = weights(3 * K + G, N, K, G, zeros, t)
    f = samd.fmt(4, not zeros)
    x = ref.ints(6, (20, K), -1, 1)
    want = (torch.clamp(x @ wg.t(), min=0).float() * (x @ wu.t()).float()).to(t)
    for M in (1, 3, 8, 12, 20):
        got = samd.gated_matvec4(x[:M].to(t), lg, sg, lu, su, G, f, "relu", zeros_g=zg, zeros_u=zu)
        assert torch.equal(got, want[:M]), M
    assert_status_clean()
