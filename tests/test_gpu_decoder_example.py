"""The example that decodes with a bounded packed cache and a layer of experts: all of the cache's and the experts' calls
together, as a decoder makes them."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("packed_decoder_example", os.path.join(ROOT, "examples", "packed_decoder.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("args", [[], ["--type", "f16", "--bits", "8", "--width", "384", "--heads", "12", "--kv-heads", "12",
                                       "--experts", "5", "--topk", "3", "--sequences", "9", "--tokens", "120"]])
def test_decodes(samd_lib, example, args):
    got = example.main(args)
    assert got["status"] == samd_lib.SAMD_OK and got["finite"]
    assert got["cuts"] >= 1 and all(1 <= n <= 128 for n in got["lengths"])
    # A lane's rounding is uniform over a step of amax / 7 (or 127) of 32 values, whose amax is about two deviations and at
    # most sqrt(32) of them: 0.29 * 5.7 / 7 = 0.24 of a value's deviation at most (0.013 in 8 bits). Of the values it goes
    # into the output as it is, of the keys through logits of deviations of about one, that is once more.
    assert got["worst"] < (0.5 if not args else 0.03)
