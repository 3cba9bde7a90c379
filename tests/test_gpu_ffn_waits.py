"""The bounded waits of the gated block's kernels with a failure on record: long
calls may give up, but end by themselves, write nothing outside their outputs,
leave the context usable, and after a reset give the words they gave before."""
import pytest
import torch

import ffn_ref as ref
from paper_1809_10572_gb300 import samd

pytestmark = pytest.mark.gpu


def calls():
    """Name -> (outputs with guard rows behind them, call)."""
    M, K, F, t = 2100, 1024, 2304, torch.bfloat16
    x, wg, wu = ref.normal(1, (M, K), t), ref.normal(2, (F, K), t, K ** -0.5), ref.normal(3, (F, K), t, K ** -0.5)
    dh = ref.normal(4, (M, F), t)
    x8 = samd.block8_quantize(x)
    _, g8, u8 = samd.gated_ffn_forward(x, wg, wu, checkpoints=True)
    d = samd.samd_ffn_desc(M, K, F, K, K, F, samd.SAMD_BF16, samd.SAMD_SILU)
    nb = samd.samd_gated_ffn_backward_workspace_size(d)
    ws = torch.empty(nb, dtype=torch.uint8, device="cuda")
    h, dx = (torch.full((M + 1, n), 5.0, dtype=t, device="cuda") for n in (F, K))
    dwg, dwu = (torch.full((F + 1, K), 5.0, dtype=t, device="cuda") for _ in range(2))
    few = ref.normal(5, (16, K), t)
    few8 = samd.block8_quantize(few)
    _, fg8, fu8 = samd.gated_ffn_forward(few, wg, wu, checkpoints=True)
    d2 = samd.samd_ffn_desc(16, K, F, K, K, F, samd.SAMD_BF16, samd.SAMD_SILU)
    dx2 = torch.full((17, K), 5.0, dtype=t, device="cuda")  # few rows: the reduction is split over clusters
    q = ref.ints(6, (20000, 4096), -8, 7)
    lanes, scales = ref.pack4(q), torch.ones((20000, 64), dtype=t, device="cuda")
    tok = ref.normal(7, (2, 4096), t)
    y = torch.full((3, 20000), 5.0, dtype=t, device="cuda")
    f = samd.fmt(4, True)
    return {
        "forward": ([h], lambda: samd.gated_ffn_forward(x, wg, wu, out=h[:M])),
        "backward": ([dx, dwg, dwu], lambda: samd.samd_gated_ffn_backward(d, dh, x8, g8, u8, wg, wu, dx, dwg, dwu, None, ws)),
        "split": ([dx2], lambda: samd.samd_gated_ffn_backward(d2, dh, few8, fg8, fu8, wg, wu, dx2, None, None, None, ws)),
        "matvec": ([y], lambda: samd.matvec4(tok, lanes, scales, 64, f, out=y[:2])),
    }


def test_calls_end_with_a_failure_on_record(samd_lib):
    todo = calls()
    first = {}
    for name, (outs, call) in todo.items():
        call()
        first[name] = [o.clone() for o in outs]
    torch.cuda.synchronize()
    assert samd.samd_device_status() == samd.SAMD_OK
    samd.samd_selftest_wait_timeout(1000)
    assert samd.samd_device_status() == samd.SAMD_ETIMEOUT
    for name, (outs, call) in todo.items():
        for _ in range(3):
            call()
        torch.cuda.synchronize()
        assert all((o[-1] == 5.0).all() for o in outs), name
    assert samd.samd_device_status(reset=True) == samd.SAMD_ETIMEOUT
    assert samd.samd_device_status() == samd.SAMD_OK
    for name, (outs, call) in todo.items():
        call()
        assert all(torch.equal(a, b) for a, b in zip(first[name], outs)), name
    assert samd.samd_device_status() == samd.SAMD_OK
