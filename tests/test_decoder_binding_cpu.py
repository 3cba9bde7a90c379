"""What the binding of the packed cache and of the experts checks and keeps, without a GPU (addresses here are never read)."""
import pytest
import torch

from paper_1809_10572_gb300 import samd


def test_a_layers_router_has_as_many_rows_as_there_are_experts():
    """With a workspace of the caller's and without one."""
    t, E, F, K, G = torch.bfloat16, 8, 96, 64, 32
    x = torch.zeros((3, K), dtype=t)

    def m(rows, k):
        return torch.zeros((rows, k // 8), dtype=torch.int32), torch.zeros((rows, k // G), dtype=t)

    mats = m(E * F, K), m(E * F, K), m(E * K, F)
    for workspace in (None, torch.zeros(1 << 16, dtype=torch.uint8)):
        for rows in (E - 1, E + 1, 2 * E):
            with pytest.raises(ValueError, match="router"):
                samd.moe_layer4(x, torch.zeros((rows, K), dtype=t), 2, *mats, G, samd.fmt(4, True), workspace=workspace)
        with pytest.raises(ValueError, match="device"):  # as many: nothing is wrong but that it all lies on the host
            samd.moe_layer4(x, torch.zeros((E, K), dtype=t), 2, *mats, G, samd.fmt(4, True), workspace=workspace)


def test_the_attentions_workspace_is_the_current_devices(monkeypatch):
    """Its size goes by the current device's SMs, as the library's call does, wherever q lies."""
    given = []
    current = [0]
    monkeypatch.setattr(samd, "_address", lambda t: 16)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    monkeypatch.setattr(samd, "samd_paged_attention_workspace_size", lambda *a: 128 * (current[0] + 1))
    monkeypatch.setattr(samd, "samd_paged_attention", lambda *a: given.append(a[-2]))
    samd._attention_workspace.cache_clear()

    def meta(*shape, dtype=torch.int32):
        return torch.empty(shape, dtype=dtype, device="meta")

    t = torch.bfloat16
    lanes, scales = meta(4, 2, 16, 16), meta(4, 2, 16, 2, dtype=t)
    cache = samd.PagedCache(lanes, scales, lanes, scales)
    for device in (0, 1, 0, 1):
        current[0] = device
        samd.paged_attention(meta(3, 4, 64, dtype=t), cache, meta(3, 40), meta(3))
    samd._attention_workspace.cache_clear()
    assert given == [128, 256, 128, 256]
