"""The serving operators' helpers and kernel forms beyond test_serving_ops.py."""
import types

import torch

from paper_2608_03537_amd import comfuse as cf


# ---------------------------------------------------------------- attention_prefix's workspace
def test_workspace_grows_rarely_and_clears_its_counters_only(monkeypatch):
    """A batch that grows step by step finds room in what an earlier step allocated; of a new workspace
    only the arrival counters are cleared."""
    made = []

    def empty(n, dtype, device):
        made.append(torch.full((n,), 255, dtype=dtype, device=device))
        return made[-1]

    def zeros(n, dtype, device):
        made.append(torch.zeros((n,), dtype=dtype, device=device))
        return made[-1]

    monkeypatch.setattr(cf, "_ws_cache", {})
    host = types.SimpleNamespace(_C=types.SimpleNamespace(_cuda_isCurrentStreamCapturing=lambda: False), empty=empty,
                                 zeros=zeros, uint8=torch.uint8, int32=torch.int32)
    head = cf.CF_PREFIX_WS_HEADER_BYTES
    for need in range(head + 4096, 1 << 23, 1 << 15):
        ws = cf._prefix_workspace(host, need, "cpu", (0, 0, "prefix"))
        assert ws.numel() >= need
    # each one half as large again as the last: from 256 KiB to 8 MiB at most 9
    assert len(made) <= 9
    for t in made:
        assert not t[:head].any() and bool((t[head:] == 255).all())
