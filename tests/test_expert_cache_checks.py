"""What the binding refuses of an expert cache's memory (CPU only; no call is made)."""
import pytest
import torch

import paper_2502_05370_amd as fm


def _cache():
    return fm.ExpertCache(2, 4, 8, 16, device="cpu")


def test_workspace_on_another_device():
    """The kernels write to the workspace through its address."""
    cache = _cache()
    x, ids, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    ws = fm.MoeWorkspace(cache, 4, 2)
    ws.buf = ws.buf.to("meta")
    with pytest.raises(ValueError, match="workspace is on meta"):
        fm.moe_experts(cache, x, ids, w, workspace=ws)
    ws.buf = torch.zeros(8, dtype=torch.uint8)
    with pytest.raises(ValueError, match="workspace must have shape"):
        fm.moe_experts(cache, x, ids, w, workspace=ws)
