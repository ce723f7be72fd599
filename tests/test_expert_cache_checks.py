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


def test_the_memory_that_calls_read_stays_the_caches():
    """Calls read weights and slots at addresses taken when the cache was made; another
    tensor in their place would leave those to whatever is allocated there next."""
    cache = _cache()
    with pytest.raises(AttributeError, match="slot_of cannot be replaced"):
        cache.slot_of = torch.arange(4, dtype=torch.int32)
    with pytest.raises(AttributeError, match="weights cannot be replaced"):
        cache.weights = torch.zeros_like(cache.weights)
    cache.slot_of[1] = 0
    cache.weights[0].fill_(1)
    cache.weights *= 2
    assert cache._desc.slot_of == cache.slot_of.data_ptr() and cache._desc.slots == cache.weights.data_ptr()
    assert cache.slot_of.tolist() == [-1, 0, -1, -1] and (cache.weights[0] == 2).all()


def test_flags_that_no_kernel_could_write():
    cache = _cache()
    x, ids, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    for flags in (torch.zeros(1, dtype=torch.int32, device="meta"), torch.zeros(1), torch.zeros(0, dtype=torch.int32)):
        cache.flags = flags
        with pytest.raises(ValueError, match="flags"):
            fm.moe_experts(cache, x, ids, w)
