"""The workspace that an expert cache keeps for calls without one of their own:
what the binding does with it, with host memory in the GPU's place (CPU only; no
call is made)."""
import types
import weakref

import pytest
import torch

import paper_2502_05370_amd as fm
import paper_2502_05370_amd.model as model


class _Buffer(torch.Tensor):
    def record_stream(self, stream):
        pass


@pytest.fixture
def cache(monkeypatch):
    monkeypatch.setattr(model, "_aligned_bytes",
                        lambda nbytes, device: torch.empty(nbytes, dtype=torch.uint8).as_subclass(_Buffer))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: types.SimpleNamespace(cuda_stream=0))
    return fm.ExpertCache(2, 8, 64, 32, device="cpu")


def test_an_enlarged_workspace_keeps_the_replaced_one(cache):
    """A graph captured around a call holds the address of the workspace that the
    call used; replays write there whatever calls came in between."""
    buffers = []
    for T in (1, 40, 100, 300):
        buffers.append(weakref.ref(cache.ensure_workspace(T, 2).buf))
    assert len({id(b()) for b in buffers}) == 4 and all(b() is not None for b in buffers)
    assert cache.ensure_workspace(7, 2) is cache.workspace


def test_few_workspaces_are_made(cache):
    """Calls of one token more at a time: a buffer for each power of two, and one above 128."""
    sizes = [cache.ensure_workspace(T, 2).nbytes for T in range(1, 400)]
    assert sizes == sorted(sizes) and len(set(sizes)) == 5
    for T, n in enumerate(sizes, 1):
        assert n >= fm.moe_workspace_bytes(64, 32, "bf16", T, 2)
    assert cache.ensure_workspace(0, 2) is cache.workspace


def test_streams_share_no_workspace(cache):
    """Calls on two streams are not ordered, and each writes h, its tickets and its
    partial sums to the workspace."""
    one, two = (types.SimpleNamespace(cuda_stream=h) for h in (5, 9))
    a, b, c = cache.ensure_workspace(9, 2, one), cache.ensure_workspace(9, 2, two), cache.ensure_workspace(9, 2)
    spans = sorted((w.buf.data_ptr(), w.buf.data_ptr() + w.nbytes) for w in (a, b, c))
    assert spans[0][1] <= spans[1][0] and spans[1][1] <= spans[2][0]
    assert cache.ensure_workspace(3, 2, one) is a and cache.ensure_workspace(3, 2, two) is b
    assert cache.ensure_workspace(3, 2) is c and cache.workspace is c
    assert cache.ensure_workspace(300, 2, two) is not b and cache.ensure_workspace(3, 2, one) is a


def test_a_workspace_that_cannot_be_made_replaces_nothing(cache, monkeypatch):
    first = cache.ensure_workspace(3, 2)

    def full(nbytes, device):
        raise torch.cuda.OutOfMemoryError("no memory")
    monkeypatch.setattr(model, "_aligned_bytes", full)
    for _ in range(3):
        with pytest.raises(torch.cuda.OutOfMemoryError):
            cache.ensure_workspace(300, 2)
    assert cache.ensure_workspace(3, 2) is first and cache._replaced == []
