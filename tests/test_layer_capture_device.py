"""A workspace that is made while a stream of its cache's device records a graph, with
another device current (CPU only: the devices are stood in for)."""
import contextlib

import pytest
import torch

import paper_2502_05370_amd as fm
from paper_2502_05370_amd import layer


@pytest.mark.parametrize("capturing", [0, 1])
@pytest.mark.parametrize("of", [0, 1])
def test_a_capture_on_the_caches_device(monkeypatch, of, capturing):
    cache = fm.KvCache(2, 100, 4, 1, 1, 8, page=16, device="cpu")
    current = [0]

    @contextlib.contextmanager
    def device(d):
        before, current[0] = current[0], torch.device(d).index
        yield
        current[0] = before

    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: current[0] == capturing)
    monkeypatch.setattr(layer, "_aligned_bytes", lambda n, device: torch.empty(n, dtype=torch.uint8))
    cache.device = torch.device("cuda", of)
    assert fm.AttnWorkspace(cache, 1).in_capture == (of == capturing)
    assert current == [0]
