"""The example's serving iterations with batch slots that hold no request."""
import pytest
import torch

from test_gpu_moe_iteration import _example

pytestmark = pytest.mark.gpu


def test_idle_slots_store_nothing():
    m = _example()
    model = m.Model(seed=7)
    x, maps, _, _ = model.iteration([[], [1, 2, 3], [], [4, 5]])
    assert model.store.size == 2
    query = m.fm.embed_pool(model.table, torch.tensor([1, 2, 3, 4, 5], dtype=torch.int32, device="cuda"),
                            torch.tensor([0, 3, 5], dtype=torch.int32, device="cuda"), model.c.d ** 0.5)
    idx, score = m.fm.match_semantic(model.store, query)
    assert idx[:, 0].tolist() == [0, 1] and (score > 0.999).all()
    # a request unlike both finds one of them, not an empty iteration
    idx, score = m.fm.match_semantic(model.store, -query.sum(dim=0, keepdim=True).to(torch.bfloat16))
    assert score[0, 0] < 0
    model.iteration([[], []])
    assert model.store.size == 2 and (x[[0, 2]] == 0).all() and (maps[[0, 2]] == 0).all()
    for n in range(90):      # past the store's end
        model.iteration([[], [n, 2 * n + 1], [7 * n + 1], [n + 300, 5, n]])
    assert model.store.size == model.c.store
