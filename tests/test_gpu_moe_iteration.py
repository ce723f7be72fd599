"""The example's serving iterations (examples/moe_iteration.py): hidden states and
expert maps against the same model computed in float64 with nothing cached, and
the search's part: a repeated batch finds its own iterations."""
import importlib.util
import os

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("moe_iteration", os.path.join(ROOT, "examples", "moe_iteration.py"))
    m = importlib.util.module_from_spec(spec)
    import sys
    sys.modules["moe_iteration"] = m
    spec.loader.exec_module(m)
    return m


def _plain(model, prompts):
    """The layers in float64, with the stream rounded to bfloat16 where the model rounds it."""
    c = model.c
    bf = lambda t: t.to(torch.bfloat16).double()
    table = model.table.cpu().double()
    x = bf(torch.stack([table[p[-1]] * c.d ** 0.5 if p else torch.zeros(c.d, dtype=torch.float64) for p in prompts]))
    maps = torch.zeros(len(prompts), c.L, c.E, dtype=torch.float64)
    margin = torch.full((len(prompts),), np.inf, dtype=torch.float64)   # smallest gap between the last expert taken and the next
    for l, layer in enumerate(model.layers):
        h = bf(x * torch.rsqrt(x.square().mean(dim=1, keepdim=True) + 1e-6))
        logits = h @ layer.gate.cpu().double().t()
        p = torch.softmax(logits, dim=1)
        out = x.clone()
        for b, prompt in enumerate(prompts):
            if not prompt:
                continue
            maps[b, l] = p[b]
            top, order = logits[b].sort(descending=True)
            margin[b] = min(margin[b], top[c.K - 1] - top[c.K])
            w = p[b, order[: c.K]] / p[b, order[: c.K]].sum()
            for k in range(c.K):
                g, u, dn = (m.double() for m in layer.host[order[k]])
                out[b] += w[k] * (dn @ (torch.nn.functional.silu(g @ h[b]) * (u @ h[b])))
        x = bf(out)
    return x, maps, margin


@pytest.mark.parametrize("slots", [16, 10, 3])
def test_iterations_match_the_plain_model(slots):
    m = _example()
    model = m.Model(m.Config(slots=slots), seed=3)
    rng = np.random.default_rng(4)
    batches = [[list(map(int, rng.integers(0, model.c.V, n))) for n in (7, 1, 0, 30, 12)] for _ in range(3)]
    for prompts in batches + batches[:1]:
        x, maps, found, loaded = model.iteration(prompts)
        want, want_maps, margin = _plain(model, prompts)
        # A stream off by one bfloat16 unit shifts logits by less than 0.05; where two
        # experts were that close the rest of the pass may take another course.
        sure = margin > 0.05
        assert sure.sum() >= 2
        err = (x.cpu().double() - want).abs().amax(dim=1) / want.abs().amax(dim=1).clamp_min(1e-9)
        assert (err[sure] < 2.0 ** -5).all(), err      # a unit (2^-7) or so in each of 6 layers
        assert ((maps.cpu().double() - want_maps).abs().amax(dim=(1, 2))[sure] < 0.05).all()
        assert (x[2] == 0).all() and (maps[2] == 0).all()
    # the repeated batch is the most similar to itself
    tokens = [t for p in batches[0] for t in p]
    off = np.cumsum([0] + [len(p) for p in batches[0]])
    q = m.fm.embed_pool(model.table, torch.tensor(tokens, dtype=torch.int32, device="cuda"),
                        torch.tensor(off, dtype=torch.int32, device="cuda"), model.c.d ** 0.5)
    idx, score = m.fm.match_semantic(model.store, q)
    assert [int(i) for i in idx[:, 0]][:2] == [0, 1] and (score[[0, 1, 3, 4], 0] > 0.99999).all()


def test_a_full_cache_finds_every_expert():
    m = _example()
    model = m.Model(m.Config(slots=16), seed=5)
    for layer in model.layers:
        layer.bring_in(range(16))
    x, maps, found, loaded = model.iteration([[1, 2, 3], [4, 5], [6]])
    assert loaded == 0 and found > 0 and all(layer.loads == 16 for layer in model.layers)


def test_tuning_the_embeddings_lowers_the_loss():
    m = _example()
    model = m.Model(seed=6)
    tok = torch.tensor([5, 9, 5, 400, -1], dtype=torch.int32, device="cuda")
    wanted = torch.randn(5, model.c.d, generator=torch.Generator().manual_seed(1)).cuda()
    before = model.table.clone()
    losses = [model.tune(tok, wanted, 0.2 / model.c.d) for _ in range(8)]
    # the distance to the mean of what a token's rows want falls by 1 - 0.2 (or
    # - 0.4 for the token that stands twice) a step
    assert all(b < a for a, b in zip(losses, losses[1:])) and losses[-1] < 0.5 * losses[0]
    same = torch.ones(model.c.V, dtype=torch.bool, device="cuda")
    same[[5, 9, 400]] = False
    assert torch.equal(before[same], model.table[same])
