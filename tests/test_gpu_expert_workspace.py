"""The workspace that an expert cache keeps for calls without one of their own,
on the GPU: results while graphs hold it, and on streams that are not ordered."""
import numpy as np
import pytest
import torch

from test_gpu_operators import _fm, _layer, dev, drawn

pytestmark = pytest.mark.gpu


def _calls(rng, E, K, d, f, T):
    """A filled cache and arguments of a call of T tokens."""
    cache, _ = _layer(rng, E, E, d, f, "bf16")
    cache.slot_of.copy_(torch.arange(E, device="cuda", dtype=torch.int32))
    x, _ = drawn(rng, (T, d), "bf16")
    ids = dev(np.stack([rng.permutation(E)[:K] for _ in range(T)]).astype(np.int32))
    return cache, x, ids, torch.rand(T, K, device="cuda")


def test_a_graph_outlives_the_growth_of_the_workspace():
    """A decode call without a workspace of its own, captured; then a prompt, which
    needs more; then memory that other work takes: replays neither write there nor
    are disturbed."""
    fm = _fm()
    rng = np.random.default_rng(1)
    T = 3
    cache, x, ids, w = _calls(rng, 8, 2, 264, 136, 200)
    y = torch.empty_like(x[:T])
    want = fm.moe_experts(cache, x[:T], ids[:T], w[:T], workspace=fm.MoeWorkspace(cache, T, 2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fm.moe_experts(cache, x[:T], ids[:T], w[:T], out=y)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            fm.moe_experts(cache, x[:T], ids[:T], w[:T], out=y)
        first = cache.workspace.nbytes
        for n in (40, 200):
            fm.moe_experts(cache, x[:n], ids[:n], w[:n])
        assert cache.workspace.nbytes > first
        other = [torch.full((first // k,), 85, dtype=torch.uint8, device="cuda") for k in (1, 1, 1, 2, 2) for _ in range(8)]
        for _ in range(3):
            y.zero_()
            graph.replay()
            side.synchronize()
            assert torch.equal(y, want) and all((t == 85).all() for t in other)


def test_unordered_streams():
    """Calls of different tokens on two streams at once, on one cache, and the
    memory of each stream's workspace after the cache is gone."""
    fm = _fm()
    rng = np.random.default_rng(2)
    cache, x, ids, w = _calls(rng, 16, 2, 1032, 520, 24)
    halves = [(x[:12], ids[:12], w[:12]), (x[12:], ids[12:], w[12:])]
    ws = fm.MoeWorkspace(cache, 12, 2)
    want = [fm.moe_experts(cache, *h, workspace=ws) for h in halves]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [[], []]
    for _ in range(40):
        got[0].append(fm.moe_experts(cache, *halves[0]))
        got[1].append(fm.moe_experts(cache, *halves[1], stream=side))
    mine, theirs = (cache.ensure_workspace(12, 2, s) for s in (None, side))
    assert mine is not theirs
    lo, n = theirs.buf.data_ptr(), theirs.nbytes
    del cache, mine, theirs
    taken = [torch.empty(n, dtype=torch.uint8, device="cuda") for _ in range(20)]
    assert not any(t.data_ptr() < lo + n and lo < t.data_ptr() + n for t in taken)
    torch.cuda.synchronize()
    assert all(torch.equal(g, v) for gs, v in zip(got, want) for g in gs)


def test_workspaces_made_during_captures():
    """Captures on a stream that has had no call: the workspace is made there, in
    the graph's memory, and outlives the graph."""
    fm = _fm()
    rng = np.random.default_rng(3)
    cache, x, ids, w = _calls(rng, 8, 2, 264, 136, 100)
    want = [fm.moe_experts(cache, x[:n], ids[:n], w[:n], workspace=fm.MoeWorkspace(cache, n, 2)) for n in (5, 100)]
    outs = [torch.empty_like(v) for v in want]
    graphs = []
    for y, n in zip(outs, (5, 100)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            fm.moe_experts(cache, x[:n], ids[:n], w[:n], out=y)
        graphs.append(g)

    def replay(which):
        for i in which:
            outs[i].zero_()
            graphs[i].replay()
            eager = fm.moe_experts(cache, x[:40], ids[:40], w[:40])
            torch.cuda.synchronize()
            assert torch.equal(outs[i], want[i])
            torch.testing.assert_close(eager.float(), want[1][:40].float(), rtol=2.0 ** -7, atol=2.0 ** -10)

    replay([0, 1, 0, 1])
    graphs[0] = None
    torch.cuda.empty_cache()
    held = [torch.full((cache.workspace.nbytes,), 85, dtype=torch.uint8, device="cuda") for _ in range(10)]
    replay([1, 1])
    assert all((t == 85).all() for t in held)
