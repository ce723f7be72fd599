"""The experts' products at sizes that take every loop of the kernels round more
than once: workgroups with several units of rows, rows of several load rounds,
experts met in several groups of places, batches of several passes; against the
float64 definition of oracle.operators."""
import numpy as np
import pytest
import torch

from oracle import operators as ref
from test_gpu_experts_long import _chosen
from test_gpu_operators import _fm, _layer, close, dev, drawn

pytestmark = pytest.mark.gpu


# 512 workgroups share the gate and up rows.  Up to 16 tokens a unit is 16 rows of an
# expert, a load round 4 KB of a row (bf16: two groups of 128 bytes for each of 8
# wavefronts); above, a unit is 128 rows.  Units of the cases: 8 x 101, 8 x 101,
# 64 x 11 for the experts in use.
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,f,E,K", [(9, 2112, 1608, 8, 4), (16, 2120, 1608, 8, 2), (40, 264, 1408, 64, 8),
                                       (100, 264, 1400, 64, 8)])
def test_more_units_than_workgroups(T, d, f, E, K, dtype):
    print(f"experts T={T} d={d} f={f} E={E} K={K} {dtype}", flush=True)
    fm = _fm()
    rng = np.random.default_rng(T + d + f)
    cache, slots = _layer(rng, E, E, d, f, dtype)
    slot_of = rng.permutation(E).astype(np.int32)
    cache.slot_of.copy_(dev(slot_of))
    x, xn = drawn(rng, (T, d), dtype)
    res, rn = drawn(rng, (T, d), dtype)
    ids = _chosen(rng, T, E, K, "even")
    assert len(np.unique(ids)) * ((f + (15 if T <= 16 else 127)) // (16 if T <= 16 else 128)) > 512
    wt = rng.random((T, K)).astype(np.float32)
    ws = fm.MoeWorkspace(cache, T, K)
    ws.buf.random_(0, 255)
    got = fm.moe_experts(cache, x, dev(ids), dev(wt), residual=res, workspace=ws)
    some = np.arange(T) if T <= 16 else np.arange(0, T, 3)
    want, bound = ref.moe_experts(xn[some], ids[some], wt[some], slots, slot_of, d, f, rn[some], dtype)
    close(got[dev(some)], want, bound, dtype)
    assert cache.check() == 0
    assert torch.equal(got, fm.moe_experts(cache, x, dev(ids), dev(wt), residual=res, workspace=ws))


# An expert's tokens beyond 64 are a second group of places, up to 128 tokens.
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [65, 97, 128])
def test_experts_of_more_than_64_tokens(T, dtype):
    fm = _fm()
    rng = np.random.default_rng(T)
    d, f, E, K = 264, 1032, 4, 4
    cache, slots = _layer(rng, E, E, d, f, dtype)
    cache.slot_of.copy_(torch.arange(E, device="cuda", dtype=torch.int32))
    x, xn = drawn(rng, (T, d), dtype)
    ids = _chosen(rng, T, E, K, "even")      # every token takes every expert
    wt = rng.random((T, K)).astype(np.float32)
    want, bound = ref.moe_experts(xn, ids, wt, slots, np.arange(E), d, f, xn, dtype)
    close(fm.moe_experts(cache, x, dev(ids), dev(wt), residual=x), want, bound, dtype)


# A pass takes as many tokens as 256 MB hold of 8 x f float32 values: 128 at f =
# 65,536 (passes of 128, 128 and 44), 512 at 16,384 (512 and 188, 512 and 100).
PASSES = [(300, 8, 65536, 9), (700, 64, 16384, 12), (612, 64, 16384, 12)]


def _wide(rng, T, d, f, E, dtype):
    fm = _fm()
    cache, slots = _layer(rng, E, E, d, f, dtype)
    cache.slot_of.copy_(torch.arange(E, device="cuda", dtype=torch.int32))
    x, xn = drawn(rng, (T, d), dtype)
    ids = _chosen(rng, T, E, 8, "skewed")
    ids[T // 2] = -1
    ids[T - 1, 3] = -1
    ws = fm.MoeWorkspace(cache, T, 8)
    ws.buf.random_(0, 255)
    return cache, slots, x, xn, ids, rng.random((T, 8)).astype(np.float32), ws


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,f,E", PASSES)
def test_passes_of_wide_experts(T, d, f, E, dtype):
    print(f"experts T={T} d={d} f={f} E={E} {dtype}", flush=True)
    fm = _fm()
    rng = np.random.default_rng(T)
    cache, slots, x, xn, ids, wt, ws = _wide(rng, T, d, f, E, dtype)
    cut = 128 if f == 65536 else 512
    some = np.unique(np.concatenate([[0, T // 2, T - 1], np.arange(cut - 3, cut + 3), np.arange(T - T % cut - 3, T, 17)]))
    want, bound = ref.moe_experts(xn[some], ids[some], wt[some], slots, np.arange(E), d, f, xn[some], dtype)
    y = x.clone()
    fm.moe_experts(cache, y, dev(ids), dev(wt), residual=y, out=y, workspace=ws)
    close(y[dev(some)], want, bound, dtype, "in place")
    assert torch.equal(y, fm.moe_experts(cache, x, dev(ids), dev(wt), residual=x, workspace=ws))
    assert cache.check() == 0


@pytest.mark.parametrize("T,d,f,E", PASSES[:2])
def test_passes_in_a_graph(T, d, f, E):
    """Replays, with other work between, equal the eager results."""
    fm = _fm()
    rng = np.random.default_rng(T + 1)
    cache, _, x, _, ids, wt, ws = _wide(rng, T, d, f, E, "bf16")
    ids, wt = dev(ids), dev(wt)
    y = torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fm.moe_experts(cache, x, ids, wt, residual=x, out=y, workspace=ws)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            fm.moe_experts(cache, x, ids, wt, residual=x, out=y, workspace=ws)
    for _ in range(4):
        x.copy_(drawn(rng, (T, d), "bf16")[0])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        assert torch.equal(got, fm.moe_experts(cache, x, ids, wt, residual=x, workspace=ws))
        torch.cuda.synchronize()
