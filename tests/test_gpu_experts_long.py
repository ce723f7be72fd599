"""The chosen experts' products of long batches (a prompt's tokens), against the
float64 definition of oracle.operators, and against the same tokens in short
calls."""
import numpy as np
import pytest
import torch

from oracle import operators as ref
from test_gpu_operators import _fm, _layer, close, dev, drawn

pytestmark = pytest.mark.gpu


def _chosen(rng, T, E, K, law):
    """[T][K] experts without repetition; "skewed": low numbers take most tokens,
    so that experts hold from none to several hundred."""
    p = np.ones(E) / E if law == "even" else 1.0 / np.arange(1, E + 1) ** 2
    score = np.log(p / p.sum()) + rng.gumbel(size=(T, E))
    return np.argsort(-score, axis=1)[:, :K].astype(np.int32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,f,E,K,law", [(129, 8, 8, 1, 1, "even"), (129, 264, 136, 4, 2, "even"),
                                           (257, 72, 264, 7, 3, "skewed"), (300, 1032, 72, 4, 2, "even"),
                                           (700, 136, 520, 9, 2, "skewed"), (1000, 104, 24, 64, 8, "skewed"),
                                           (640, 512, 256, 5, 1, "even"),
                                           # enough units of rows for the wide ones, of either product
                                           (640, 64, 4104, 10, 2, "even"), (640, 8200, 64, 10, 2, "even")])
def test_long_batch(T, d, f, E, K, law, dtype):
    print(f"experts T={T} d={d} f={f} E={E} K={K} {law} {dtype}", flush=True)
    fm = _fm()
    rng = np.random.default_rng(T + d + f)
    S = E + 2
    cache, slots = _layer(rng, E, S, d, f, dtype)
    slot_of = rng.permutation(S)[:E].astype(np.int32)
    if E > 5:
        slot_of[1] = -1                      # not held
    cache.slot_of.copy_(dev(slot_of))
    x, xn = drawn(rng, (T, d), dtype)
    res, rn = drawn(rng, (T, d), dtype)
    ids = _chosen(rng, T, E, K, law)
    ids[T // 2, K // 2] = -1
    ids[5] = -1                              # a token without experts
    ids[6] = ids[6, 0]                       # one expert, K times
    wt = rng.random((T, K)).astype(np.float32)
    ws = fm.MoeWorkspace(cache, T, K)
    ws.buf.random_(0, 255)
    want, bound = ref.moe_experts(xn, ids, wt, slots, slot_of, d, f, rn, dtype)
    got = fm.moe_experts(cache, x, dev(ids), dev(wt), residual=res, workspace=ws)
    close(got, want, bound, dtype)
    assert cache.check() == (fm.FM_FLAG_EXPERT_MISSING if E > 5 and (ids == 1).any() else 0)
    assert torch.equal(got, fm.moe_experts(cache, x, dev(ids), dev(wt), residual=res, workspace=ws))
    # in place, without a residual, and then over the input
    want, bound = ref.moe_experts(xn, ids, wt, slots, slot_of, d, f, None, dtype)
    close(fm.moe_experts(cache, x, dev(ids), dev(wt), workspace=ws), want, bound, dtype, "no residual")
    y = x.clone()
    fm.moe_experts(cache, y, dev(ids), dev(wt), residual=y, out=y, workspace=ws)
    want, bound = ref.moe_experts(xn, ids, wt, slots, slot_of, d, f, xn, dtype)
    close(y, want, bound, dtype, "in place")


@pytest.mark.parametrize("T", [145, 160, 192, 255, 256, 300])
def test_long_batch_on_one_expert(T):
    """Every size of an expert's last group of places."""
    fm = _fm()
    rng = np.random.default_rng(T)
    d, f, E = 136, 136, 3
    cache, slots = _layer(rng, E, E, d, f, "bf16")
    cache.slot_of.copy_(torch.arange(E, device="cuda", dtype=torch.int32))
    x, xn = drawn(rng, (T, d), "bf16")
    ids = np.full((T, 1), 2, np.int32)
    wt = rng.random((T, 1)).astype(np.float32)
    want, bound = ref.moe_experts(xn, ids, wt, slots, np.arange(E), d, f, None, "bf16")
    close(fm.moe_experts(cache, x, dev(ids), dev(wt)), want, bound, "bf16")


@pytest.mark.parametrize("rest", [3, 40, 100, 1000])
def test_more_than_one_launch_of_a_long_batch(rest):
    """4,096 tokens and some more: each token as in a call of its own neighbours."""
    fm = _fm()
    rng = np.random.default_rng(rest)
    d, f, E, K, T = 64, 72, 64, 8, 4096 + rest
    cache, slots = _layer(rng, E, E, d, f, "f32")
    cache.slot_of.copy_(torch.arange(E, device="cuda", dtype=torch.int32))
    x, xn = drawn(rng, (T, d), "f32")
    ids = _chosen(rng, T, E, K, "skewed")
    wt = rng.random((T, K)).astype(np.float32)
    got = fm.moe_experts(cache, x, dev(ids), dev(wt), residual=x)
    some = np.unique(np.concatenate([np.arange(0, 4096, 97), np.arange(4090, T)[:40], [T - 1]]))
    want, bound = ref.moe_experts(xn[some], ids[some], wt[some], slots, np.arange(E), d, f, xn[some], "f32")
    close(got[dev(some)], want, bound, "f32")


def test_long_batch_nothing_to_do():
    fm = _fm()
    rng = np.random.default_rng(0)
    cache, _ = _layer(rng, 6, 2, 64, 32, "bf16")
    cache.weights.fill_(float("nan"))
    T = 200
    x, _ = drawn(rng, (T, 64), "bf16")
    ids = torch.full((T, 2), -1, dtype=torch.int32, device="cuda")
    w = torch.ones(T, 2, device="cuda")
    assert torch.equal(fm.moe_experts(cache, x, ids, w, residual=x), x)
    assert (fm.moe_experts(cache, x, ids, w) == 0).all() and cache.check() == 0
    ids[130, 0] = 1
    assert (fm.moe_experts(cache, x, ids, w) == 0).all() and cache.check() == fm.FM_FLAG_EXPERT_MISSING
    ids[130, 0], cache.slot_of[1] = 6, 2
    ids[40, 1] = 1
    assert (fm.moe_experts(cache, x, ids, w) == 0).all() and cache.check() == fm.FM_FLAG_INDEX_RANGE


def test_long_batch_keeps_apart():
    """NaN and infinities stay with the token, the expert and the row that hold them."""
    fm = _fm()
    rng = np.random.default_rng(3)
    d, f, E, T = 72, 40, 5, 333
    cache, _ = _layer(rng, E, E, d, f, "bf16")
    cache.slot_of.copy_(torch.arange(E, device="cuda", dtype=torch.int32))
    x, _ = drawn(rng, (T, d), "bf16")
    ids = dev(_chosen(rng, T, 4, 2, "even"))
    wt = torch.rand(T, 2, device="cuda")
    clean = fm.moe_experts(cache, x, ids, wt, residual=x)
    cache.weights[4] = float("nan")                # an expert that no token takes
    assert torch.equal(clean, fm.moe_experts(cache, x, ids, wt, residual=x))
    bad = x.clone()
    bad[211] = float("inf")
    got = fm.moe_experts(cache, bad, ids, wt, residual=x)
    keep = torch.arange(T, device="cuda") != 211
    assert not torch.isfinite(got[211]).any() and torch.equal(got[keep], clean[keep])
    ids[2, 0] = 4
    got = fm.moe_experts(cache, x, ids, wt, residual=x)
    keep = torch.arange(T, device="cuda") != 2
    assert torch.isnan(got[2]).all() and torch.equal(got[keep], clean[keep])
    cache.weights[4] = cache.weights[0]
    base = fm.moe_experts(cache, x, ids, wt, residual=x)
    cache.weights[4, 2 * d * f + 70 * f + 3] = float("nan")
    got = fm.moe_experts(cache, x, ids, wt, residual=x)
    assert torch.isnan(got[2, 70]) and torch.isnan(got).sum() == 1
    got[2, 70] = base[2, 70]
    assert torch.equal(got, base)


def test_far_slots_of_a_long_batch():
    """An expert in the first slot and in one past 2^32 elements; the long batch
    agrees with its tokens in short calls to the rounding of the output."""
    fm = _fm()
    rng = np.random.default_rng(5)
    slots, d, f, T = 90, 4096, 4096, 300
    cache = fm.ExpertCache(slots, 2, d, f)
    cache.weights[0].normal_(std=d ** -0.5)
    cache.weights[1:-1] = float("nan")
    cache.weights[-1] = cache.weights[0]
    x, _ = drawn(rng, (T, d), "bf16")
    ids = torch.zeros((T, 1), dtype=torch.int32, device="cuda")
    w = torch.ones((T, 1), device="cuda")
    out = []
    for s in (0, slots - 1):
        cache.slot_of[0] = s
        out.append(fm.moe_experts(cache, x, ids, w))
    assert torch.isfinite(out[0]).all() and torch.equal(*out)
    short = torch.cat([fm.moe_experts(cache, x[i:i + 100], ids[:100], w[:100]) for i in range(0, T, 100)])
    torch.testing.assert_close(out[0].float(), short.float(), rtol=2.0 ** -7, atol=2.0 ** -9)
