"""Attention where weights are far below the largest one, or zero, and values are
large or infinite."""
import math

import numpy as np
import pytest
import torch

from oracle import layer as ref
from oracle.operators import rounding
from test_gpu_attention import check, drawn, filled
from test_gpu_kv_pages import DT, _fm, i32

pytestmark = pytest.mark.gpu

LN2 = math.log(2.0)


def _scored(rng, scores, dtype, D=64, page=16):
    """A cache whose query (1, 0, 0, ...) scores the tokens of each slot like this -> cache, queries, keys, values [n][D]
    by slot (tensors that `put` writes again)."""
    length = [len(s) for s in scores]
    cache, _, v = filled(rng, length, 1, D, page, dtype)
    keys = [torch.zeros(n, 1, D) for n in length]
    for k, s in zip(keys, scores):
        k[:, 0, 0] = torch.tensor(s)
    values = [torch.from_numpy(x.copy()) for x in v]
    q = torch.zeros(len(scores), 2, D)
    q[:, :, 0] = 1.0
    return cache, q.to(DT[dtype]).cuda(), keys, values


def _put(cache, keys, values, dtype):
    """-> what the cache holds, float64 by slot."""
    k, v = (torch.cat(t).to(DT[dtype]).cuda() for t in (keys, values))
    ends = np.cumsum([0] + [len(t) for t in keys])
    _fm().kv_write(cache, 0, k, v, offsets=i32(ends))
    return tuple(np.split(t.double().cpu().numpy(), ends[1:-1]) for t in (k, v))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("low,size", [(-math.inf, 1e38), (-200.0, 1e36), (-200.0, 1e38)])
def test_large_values_of_no_weight(low, size, dtype):
    """Tokens whose score is minus infinity, or 288 powers of two below the others', have no part, whatever their
    values are: one part in 2^126 of each of 35 values of 10^38 (10^36) would be 41 (0.41).  A wavefront whose tokens
    all score -200 weighs them by 1 until it meets the others: eight of 10^38 or more are past float32, and the result
    is then no number."""
    rng = np.random.default_rng(1)
    cache, q, keys, values = _scored(rng, [[0.0] * 5 + [low] * 35, [low] * 20 + [0.0, 0.5] + [low] * 50], dtype)
    for s in range(2):
        values[s][keys[s][:, 0, 0] == low] = size
    k, v = _put(cache, keys, values, dtype)
    lse = torch.empty(2, 2, device="cuda")
    got = _fm().attn_decode(cache, 0, q, 1.0, lse=lse)
    keep = [range(5), range(20, 22)]
    for s in range(2):
        if low == -200.0 and size == 1e38 and torch.isnan(got[s]).all():
            continue
        check(got[s:s + 1], lse[s:s + 1], q[s:s + 1].float().cpu().numpy(), [k[s][keep[s]]], [v[s][keep[s]]],
              np.float32(1.0), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("power", [20, 70, 103, 111, 118, 122, 125])
def test_small_weights_keep_their_size(power, dtype):
    """One token of weight 2^-power, and values so large that it is all of the result.  A bf16 weight is off by 2^-15 of
    itself (in the oracle's bound), or by one step of the type at its smallest, 2^-133."""
    rng = np.random.default_rng(power)
    score = float(torch.tensor(-power * LN2).to(DT[dtype]))
    while score < -125.9 * LN2:      # (bf16 scores are rounded)
        score = float(torch.nextafter(torch.tensor(score).to(DT[dtype]), torch.tensor(0.0).to(DT[dtype])))
    cache, q, keys, values = _scored(rng, [[score] + [0.0] * 30, [0.0] * 30 + [score]], dtype)
    for s in range(2):
        values[s] = torch.zeros(31, 1, 64)
        values[s][keys[s][:, 0, 0] == score] = torch.from_numpy(rng.uniform(1, 2, (1, 64)).astype(np.float32)) * 2.0 ** power
    k, v = _put(cache, keys, values, dtype)
    got = _fm().attn_decode(cache, 0, q, 1.0).double().cpu().numpy()
    for s in range(2):
        want, bound, *_ = ref.attention(q[s, 0].double().cpu().numpy(), k[s][:, 0], v[s][:, 0], 1.0, dtype)
        limit = bound + (2.0 ** -133 * np.abs(v[s][:, 0]).sum(0) / 30 if dtype == "bf16" else 0.0)
        limit = limit + rounding(dtype) * (np.abs(want) + limit) * (1 + 2.0 ** -8)
        bad = np.abs(got[s] - want) > limit
        assert not bad.any(), (s, got[s][bad][:4], np.broadcast_to(want, got[s].shape)[bad][:4])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_values_of_any_weight(dtype):
    """An infinite value gives infinity under any weight that is not zero (one that is a whole power of two, that of a
    single token, tiny ones), and NaN under a weight of zero."""
    rng = np.random.default_rng(3)
    inf = math.inf
    scores = [[0.0], [0.0] * 7, [0.0] * 3 + [-70 * LN2] + [0.0] * 40, [0.0] * 3 + [-100 * LN2] + [0.0] * 40,
              [0.0] * 3 + [-124 * LN2] + [0.0] * 40, [0.0] * 3 + [-inf] + [0.0] * 40]
    at = [0, 4, 3, 3, 3, 3]
    cache, q, keys, values = _scored(rng, scores, dtype)
    for s in range(6):
        values[s][at[s], 0, 3:6] = torch.tensor([inf, -inf, math.nan])
    _put(cache, keys, values, dtype)
    got = _fm().attn_decode(cache, 0, q, 1.0).float()
    assert (got[:5, :, 3] == inf).all() and (got[:5, :, 4] == -inf).all() and torch.isnan(got[:, :, 5]).all()
    assert torch.isnan(got[5, :, 3:5]).all()
    rest = [d for d in range(64) if d not in (3, 4, 5)]
    assert torch.isfinite(got[:, :, rest]).all()
