"""Infinities, NaN and pages outside the pool in sequences that several workgroups
share: whole parts of a sequence without a score, or with nothing but NaN, joined
with others."""
import numpy as np
import pytest
import torch

from oracle import layer as ref
from oracle.operators import rounding
from test_gpu_attention import check, drawn, filled
from test_gpu_kv_pages import DT, _fm, i32

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")
SCALE = np.float32(0.125)


def _cache(rng, n, B, dtype, page=64):
    """B slots of n tokens, one key head of 64; queries with a first dimension of 1."""
    cache, k, v = filled(rng, [n] * B, 1, 64, page, dtype)
    q, _ = drawn(rng, (B, 3, 64), dtype)
    q[:, :, 0] = 1.0
    return cache, q, [torch.from_numpy(x.copy()) for x in k], [torch.from_numpy(x.copy()) for x in v]


def _attend(cache, q, k, v, dtype):
    n = [len(t) for t in k]
    kt, vt = (torch.cat(t).cuda().to(DT[dtype]) for t in (k, v))
    _fm().kv_write(cache, 0, kt, vt, offsets=i32(np.cumsum([0] + n)))
    lse = torch.empty(q.shape[:2], device="cuda")
    got = _fm().attn_decode(cache, 0, q, lse=lse)
    assert cache.check() == 0
    return got, lse


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1500, 3000, 20000])
def test_parts_without_a_score(n, dtype):
    """Scores of minus infinity across whole parts, but for one token, and everywhere."""
    print(f"n={n} {dtype}", flush=True)
    rng = np.random.default_rng(n)
    cache, q, k, v = _cache(rng, n, 6, dtype)
    keep = [[i for i in range(n) if not n // 5 <= i < 3 * n // 5], range(n - 1, n), range(1), [], range(n // 2, n // 2 + 1),
            [i for i in range(n) if i % 1000 < 100]]
    for s in range(6):
        gone = np.ones(n, bool)
        gone[list(keep[s])] = False
        k[s][torch.from_numpy(gone), 0, 0] = -INF
    got, lse = _attend(cache, q, k, v, dtype)
    check(got, lse, q.float().cpu().numpy(), [k[s].numpy()[list(keep[s])] for s in range(6)],
          [v[s].numpy()[list(keep[s])] for s in range(6)], SCALE, dtype)
    assert (got[3] == 0).all() and (lse[3] == -INF).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1500, 3000, 20000])
def test_infinities_and_nan_in_one_part(n, dtype):
    """A score of NaN or plus infinity anywhere is NaN everywhere, also where no other token of its part, or of the
    whole sequence, has a score; infinite values are those of their column."""
    print(f"n={n} {dtype}", flush=True)
    rng = np.random.default_rng(n + 1)
    cache, q, k, v = _cache(rng, n, 8, dtype)
    k[0][n // 2, 0, 3] = NAN
    k[1][n - 1, 0, 0], k[2][5, 0, 0] = INF, INF
    k[1][:, 0, 1:], k[2][:, 0, 1:] = 0, 0
    k[3][n // 4: 3 * n // 4, 0, 0] = -INF
    k[3][n // 2, 0, 0] = NAN
    k[4][:, 0, 0] = -INF
    k[4][n // 3, 0, 0] = NAN
    v[5][n // 3, 0, 3], v[5][n - 1, 0, 4], v[5][7, 0, 5] = INF, -INF, NAN
    v[6][n // 3, 0, 3], v[6][n - 2, 0, 3] = INF, -INF
    got, lse = _attend(cache, q, k, v, dtype)
    for s in range(5):
        assert torch.isnan(got[s]).all() and torch.isnan(lse[s]).all(), s
    assert (got[5, :, 3] == INF).all() and (got[5, :, 4] == -INF).all() and torch.isnan(got[5, :, 5]).all()
    assert torch.isnan(got[6, :, 3]).all()
    qn = q.float().cpu().numpy()
    for s in (5, 6, 7):
        rest = [d for d in range(64) if s == 7 or d not in (3, 4, 5)]
        for h in range(3):
            clean = v[s][:, 0].numpy().copy()
            clean[~np.isfinite(clean)] = 0
            want, bound, l, lb = ref.attention(qn[s, h], k[s][:, 0].numpy(), clean, SCALE, dtype)
            limit = bound + rounding(dtype) * (np.abs(want) + bound) * (1 + 2.0 ** -8)
            assert (np.abs(got[s, h].float().cpu().numpy() - want)[rest] <= limit[rest]).all()
            assert abs(float(lse[s, h]) - l) <= lb


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1500, 3000, 20000])
def test_parts_on_pages_outside_the_pool(n, dtype):
    """A quarter of a sequence, its end, and all of it on pages that there are not."""
    print(f"n={n} {dtype}", flush=True)
    rng = np.random.default_rng(n + 2)
    cache, q, k, v = _cache(rng, n, 4, dtype)
    entries = -(-n // 64)
    gone = [range(entries // 4, entries // 2), range(entries - 2, entries), range(entries), range(0)]
    for s in range(4):
        for i in gone[s]:
            cache.table[s, i] = 10 ** 7 if i % 2 else -1
    lse = torch.empty(q.shape[:2], device="cuda")
    got = _fm().attn_decode(cache, 0, q, lse=lse)
    assert cache.check() == _fm().FM_FLAG_INDEX_RANGE
    keep = [[t for t in range(n) if t // 64 not in gone[s]] for s in range(4)]
    check(got, lse, q.float().cpu().numpy(), [k[s].numpy()[keep[s]] for s in range(4)],
          [v[s].numpy()[keep[s]] for s in range(4)], SCALE, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_an_end_as_long_as_a_part_that_nothing_sees(dtype):
    """Windows and first tokens that leave whole parts' worth of tokens out, filled with NaN."""
    rng = np.random.default_rng(5)
    n = 9000
    cache, q, k, v = _cache(rng, n, 3, dtype)
    for s, (lo, hi) in enumerate([(0, 8000), (0, 4001), (0, 0)]):
        k[s][lo:hi], v[s][lo:hi] = NAN, NAN
    kt, vt = (torch.cat(t).cuda().to(DT[dtype]) for t in (k, v))
    _fm().kv_write(cache, 0, kt, vt, offsets=i32([0, n, 2 * n, 3 * n]))
    first = i32([8000, 4001, 0])
    lse = torch.empty(3, 3, device="cuda")
    got = _fm().attn_decode(cache, 0, q, first=first, lse=lse)
    check(got, lse, q.float().cpu().numpy(), [t.numpy() for t in k], [t.numpy() for t in v], SCALE, dtype, [8000, 4001, 0])
