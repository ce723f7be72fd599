"""Attention of one new token per slot over a paged cache, on the GPU, against
oracle.layer.attention within its bound and one rounding of the output's type.
Every page starts as NaN, so that whatever lies outside a slot's tokens would
show in its result."""
import numpy as np
import pytest
import torch

from oracle import layer as ref
from oracle.operators import rounding
from test_gpu_kv_pages import DT, _fm, i32

pytestmark = pytest.mark.gpu


def drawn(rng, shape, dtype, scale=1.0):
    t = torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).cuda().to(DT[dtype])
    return t, t.float().cpu().numpy()


def filled(rng, length, heads, head_dim, page, dtype, layers=1, layer=0, spare=3, scale=1.0):
    """A cache of slots of these lengths on shuffled pages -> (cache, keys, values by slot)."""
    fm = _fm()
    B, W = len(length), max(1, -(-max(length) // page) + 1)
    need = sum(-(-n // page) for n in length)
    cache = fm.KvCache(B, W * page, need + spare, layers, heads, head_dim, dtype, page=page)
    cache.pages.fill_(float("nan"))
    order = rng.permutation(need + spare)
    table, refs, at = np.full((B, W), -1), np.zeros(need + spare), 0
    for s, n in enumerate(length):
        p = -(-n // page)
        table[s, :p] = order[at:at + p]
        refs[order[at:at + p]] = 1
        at += p
    cache.table.copy_(i32(table)), cache.length.copy_(i32(length)), cache.refs.copy_(i32(refs))
    T = sum(length)
    k, kn = drawn(rng, (T, heads, head_dim), dtype, scale)
    v, vn = drawn(rng, (T, heads, head_dim), dtype)
    fm.kv_write(cache, layer, k, v, offsets=i32(np.cumsum([0] + list(length))))
    ends = np.cumsum(length)[:-1]
    return cache, np.split(kn, ends), np.split(vn, ends)


def check(got, lse, q, k, v, scale, dtype, lo=None, on=None, what=""):
    B, Hq, D = q.shape
    got, lse = got.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    for s in range(B):
        first = 0 if lo is None else min(max(0, lo[s]), len(k[s]))
        if on is not None and not on[s]:
            first = len(k[s])
        for h in range(Hq):
            head = h // (Hq // k[s].shape[1])
            want, bound, l, lb = ref.attention(q[s, h], k[s][first:, head], v[s][first:, head], scale, dtype)
            limit = bound + rounding(dtype) * (np.abs(want) + bound) * (1 + 2.0 ** -8) + 2.0 ** -120
            bad = ~(np.abs(got[s, h] - want) <= limit)
            assert not bad.any(), (what, s, h, np.flatnonzero(bad)[:4], got[s, h][bad][:4], want[bad][:4], limit[bad][:4])
            assert lse[s, h] == l or abs(lse[s, h] - l) <= lb, (what, s, h, lse[s, h], l, lb)


CASES = [   # lengths, query heads, heads, head_dim, page
    ([1], 1, 1, 8, 16), ([1, 2, 15, 16, 17, 31, 32, 33, 0, 48], 4, 2, 64, 16), ([300, 0, 5], 5, 1, 128, 32),
    ([64, 65, 63, 128], 16, 16, 128, 64), ([777, 100], 17, 1, 96, 48), ([129, 250], 24, 1, 80, 16),
    ([50, 1000], 8, 8, 16, 1024), ([333], 40, 1, 40, 32), ([90, 2], 14, 2, 256, 128), ([70, 45], 3, 3, 200, 16),
    ([2500, 31], 32, 4, 72, 256), ([5], 128, 2, 24, 16), ([140, 260], 6, 3, 160, 64), ([90], 2, 1, 192, 16),
    ([66], 2, 2, 224, 32), ([34, 200], 4, 4, 112, 16), ([520], 4, 1, 144, 16), ([61, 77], 2, 1, 176, 32),
    ([61, 77], 2, 1, 208, 32), ([40], 2, 1, 240, 16), ([100], 2, 1, 48, 16), ([18], 1, 1, 56, 16)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("length,q_heads,heads,head_dim,page", CASES)
def test_attention(length, q_heads, heads, head_dim, page, dtype):
    print(f"length={length} q_heads={q_heads} heads={heads} head_dim={head_dim} page={page} {dtype}", flush=True)
    rng = np.random.default_rng(sum(length) + head_dim)
    cache, k, v = filled(rng, length, heads, head_dim, page, dtype, layers=2, layer=1)
    q, qn = drawn(rng, (len(length), q_heads, head_dim), dtype)
    lse = torch.empty(len(length), q_heads, device="cuda")
    got = _fm().attn_decode(cache, 1, q, lse=lse)
    assert got.dtype == DT[dtype]
    check(got, lse, qn, k, v, np.float32(head_dim ** -0.5), dtype)
    assert cache.check() == 0
    again = _fm().attn_decode(cache, 1, q)
    assert torch.equal(got, again)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [0, 1, 15, 16, 17, 100, 5000])
def test_windows_first_tokens_and_idle_slots(window, dtype):
    rng = np.random.default_rng(window)
    length = [200, 1, 0, 37, 64, 130, 90, 2000]
    first = [-5, 0, 0, 36, 64, 129, 2 ** 31 - 1, 1000]
    on = [1, 1, 1, 1, 1, 0, 1, 1]
    cache, k, v = filled(rng, length, 2, 64, 32, dtype)
    q, qn = drawn(rng, (8, 6, 64), dtype)
    for use_first in (False, True):
        lse = torch.full((8, 6), 5.0, device="cuda")
        got = _fm().attn_decode(cache, 0, q, 0.3, window=window, first=i32(first) if use_first else None,
                                active=torch.tensor(on, dtype=torch.uint8, device="cuda"), lse=lse)
        lo = [max(0, first[s] if use_first else 0, length[s] - window if window else 0) for s in range(8)]
        check(got, lse, qn, k, v, np.float32(0.3), dtype, lo, on, (window, use_first))
    assert cache.check() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group,heads,head_dim", [
    (17, 1, 32), (24, 2, 64), (31, 1, 72), (32, 2, 96), (33, 1, 128), (48, 1, 128), (24, 1, 160), (17, 2, 176),
    (50, 1, 200), (20, 1, 224), (32, 1, 256), (128, 1, 64), (24, 1, 16), (18, 1, 56), (40, 1, 208)])
def test_more_than_sixteen_queries_per_key_head(group, heads, head_dim, dtype):
    """Tiles of 32 queries, whole and not; sequences that are one wavefront's, a workgroup's, and cut."""
    print(f"group={group} heads={heads} head_dim={head_dim} {dtype}", flush=True)
    rng = np.random.default_rng(group + head_dim)
    for length, window in (([1, 0, 16, 37, 250, 3], 0), ([5000, 2, 1300], 0), ([700, 90], 333)):
        cache, k, v = filled(rng, length, heads, head_dim, 32, dtype)
        q, qn = drawn(rng, (len(length), group * heads, head_dim), dtype)
        lse = torch.empty(len(length), group * heads, device="cuda")
        got = _fm().attn_decode(cache, 0, q, window=window, lse=lse)
        lo = [max(0, n - window) if window else 0 for n in length]
        check(got, lse, qn, k, v, np.float32(head_dim ** -0.5), dtype, lo)
        assert cache.check() == 0
        assert torch.equal(got, _fm().attn_decode(cache, 0, q, window=window))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale,spread", [(2.0, 4.0), (-1.5, 2.0), (0.0, 1.0), (1e-4, 1.0), (30.0, 3.0)])
def test_scores_of_any_size(scale, spread, dtype):
    """Sharp and flat weights, negative scales; scores in the thousands."""
    rng = np.random.default_rng(5)
    cache, k, v = filled(rng, [900, 64, 3], 1, 64, 16, dtype, scale=spread)
    q, qn = drawn(rng, (3, 4, 64), dtype, spread)
    lse = torch.empty(3, 4, device="cuda")
    check(_fm().attn_decode(cache, 0, q, scale, lse=lse), lse, qn, k, v, np.float32(scale), dtype)


def test_queries_that_are_parts_of_longer_rows():
    rng = np.random.default_rng(6)
    cache, k, v = filled(rng, [70, 41, 9], 2, 64, 16, "bf16")
    wide, wn = drawn(rng, (3, 12, 64), "bf16")
    lse = torch.empty(3, 4, device="cuda")
    got = _fm().attn_decode(cache, 0, wide[:, 3:7], lse=lse)
    check(got, lse, wn[:, 3:7], k, v, np.float32(0.125), "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_contexts(dtype):
    """More tokens than the units that the work is cut into, on many small pages; few and many slots."""
    rng = np.random.default_rng(7)
    cache, k, v = filled(rng, [70001, 3, 20000], 1, 32, 16, dtype)
    q, qn = drawn(rng, (3, 3, 32), dtype, 2.0)
    lse = torch.empty(3, 3, device="cuda")
    check(_fm().attn_decode(cache, 0, q, lse=lse), lse, qn, k, v, np.float32(32 ** -0.5), dtype)


def test_many_slots():
    """Hundreds of slots, most of them short, one long, some idle."""
    rng = np.random.default_rng(8)
    length = list(rng.integers(0, 40, 700))
    length[300] = 9000
    on = (rng.random(700) < 0.9).astype(int)
    on[300] = 1
    cache, k, v = filled(rng, [int(n) for n in length], 1, 64, 16, "bf16")
    q, qn = drawn(rng, (700, 2, 64), "bf16")
    lse = torch.empty(700, 2, device="cuda")
    got = _fm().attn_decode(cache, 0, q, active=torch.tensor(on, dtype=torch.uint8, device="cuda"), lse=lse)
    check(got, lse, qn, k, v, np.float32(0.125), "bf16", on=on)


def test_shared_pages():
    """Forked slots read the same pages, and their own after they have grown."""
    fm = _fm()
    rng = np.random.default_rng(9)
    cache, k, v = filled(rng, [45, 0, 0, 7], 2, 64, 16, "bf16", spare=10)
    fm.kv_fork(cache, i32([-1, 0, 0, -1]))
    granted = fm.kv_resize(cache, i32([1, 1, 0, 0]))
    assert granted.tolist() == [1, 1, 0, 0]
    rows, rn = drawn(rng, (4, 4, 64), "bf16")
    fm.kv_write(cache, 0, rows[:, :2], rows[:, 2:], active=granted)
    k, v = [k[0], k[0], k[0], k[3]], [v[0], v[0], v[0], v[3]]
    for s in range(2):
        k[s], v[s] = np.concatenate([k[s], rn[s: s + 1, :2]]), np.concatenate([v[s], rn[s: s + 1, 2:]])
    q, qn = drawn(rng, (4, 4, 64), "bf16")
    lse = torch.empty(4, 4, device="cuda")
    check(fm.attn_decode(cache, 0, q, lse=lse), lse, qn, k, v, np.float32(0.125), "bf16")
    assert cache.check() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinities_and_nan(dtype):
    """In visible places they follow the formula; in places that are not seen they have no part."""
    fm = _fm()
    rng = np.random.default_rng(10)
    n = 40
    cache, k, v = filled(rng, [n] * 6, 1, 64, 16, dtype)
    q, qn = drawn(rng, (6, 2, 64), dtype)
    inf, nan = float("inf"), float("nan")
    q[:, :, 0] = 1.0
    kt, vt = fm.kv_read(cache, 0, T=6 * n, offsets=i32(np.arange(7) * n))
    kt, vt = kt.view(6, n, 1, 64), vt.view(6, n, 1, 64)
    kt[0, 5, 0, 0] = -inf              # a token of no weight
    vt[1, 7, 0, 3], vt[1, 8, 0, 4], vt[1, 9, 0, 5] = inf, -inf, nan
    kt[2, :, 0, 0] = -inf              # no token of any weight
    kt[3, 11, 0, 2] = nan
    kt[4, 2, 0, 0], vt[4, 1] = nan, nan     # not seen by the window
    kt[5, 39, 0, 0] = inf
    kt[5, :, 0, 1:] = 0
    fm.kv_write(cache, 0, kt.view(-1, 1, 64), vt.view(-1, 1, 64), offsets=i32(np.arange(7) * n))
    lse = torch.empty(6, 2, device="cuda")
    got = fm.attn_decode(cache, 0, q, lse=lse).float()
    qn = q.float().cpu().numpy()
    kn, vn = kt.float().cpu().numpy(), vt.float().cpu().numpy()
    scale = np.float32(0.125)
    keep = [i for i in range(n) if i != 5]
    check(got[:1].to(DT[dtype]), lse[:1], qn[:1], [kn[0][keep]], [vn[0][keep]], scale, dtype)
    clean = vn[1].copy()
    clean[~np.isfinite(clean)] = 0
    assert (got[1, :, 3] == inf).all() and (got[1, :, 4] == -inf).all() and torch.isnan(got[1, :, 5]).all()
    rest = [d for d in range(64) if d not in (3, 4, 5)]
    for h in range(2):
        want, bound, *_ = ref.attention(qn[1, h], kn[1][:, 0], clean[:, 0], scale, dtype)
        limit = bound + rounding(dtype) * (np.abs(want) + bound) * (1 + 2.0 ** -8)
        assert (np.abs(got[1, h].cpu().numpy() - want)[rest] <= limit[rest]).all()
    assert (got[2] == 0).all() and (lse[2] == -inf).all()
    assert torch.isnan(got[3]).all() and torch.isnan(lse[3]).all()
    assert torch.isnan(got[5]).all()
    lse4 = torch.empty(6, 2, device="cuda")
    seen = fm.attn_decode(cache, 0, q, window=30, lse=lse4)
    check(seen[4:5], lse4[4:5], qn[4:5], [kn[4][10:]], [vn[4][10:]], scale, dtype)


def test_pages_outside_the_pool():
    """Their tokens are left out and flagged; so is nothing past the slot's end."""
    rng = np.random.default_rng(11)
    cache, k, v = filled(rng, [100, 100, 20], 1, 64, 16, "bf16")
    cache.table[0, 2], cache.table[1, 0], cache.table[1, 6], cache.table[2, 2] = 10 ** 6, -1, -2 ** 31, 77
    q, qn = drawn(rng, (3, 2, 64), "bf16")
    lse = torch.empty(3, 2, device="cuda")
    got = _fm().attn_decode(cache, 0, q, lse=lse)
    assert cache.check() == _fm().FM_FLAG_INDEX_RANGE
    keep = [[i for i in range(100) if not 32 <= i < 48], list(range(16, 96)), list(range(20))]
    check(got, lse, qn, [k[s][keep[s]] for s in range(3)], [v[s][keep[s]] for s in range(3)], np.float32(0.125), "bf16")
    cache.length.copy_(i32([10 ** 9, -3, 0]))     # lengths past the table, below zero
    cache.table.fill_(-1)
    got = _fm().attn_decode(cache, 0, q, lse=lse)
    assert (got == 0).all() and (lse == float("-inf")).all()
    assert cache.check() == _fm().FM_FLAG_INDEX_RANGE
