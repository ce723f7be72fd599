"""Paged attention where the batch's work is dealt out in ways that only large
batches meet: tiles of a few steps that a wavefront takes alone, groups of longer
tiles with one for each wavefront, two workgroups per CU by the lengths, and more
than 128 queries per key head, whose tiles take turns."""
import numpy as np
import pytest
import torch

from oracle import layer as ref
from oracle.operators import rounding
from test_gpu_attention import check, drawn, filled
from test_gpu_kv_pages import DT, _fm, i32

pytestmark = pytest.mark.gpu


def _large(length, heads, head_dim, page, dtype, seed):
    """A cache of these lengths on shuffled pages, everything else NaN -> cache, keys, values [tokens][heads][head_dim] on
    the GPU."""
    fm = _fm()
    g = torch.Generator(device="cuda").manual_seed(seed)
    pages = [-(-n // page) for n in length]
    W, need = max(1, max(pages)) + 1, sum(pages)
    cache = fm.KvCache(len(length), W * page, need + 3, 1, heads, head_dim, dtype, page=page)
    cache.pages.fill_(float("nan"))
    order = torch.randperm(need + 3, generator=g, device="cuda")[:need].to(torch.int32)
    used = torch.arange(W, device="cuda")[None, :] < torch.tensor(pages, device="cuda")[:, None]
    cache.table[used] = order
    cache.refs[order.long()] = 1
    cache.length.copy_(i32(length))
    k, v = (torch.randn(sum(length), heads, head_dim, generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
    fm.kv_write(cache, 0, k, v, offsets=i32(np.cumsum([0] + list(length))))
    return cache, k, v


def _sample(rng, got, lse, q, k, v, length, dtype, n=400):
    """Random query heads of all slots against the oracle; every value finite."""
    B, Hq, D = q.shape
    assert torch.isfinite(got).all()
    ends = np.cumsum([0] + list(length))
    for s, h in zip(rng.integers(0, B, n), rng.integers(0, Hq, n)):
        head = int(h) // (Hq // k.shape[1])
        rows = slice(int(ends[s]), int(ends[s + 1]))
        kn, vn = (t[rows, head].float().cpu().numpy() for t in (k, v))
        want, bound, l, lb = ref.attention(q[s, h].float().cpu().numpy(), kn, vn, np.float32(D ** -0.5), dtype)
        limit = bound + rounding(dtype) * (np.abs(want) + bound) * (1 + 2.0 ** -8) + 2.0 ** -120
        off = np.abs(got[s, h].float().cpu().numpy().astype(np.float64) - want)
        assert (off <= limit).all(), (s, h, length[s], off.max())
        assert float(lse[s, h]) == l or abs(float(lse[s, h]) - l) <= lb, (s, h, length[s])


# heads, head_dim, group, slots, lengths from and below: with one query head on each, steps of 32 to 128 tokens
CASES = [(32, 64, 1, 64, 70, 125), (32, 64, 2, 64, 0, 130), (32, 72, 1, 128, 380, 420), (32, 128, 1, 64, 780, 820),
         (32, 96, 3, 96, 200, 260), (16, 16, 4, 200, 1, 700), (8, 128, 4, 300, 0, 300), (4, 256, 2, 256, 30, 90)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,head_dim,group,B,lo,hi", CASES)
def test_many_short_tiles(heads, head_dim, group, B, lo, hi, dtype):
    print(f"heads={heads} head_dim={head_dim} group={group} B={B} lengths {lo}..{hi} {dtype}", flush=True)
    rng = np.random.default_rng(heads + head_dim + B)
    length = [int(n) for n in rng.integers(lo, hi, B)]
    length[B // 2] = 5 * hi + 3       # one that is not like the others
    cache, k, v = _large(length, heads, head_dim, 32, dtype, B)
    g = torch.Generator(device="cuda").manual_seed(2)
    q = torch.randn(B, heads * group, head_dim, generator=g, device="cuda").to(DT[dtype])
    lse = torch.empty(B, heads * group, device="cuda")
    got = _fm().attn_decode(cache, 0, q, lse=lse)
    assert cache.check() == 0
    _sample(rng, got, lse, q, k, v, length, dtype)
    again = torch.empty_like(lse)
    assert torch.equal(got, _fm().attn_decode(cache, 0, q, lse=again)) and torch.equal(lse, again)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group,heads,head_dim", [(129, 1, 64), (145, 2, 40), (300, 1, 72), (300, 3, 128), (511, 2, 32),
                                                  (1024, 1, 64), (200, 1, 256)])
def test_more_than_128_queries_per_key_head(group, heads, head_dim, dtype):
    """Nine tiles of 16 queries and more take turns; the last turn has workgroups without a query.  Sequences that are
    empty, a wavefront's, a workgroup's, and cut."""
    print(f"group={group} heads={heads} head_dim={head_dim} {dtype}", flush=True)
    rng = np.random.default_rng(group + head_dim)
    for length, window in (([1, 0, 16, 37, 250, 3], 0), ([5000, 2, 0, 1300], 0), ([700, 90], 333)):
        cache, k, v = filled(rng, length, heads, head_dim, 32, dtype)
        q, qn = drawn(rng, (len(length), group * heads, head_dim), dtype)
        lse = torch.empty(len(length), group * heads, device="cuda")
        raw = torch.full((q.numel() + 512,), 5.0, device="cuda").to(DT[dtype])
        got = raw[256:256 + q.numel()].view(q.shape)
        ws = _fm().AttnWorkspace(cache, group * heads)
        _fm().attn_decode(cache, 0, q, window=window, lse=lse, out=got, workspace=ws)
        lo = [max(0, n - window) if window else 0 for n in length]
        check(got, lse, qn, k, v, np.float32(head_dim ** -0.5), dtype, lo)
        assert cache.check() == 0 and (raw[:256] == 5).all() and (raw[256 + q.numel():] == 5).all()
        from paper_2502_05370_amd import _lib
        assert not ws.buf[: _lib.FM_ATTN_TICKET_BYTES].any()
        assert torch.equal(got, _fm().attn_decode(cache, 0, q, window=window, workspace=ws))
