"""Rows of many new tokens to the cache's pages and back: calls of at least 16,384
pieces (16 tokens of a head by 64 bytes), whose wavefronts take four pieces each and
whose stores pass the caches by.  Bit for bit at the documented places; everything
else stays as it was."""
import numpy as np
import pytest
import torch

from test_gpu_kv_pages import BITS, DT, SIZE, _fm, i32, pair, places

pytestmark = pytest.mark.gpu


def _maps(c, layer):
    """Elements of a page: keys and values [page][heads][head_dim] of a layer, and which ones no layer's padding is."""
    at = [torch.from_numpy(places(c, layer, kv, c["page"], c["head_dim"])).cuda() for kv in (False, True)]
    n = 16 // c["size"]
    width = -(-c["head_dim"] * c["size"] // 64) * 4 * n
    whole = torch.zeros(c["layers"], 2, c["heads"] * c["page"] * width, dtype=torch.bool)
    for kv in (0, 1):
        one = torch.from_numpy(places({**c, "layers": 1}, 0, bool(kv), c["page"], c["head_dim"]).ravel())
        whole[:, kv, one - (kv * whole.shape[2])] = True
    return at, whole.view(-1).cuda()


def _written(before, table, page, at, slot, pos, rows):
    """The pages after rows [2][T][heads][head_dim] of bits went to the places pos of the slots."""
    want = before.clone()
    pages = table[slot, pos // page].long()
    for place, src in zip(at, rows):
        want[pages[:, None, None], place[pos % page]] = src
    return want


def _pieces(c, blocks):
    return blocks * c["heads"] * -(-c["head_dim"] * c["size"] // 64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,head_dim,page,mean", [(8, 200, 48, 750), (8, 128, 64, 900), (3, 72, 16, 3000),
                                                       (32, 40, 32, 500)])
def test_prompts_of_many_rows(heads, head_dim, page, mean, dtype):
    """Spans that begin and end inside blocks and pages, an idle slot, one without rows, one token, the last of several
    layers; rows between others of a wider tensor."""
    fm = _fm()
    print(f"heads={heads} head_dim={head_dim} page={page} mean={mean} {dtype}", flush=True)
    rng = np.random.default_rng(heads + head_dim)
    B, layers, layer = 12, 2, 1
    new = [int(n) for n in rng.integers(mean // 2, 3 * mean // 2, B)]
    new[3], new[5] = 0, 1
    before = [int(n) for n in rng.integers(0, 3 * page, B)]
    length = [a + n for a, n in zip(before, new)]
    T, held = sum(new), sum(-(-n // page) for n in length)
    cache, _ = pair(B, max(length) + page, held + 5, page, layers, heads, head_dim, dtype)
    c = dict(page=page, layers=layers, heads=heads, head_dim=head_dim, size=SIZE[dtype])
    assert _pieces(c, T // 16 + 2 * B) >= 16384
    fm.kv_resize(cache, i32(length))
    assert cache.check() == 0
    on = torch.ones(B, dtype=torch.uint8, device="cuda")
    on[7] = 0
    g = torch.Generator(device="cuda").manual_seed(1)
    kv = torch.randn(T, 2 * heads + 1, head_dim, generator=g, device="cuda").to(DT[dtype])
    k, v = kv[:, :heads], kv[:, heads:2 * heads]
    offsets = i32(np.cumsum([0] + new))
    raw = cache.pages.view(BITS[dtype])
    was = raw.clone()
    fm.kv_write(cache, layer, k, v, offsets=offsets, active=on)
    assert cache.check() == 0
    slot = torch.repeat_interleave(torch.arange(B), torch.tensor(new))
    pos = torch.cat([torch.arange(a, a + n) for a, n in zip(before, new)])
    taken = (slot != 7).cuda()
    slot, pos = slot.cuda(), pos.cuda()
    at, inside = _maps(c, layer)
    rows = [t.contiguous().view(BITS[dtype])[taken] for t in (k, v)]
    want = _written(was, cache.table, page, at, slot[taken], pos[taken], rows)
    assert torch.equal(raw[:, inside], want[:, inside])
    # padding of written rows is zero, other padding, pages and layers are untouched
    assert ((raw == want) | (raw == 0))[:, ~inside].all()
    untouched = torch.ones(len(raw), dtype=torch.bool, device="cuda")
    untouched[cache.table[slot[taken], pos[taken] // page].long()] = False
    assert untouched.sum() >= 5 and torch.equal(raw[untouched], was[untouched])
    # back: a slot that is idle leaves its rows alone
    out = torch.full((T, 2 * heads, head_dim), 7.0, device="cuda").to(DT[dtype])
    fm.kv_read(cache, layer, offsets=offsets, active=on, out=(out[:, :heads], out[:, heads:]))
    assert torch.equal(out[taken], kv[:, :2 * heads][taken]) and (out[~taken] == 7).all()
    assert cache.check() == 0 and torch.equal(raw[:, inside], want[:, inside])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,heads,head_dim,page", [(256, 32, 128, 16), (700, 17, 80, 32)])
def test_one_token_of_many_slots(B, heads, head_dim, page, dtype):
    """A row per slot: slots without tokens, idle ones, ones whose last page is shared or no page of the pool."""
    fm = _fm()
    print(f"B={B} heads={heads} head_dim={head_dim} page={page} {dtype}", flush=True)
    rng = np.random.default_rng(B)
    length = rng.integers(0, 2 * page + 1, B)
    length[:4], length[9:11] = [0, 1, page, page + 1], page // 2 + 1
    cache, _ = pair(B, 2 * page, int((-(-length // page)).sum()) + 3, page, 1, heads, head_dim, dtype)
    c = dict(page=page, layers=1, heads=heads, head_dim=head_dim, size=SIZE[dtype])
    assert _pieces(c, B) >= 16384
    fm.kv_resize(cache, i32(length))
    on = torch.from_numpy((rng.random(B) < 0.9).astype(np.uint8)).cuda()
    on[:12] = 1
    cache.table[9, 0] = 10 ** 6
    cache.refs[cache.table[10, 0].long()] = 2
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(B, heads, head_dim, generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
    raw = cache.pages.view(BITS[dtype])
    was = raw.clone()
    fm.kv_write(cache, 0, k, v, active=on)
    assert cache.check() == fm.FM_FLAG_INDEX_RANGE | fm.FM_FLAG_PAGE_SHARED
    slot = torch.arange(B, device="cuda")
    read = (on != 0) & (cache.length > 0) & (slot != 9)
    taken = read & (slot != 10)
    pos = cache.length.long() - 1
    at, inside = _maps(c, 0)
    rows = [t.view(BITS[dtype])[taken] for t in (k, v)]
    want = _written(was, cache.table, page, at, slot[taken], pos[taken], rows)
    assert torch.equal(raw[:, inside], want[:, inside])
    got = fm.kv_read(cache, 0, active=on)
    assert cache.check() == fm.FM_FLAG_INDEX_RANGE
    for t, g_, place in zip((k, v), got, at):
        assert torch.equal(g_[taken], t[taken]) and not g_[~read].any()
        held = raw[cache.table[10, 0].long()][place[page // 2]]
        assert torch.equal(g_[10].view(BITS[dtype]), held)
