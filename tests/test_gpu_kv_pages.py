"""The key-value cache's pages on the GPU through the public binding: sequences of
calls against oracle.layer.Pages (tables, counts and contents, bit for bit), rows
written and read at their documented places."""
import numpy as np
import pytest
import torch

from oracle import layer as ref

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
BITS = {"f32": torch.int32, "bf16": torch.int16}
SIZE = {"f32": 4, "bf16": 2}


def _fm():
    import paper_2502_05370_amd as fm
    return fm


def i32(a):
    return torch.tensor(np.asarray(a, np.int64), dtype=torch.int32, device="cuda")


def bits(t):
    return t.view(BITS["bf16" if t.dtype == torch.bfloat16 else "f32"]).cpu().numpy()


def pair(slots, max_tokens, pages, page=16, layers=1, heads=1, head_dim=8, dtype="bf16", seed=0):
    """A cache of random contents, and the oracle's."""
    cache = _fm().KvCache(slots, max_tokens, pages, layers, heads, head_dim, dtype, page=page)
    g = torch.Generator(device="cuda").manual_seed(seed)
    raw = cache.pages.view(BITS[dtype])
    raw.copy_(torch.randint(-2 ** 15, 2 ** 15, raw.shape, generator=g, device="cuda"))
    return cache, ref.Pages(cache.table.cpu().numpy(), cache.length.cpu().numpy(), cache.refs.cpu().numpy(),
                            bits(cache.pages), page)


def same(cache, want, what=""):
    for name in ("table", "length", "refs"):
        got = getattr(cache, name).cpu().numpy()
        assert (got == getattr(want, name)).all(), (what, name, got, getattr(want, name))
    live = want.refs > 0
    assert (bits(cache.pages)[live] == want.content[live]).all(), what
    want.check()


@pytest.mark.parametrize("slots,W,pages,page", [(1, 3, 2, 16), (5, 4, 12, 16), (70, 9, 300, 48), (1100, 3, 1500, 16),
                                                (12, 40, 5000, 32), (3, 200, 400, 16)])
def test_random_calls(slots, W, pages, page):
    """Growth, drops, forks, compactions and copies in any order, pages running out on the way."""
    fm = _fm()
    print(f"slots={slots} W={W} pages={pages} page={page}", flush=True)
    rng = np.random.default_rng(slots + W)
    cache, want = pair(slots, W * page, pages, page)
    refusals = 0
    for turn in range(40):
        kind = rng.choice(["resize", "resize", "one", "fork", "compact", "copy"])
        what = (turn, kind)
        if kind in ("resize", "one"):
            if kind == "one":
                delta = rng.integers(0, 2, slots)
            else:
                delta = np.where(rng.random(slots) < 0.5, rng.integers(-2 * page, 3 * page, slots), 0)
                delta[rng.random(slots) < 0.1] = -2 ** 31
                delta[rng.random(slots) < 0.02] = 2 ** 31 - 1
            granted = fm.kv_resize(cache, i32(delta)).cpu().numpy()
            g, refused = want.resize(delta)
            assert (granted == g).all(), what
            assert cache.check() == (fm.FM_FLAG_PAGES_FULL if refused else 0), what
            refusals += refused
        elif kind == "fork":
            parent = np.where(rng.random(slots) < 0.3, rng.integers(-1, slots, slots), -1)
            fm.kv_fork(cache, i32(parent))
            assert not want.fork(parent)
        elif kind == "compact":
            assert fm.kv_compact(cache).item() == want.compact()
        else:
            n = int(rng.integers(0, min(pages, 40) + 1))
            src, dst = rng.integers(0, pages, n), rng.integers(0, pages, n)
            fm.kv_copy(cache, i32(src), i32(dst))
            assert cache.check() == (fm.FM_FLAG_INDEX_RANGE if want.copy(src, dst) else 0), what
        same(cache, want, what)
    assert refusals > 0 or pages >= 400   # (the two largest pools may suffice)


@pytest.mark.parametrize("max_tokens", [160, 2048, 4096, 4112, 6000])
def test_forks_of_any_shape(max_tokens):
    """One parent of many, chains, cycles, itself, parents out of range, empty parents; tables that a workgroup holds
    and larger ones."""
    fm = _fm()
    cache, want = pair(8, max_tokens, 60)
    delta = [5, 16, 33, 100, 0, 1, 48, 47]
    fm.kv_resize(cache, i32(delta)), want.resize(delta)
    for parent in ([1, 2, 3, 0, -1, -1, -1, -1], [3] * 8, [0, 1, 2, 3, 4, 5, 6, 7], [4, 4, -1, -1, -1, 0, 1, 5],
                   [-5, 8, 2 ** 31 - 1, 1, -2 ** 31, 7, 6, 5]):
        fm.kv_fork(cache, i32(parent))
        assert cache.check() == (fm.FM_FLAG_INDEX_RANGE if want.fork(parent) else 0)
        same(cache, want, parent)
        delta = [1, 0, 1, 0, 1, 0, 1, 1]
        fm.kv_resize(cache, i32(delta)), want.resize(delta)
        same(cache, want, parent)


def test_large_pages_are_copied_whole():
    """Pages of more than one turn of a workgroup, not a multiple of it, for every kind of move."""
    fm = _fm()
    cache, want = pair(6, 256, 24, page=64, layers=3, heads=5, head_dim=72, dtype="f32")
    assert cache.page_bytes % 16384 != 0 and cache.page_bytes > 10 * 16384
    for step, call in (([70, 1, 0, 200, 0, 0], "resize"), ([-1, -1, 0, -1, 0, 3], "fork"), ([3, 0, 5, 9, 1, 1], "resize"),
                       ([-100, 0, 0, 0, 0, 0], "resize"), (None, "compact")):
        if call == "compact":
            fm.kv_compact(cache), want.compact()
        else:
            getattr(fm, "kv_" + call)(cache, i32(step)), getattr(want, call)(step)
        same(cache, want, call)
    fm.kv_copy(cache, i32([0, 1]), i32([22, 23])), want.copy([0, 1], [22, 23])
    assert (bits(cache.pages)[[22, 23]] == want.content[[22, 23]]).all()


def test_tables_that_do_not_fit():
    """Page numbers outside the pool, in tables that a caller filled: never followed, flagged; lengths past the table."""
    fm = _fm()
    cache, _ = pair(4, 64, 6)
    cache.table.copy_(i32([[0, 99, -1, -1], [-7, 1, -1, -1], [2, 3, 4, 5], [-1, -1, -1, -1]]))
    cache.length.copy_(i32([20, 17, 1000, -5]))
    cache.refs.copy_(i32([1, 1, 1, 1, 1, 1]))
    fm.kv_resize(cache, i32([1, 0, 1, 0]))          # behind page 99; past the table
    assert cache.check() == fm.FM_FLAG_INDEX_RANGE | fm.FM_FLAG_PAGES_FULL
    assert cache.length.tolist() == [20, 17, 1000, -5]
    fm.kv_fork(cache, i32([-1, -1, -1, 0]))
    assert cache.check() == fm.FM_FLAG_INDEX_RANGE and cache.refs.tolist() == [2, 1, 1, 1, 1, 1]
    fm.kv_resize(cache, i32([-50, -50, -16, -50]))
    assert cache.check() == fm.FM_FLAG_INDEX_RANGE
    assert cache.refs.tolist() == [0, 0, 1, 1, 1, 0] and cache.length.tolist() == [0, 0, 48, 0]
    k = torch.ones(4, 1, 8, dtype=torch.bfloat16, device="cuda")
    cache.table[2, 2] = 6
    fm.kv_write(cache, 0, k, k)
    assert cache.check() == fm.FM_FLAG_INDEX_RANGE


# ---------------------------------------------------------------- rows

def places(c, layer, values, T, head_dim):
    """[T][heads][head_dim] elements of a page."""
    return np.array([[[ref.place(c, layer, values, h, t, d) for d in range(head_dim)] for h in range(c["heads"])]
                     for t in range(T)])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("head_dim,heads,page,layers", [(8, 1, 16, 1), (64, 2, 32, 2), (72, 9, 48, 1), (128, 3, 64, 3),
                                                        (200, 1, 16, 2), (256, 17, 16, 1)])
def test_rows_land_at_their_places(head_dim, heads, page, layers, dtype):
    """Prompts and single tokens, spans that begin and end inside blocks and pages; nothing else changes but padding."""
    fm = _fm()
    print(f"head_dim={head_dim} heads={heads} page={page} layers={layers} {dtype}", flush=True)
    rng = np.random.default_rng(head_dim)
    B, layer = 6, layers - 1
    cache, _ = pair(B, 4 * page, 4 * B, page, layers, heads, head_dim, dtype)
    c = dict(page=page, layers=layers, heads=heads, head_dim=head_dim, size=SIZE[dtype])
    at = [places(c, layer, kv, page, head_dim) for kv in (False, True)]
    length = [1, 17, page, 2 * page + 5, 3 * page - 1, 40]
    fm.kv_resize(cache, i32(length))
    table = cache.table.cpu().numpy()
    raw = cache.pages.view(BITS[dtype])
    for new in ([1, 2, page, 2 * page + 5, 21, 0], [1, 1, 3, 7, 16, 23], None):
        before = raw.cpu().numpy().copy()
        n = [1] * B if new is None else new
        T = sum(n)
        # rows of a projection that holds keys and values side by side
        kv = torch.from_numpy(rng.standard_normal((T, 2 * heads + 1, head_dim)).astype(np.float32)).cuda().to(DT[dtype])
        k, v = kv[:, :heads], kv[:, heads:2 * heads]
        offsets = None if new is None else i32(np.cumsum([0] + new))
        fm.kv_write(cache, layer, k, v, offsets=offsets)
        assert cache.check() == 0
        want = before.copy()
        for src, place in ((k, at[0]), (v, at[1])):
            src = bits(src.contiguous())
            row = 0
            for s in range(B):
                for t in range(length[s] - n[s], length[s]):
                    want[table[s, t // page]][place[t % page]] = src[row]
                    row += 1
        got = raw.cpu().numpy()
        inside = np.zeros(got.shape[1], bool)
        for l in range(layers):
            for kv_ in (False, True):
                inside[places(c, l, kv_, page, head_dim).ravel()] = True
        assert (got[:, inside] == want[:, inside]).all()
        # padding of written rows is zero, other padding is untouched
        assert ((got[:, ~inside] == want[:, ~inside]) | (got[:, ~inside] == 0)).all()
        out = fm.kv_read(cache, layer, T=T, offsets=offsets)
        assert torch.equal(out[0], k) and torch.equal(out[1], v)
        wide = torch.full((T, 2 * heads, head_dim), 7.0, dtype=DT[dtype], device="cuda")
        fm.kv_read(cache, layer, offsets=offsets, out=(wide[:, :heads], wide[:, heads:]))
        assert torch.equal(wide[:, :heads], k) and torch.equal(wide[:, heads:], v)


def test_rows_that_are_left_out():
    """Idle slots, empty slots, more rows than tokens, shared pages, odd offsets."""
    fm = _fm()
    cache, _ = pair(5, 64, 20)
    fm.kv_resize(cache, i32([3, 20, 0, 18, 5]))
    rows = torch.arange(1, 9, device="cuda").to(torch.bfloat16)[:, None, None].expand(8, 1, 8).contiguous()
    before = bits(cache.pages)
    on = torch.tensor([1, 0, 1, 0, 0], dtype=torch.uint8, device="cuda")
    fm.kv_write(cache, 0, rows[:5], rows[:5], active=on)        # slot 2 holds nothing
    assert cache.check() == 0
    k, v = fm.kv_read(cache, 0)
    assert (k[0] == 1).all() and (v[0] == 1).all() and (k[2] == 0).all()
    changed = (bits(cache.pages) != before).any(axis=1)
    assert np.flatnonzero(changed).tolist() == [0]
    # slot 0 has 3 tokens for 4 rows; slot 1 takes its last 2; slot 3 none; slot 4's end lies past the rows
    fm.kv_write(cache, 0, rows, rows, offsets=i32([0, 4, 6, 6, 3, 100]))
    assert cache.check() == fm.FM_FLAG_INDEX_RANGE
    k, _ = fm.kv_read(cache, 0, T=8, offsets=i32([0, 3, 5, 5, 5, 8]))
    assert k[:, 0, 0].tolist()[3:] == [5.0, 6.0, 6.0, 7.0, 8.0] and k[2, 0, 0] == 1
    cache.check()
    fm.kv_fork(cache, i32([-1, -1, 1, -1, -1]))
    fm.kv_write(cache, 0, rows[:5], rows[:5])
    assert cache.check() == fm.FM_FLAG_PAGE_SHARED
    k, _ = fm.kv_read(cache, 0)
    assert k[:, 0, 0].tolist() == [1.0, 6.0, 6.0, 4.0, 5.0]
    # spans that overlap: every slot's tokens from the same rows, more blocks than ascending offsets have
    cache, _ = pair(3, 64, 12)
    fm.kv_resize(cache, i32([40, 40, 40]))
    many = torch.arange(40, device="cuda").to(torch.bfloat16)[:, None, None].expand(40, 1, 8).contiguous()
    out = torch.zeros_like(many), torch.zeros_like(many)
    for s in range(3):
        lo = [0, 0, 0, 0]
        lo[s + 1:] = [40] * (3 - s)
        fm.kv_write(cache, 0, many + s, many, offsets=i32(lo))
    for s in range(3):
        lo = [0] * (s + 1) + [40] * (3 - s)
        fm.kv_read(cache, 0, offsets=i32(lo), out=out)
        assert torch.equal(out[0], many + s) and torch.equal(out[1], many)


def test_offsets_that_fall_back():
    """Offsets that do not ascend name the same rows for several slots: all are written."""
    fm = _fm()
    cache, _ = pair(7, 64, 40)
    fm.kv_resize(cache, i32([40] * 7))
    rows = torch.arange(1, 41, device="cuda").to(torch.bfloat16)[:, None, None].expand(40, 1, 8).contiguous()
    fm.kv_write(cache, 0, rows, rows, offsets=i32([0, 40, 0, 40, 0, 40, 0, 40]))
    for s in range(7):
        out = torch.zeros_like(rows), torch.zeros_like(rows)
        fm.kv_read(cache, 0, offsets=i32([0] * (s + 1) + [40] * (7 - s)), out=out)
        want = rows if s % 2 == 0 else 0 * rows
        if s % 2 == 0:
            assert torch.equal(out[0], want) and torch.equal(out[1], want)
    assert cache.check() == 0
