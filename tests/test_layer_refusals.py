"""What the paged cache, its attention and the norms around a block refuse, before
anything reaches a GPU: status codes of the C ABI, sizes, and the binding's checks
of tensors (CPU only; no call enqueues anything)."""
import ctypes as C

import pytest
import torch

import paper_2502_05370_amd as fm
from paper_2502_05370_amd import _lib as L

P = 0x10000          # an aligned address; refused calls never follow it
lib = L.load()

CACHE = dict(n_slots=4, max_pages=8, n_pages=20, page=32, layers=2, heads=2, head_dim=64, dtype=1, pages=P, table=P,
             length=P, refs=P)
RESIZE = dict(delta=P, granted=None, flags=None, scratch=P, scratch_bytes=1 << 20, stream=None)
FORK = dict(parent=P, flags=None, scratch=P, scratch_bytes=1 << 20, stream=None)
COMPACT = dict(live=None, flags=None, scratch=P, scratch_bytes=1 << 20, stream=None)
COPY = dict(src=P, dst=P, n=3, flags=None, scratch=P, scratch_bytes=1 << 20, stream=None)
ROWS = dict(layer=1, k=P, k_stride=128, v=2 * P, v_stride=128, offsets=None, T=4, active=None, flags=None, stream=None)
ATTN = dict(layer=0, q=P, q_stride=512, q_heads=8, scale=0.1, window=0, first=None, active=None, out=2 * P, lse=None,
            flags=None, workspace=P, workspace_bytes=1 << 28, stream=None)
ON_CACHE = {"fm_kv_resize": RESIZE, "fm_kv_fork": FORK, "fm_kv_compact": COMPACT, "fm_kv_copy": COPY,
            "fm_kv_write": ROWS, "fm_kv_read": ROWS, "fm_attn_decode": ATTN}


@pytest.mark.parametrize("change,status", [
    (dict(n_slots=0), 1), (dict(n_slots=65537), 1), (dict(max_pages=0), 1), (dict(max_pages=(1 << 25) + 1), 2),
    (dict(n_slots=65536, max_pages=4097), 2), (dict(n_pages=0), 1), (dict(n_pages=(1 << 24) + 1), 1), (dict(page=0), 1),
    (dict(page=24), 2), (dict(page=1040), 2), (dict(layers=0), 1), (dict(layers=1025), 1), (dict(heads=0), 1),
    (dict(heads=1025), 1), (dict(head_dim=0), 1), (dict(head_dim=60), 2), (dict(head_dim=264), 2), (dict(dtype=2), 1),
    (dict(layers=1024, heads=64, head_dim=256, page=64), 2), (dict(pages=None), 1), (dict(pages=P + 16), 1),
    (dict(table=None), 1), (dict(table=P + 2), 1), (dict(length=None), 1), (dict(refs=None), 1), (dict(refs=P + 1), 1)])
@pytest.mark.parametrize("fn", list(ON_CACHE))
def test_cache_refused(fn, change, status):
    desc = L.KvCacheDesc(*{**CACHE, **change}.values())
    assert getattr(lib, fn)(C.byref(desc), *ON_CACHE[fn].values()) == status
    assert lib.fm_last_error().decode() != ""


@pytest.mark.parametrize("fn,change,status", [
    ("fm_kv_resize", dict(delta=None), 1), ("fm_kv_resize", dict(delta=P + 2), 1),
    ("fm_kv_resize", dict(scratch=None), 1), ("fm_kv_resize", dict(scratch=P + 128), 1),
    ("fm_kv_resize", dict(scratch_bytes=100), 1), ("fm_kv_resize", dict(flags=P + 1), 1),
    ("fm_kv_fork", dict(parent=None), 1), ("fm_kv_fork", dict(parent=P + 1), 1), ("fm_kv_fork", dict(scratch_bytes=0), 1),
    ("fm_kv_compact", dict(live=P + 2), 1), ("fm_kv_compact", dict(scratch=None), 1),
    ("fm_kv_copy", dict(n=-1), 1), ("fm_kv_copy", dict(n=21), 1), ("fm_kv_copy", dict(src=None), 1),
    ("fm_kv_copy", dict(dst=P + 2), 1), ("fm_kv_copy", dict(n=0, src=None, dst=None), 0),
    ("fm_kv_write", dict(layer=2), 1), ("fm_kv_write", dict(layer=-1), 1), ("fm_kv_write", dict(k=None), 1),
    ("fm_kv_write", dict(v=P + 8), 1), ("fm_kv_write", dict(k_stride=127), 1), ("fm_kv_write", dict(v_stride=132), 1),
    ("fm_kv_write", dict(T=3), 1), ("fm_kv_write", dict(T=-1, offsets=P), 1), ("fm_kv_write", dict(offsets=P + 2), 1),
    ("fm_kv_write", dict(T=0, offsets=P, k=None, v=None), 0), ("fm_kv_write", dict(flags=P + 2), 1),
    ("fm_kv_write", dict(T=(1 << 24) + 1, offsets=P), 1),
    ("fm_kv_read", dict(v=P), 1), ("fm_kv_read", dict(layer=2), 1), ("fm_kv_read", dict(k=None), 1), ("fm_kv_read", dict(T=3), 1),
    ("fm_attn_decode", dict(layer=2), 1), ("fm_attn_decode", dict(q=None), 1), ("fm_attn_decode", dict(q=P + 8), 1),
    ("fm_attn_decode", dict(q_stride=511), 1), ("fm_attn_decode", dict(q_stride=516), 1),
    ("fm_attn_decode", dict(q_heads=0), 1), ("fm_attn_decode", dict(q_heads=7), 1),
    ("fm_attn_decode", dict(q_heads=1026, q_stride=1 << 20), 1), ("fm_attn_decode", dict(window=-1), 1),
    ("fm_attn_decode", dict(scale=3e38), 1), ("fm_attn_decode", dict(scale=float("nan")), 1), ("fm_attn_decode", dict(scale=float("inf")), 1),
    ("fm_attn_decode", dict(first=P + 2), 1), ("fm_attn_decode", dict(lse=P + 2), 1), ("fm_attn_decode", dict(out=None), 1),
    ("fm_attn_decode", dict(out=P + 8), 1), ("fm_attn_decode", dict(out=P), 1), ("fm_attn_decode", dict(workspace=None), 1),
    ("fm_attn_decode", dict(workspace=P + 16), 1), ("fm_attn_decode", dict(workspace_bytes=0), 1)])
def test_calls_refused(fn, change, status):
    desc = L.KvCacheDesc(*CACHE.values())
    assert getattr(lib, fn)(C.byref(desc), *{**ON_CACHE[fn], **change}.values()) == status
    assert (lib.fm_last_error().decode() != "") == (status != 0)


def test_more_work_than_places():
    desc = L.KvCacheDesc(*{**CACHE, "n_slots": 65536, "max_pages": 4096, "page": 1024, "heads": 128}.values())
    desc.layers, desc.head_dim = 1, 8
    call = {**ATTN, "q_stride": 4096, "q_heads": 128}
    assert lib.fm_attn_workspace_bytes(C.byref(desc), 128) == 0
    assert lib.fm_attn_decode(C.byref(desc), *call.values()) == L.FM_ERR_UNSUPPORTED
    assert lib.fm_kv_scratch_bytes(C.byref(desc)) > 0


@pytest.mark.parametrize("fn", list(ON_CACHE))
def test_null_cache(fn):
    assert getattr(lib, fn)(None, *ON_CACHE[fn].values()) == L.FM_ERR_INVALID


NORM = dict(x=P, y=P, post=P, gate=P, kind=1, scale=1.0, pre=P, eps=1e-6, T=4, d=64, dtype=1, r=P, h=2 * P, stream=None)
GRAD = dict(dr=P, dh=P, x=P, y=P, post=P, gate=P, kind=1, scale=1.0, pre=P, eps=1e-6, T=4, d=64, dtype=1, accumulate=0,
            dx=P, dy=2 * P, dpost=3 * P, dgate=4 * P, dpre=5 * P, scratch=P, scratch_bytes=1 << 24, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=3), 1), (dict(T=-1), 1), (dict(T=(1 << 24) + 1), 1), (dict(d=0), 1), (dict(d=60), 2), (dict(d=16392), 2),
    (dict(kind=4), 1), (dict(kind=-1), 1), (dict(kind=0), 1), (dict(gate=None), 1), (dict(eps=-1e-6), 1),
    (dict(eps=float("nan")), 1), (dict(eps=float("inf")), 1), (dict(x=None), 1), (dict(y=None), 1), (dict(x=P + 8), 1),
    (dict(post=P + 4), 1), (dict(pre=P + 2), 1), (dict(gate=P + 8), 1), (dict(kind=2, gate=P + 1), 1)])
def test_norms_refused(change, status):
    for fn, base in (("fm_block_norm", NORM), ("fm_block_norm_grad", GRAD)):
        assert getattr(lib, fn)(*{**base, **change}.values()) == status
        assert lib.fm_last_error().decode() != ""


@pytest.mark.parametrize("fn,change,status", [
    ("fm_block_norm", dict(r=None), 1), ("fm_block_norm", dict(h=None), 1), ("fm_block_norm", dict(pre=None), 1),
    ("fm_block_norm", dict(h=P), 1), ("fm_block_norm_grad", dict(dy=P), 1), ("fm_block_norm_grad", dict(dpre=3 * P), 1),
    ("fm_block_norm_grad", dict(kind=3, dgate=2 * P), 1), ("fm_block_norm", dict(r=P + 8), 1), ("fm_block_norm", dict(h=P + 8), 1),
    ("fm_block_norm", dict(y=None, post=None, gate=None, kind=0), 1),
    ("fm_block_norm", dict(y=None, post=None, gate=None, kind=0, r=None, pre=None, h=None), 1),
    ("fm_block_norm", dict(T=0, x=None, y=None, gate=None, r=None, h=None), 0),
    ("fm_block_norm_grad", dict(dr=None, dh=None), 1), ("fm_block_norm_grad", dict(dh=None), 1),
    ("fm_block_norm_grad", dict(pre=None), 1), ("fm_block_norm_grad", dict(dpre=None), 1),
    ("fm_block_norm_grad", dict(dpost=None), 1), ("fm_block_norm_grad", dict(dgate=None), 1),
    ("fm_block_norm_grad", dict(dx=None), 1), ("fm_block_norm_grad", dict(dy=None), 1),
    ("fm_block_norm_grad", dict(dx=P + 8), 1), ("fm_block_norm_grad", dict(dpost=P + 2), 1),
    ("fm_block_norm_grad", dict(kind=3, dgate=P + 4), 1), ("fm_block_norm_grad", dict(scratch=None), 1),
    ("fm_block_norm_grad", dict(scratch=P + 64), 1), ("fm_block_norm_grad", dict(scratch_bytes=256), 1)])
def test_norm_arguments_refused(fn, change, status):
    base = NORM if fn == "fm_block_norm" else GRAD
    assert getattr(lib, fn)(*{**base, **change}.values()) == status
    assert (lib.fm_last_error().decode() != "") == (status != 0)


def test_sizes():
    # 2 layers x keys and values x 3 heads x 48 tokens x 72 float32 padded to 80
    assert lib.fm_kv_page_bytes(2, 3, 72, 48, 0) == 2 * 2 * 3 * 48 * 320
    assert lib.fm_kv_page_bytes(2, 3, 72, 48, 1) == 2 * 2 * 3 * 48 * 192
    assert lib.fm_kv_page_bytes(1, 1, 8, 16, 1) == 2 * 16 * 64
    for bad in ((0, 1, 8, 16, 1), (1, 1, 9, 16, 1), (1, 1, 8, 20, 1), (1, 1, 8, 16, 5)):
        assert lib.fm_kv_page_bytes(*bad) == 0
    desc = L.KvCacheDesc(*{**CACHE, "pages": None, "table": None, "length": None, "refs": None}.values())
    # count, two lists of 20 pages, two of 4 slots, a list of 20 pages, the table, each 256-byte aligned
    assert lib.fm_kv_scratch_bytes(C.byref(desc)) == 7 * 256
    assert lib.fm_attn_workspace_bytes(C.byref(desc), 8) > 0
    assert lib.fm_attn_workspace_bytes(C.byref(desc), 7) == 0
    desc.page = 20
    assert lib.fm_kv_scratch_bytes(C.byref(desc)) == 0 and lib.fm_attn_workspace_bytes(C.byref(desc), 8) == 0
    assert lib.fm_kv_scratch_bytes(None) == 0 and lib.fm_attn_workspace_bytes(None, 8) == 0
    assert lib.fm_block_norm_scratch_bytes(4, 64) == 4 * 2 * 64 * 4
    assert lib.fm_block_norm_scratch_bytes(0, 64) == 2 * 64 * 4
    for bad in ((-1, 64), (4, 0), (4, 60), (4, 16392)):
        assert lib.fm_block_norm_scratch_bytes(*bad) == 0


# ---------------------------------------------------------------- the binding

BF, I32 = torch.bfloat16, torch.int32


def _cache(**kw):
    return fm.KvCache(**{**dict(slots=4, max_tokens=100, pages=20, layers=2, heads=2, head_dim=64, page=32, device="cpu"),
                         **kw})


@pytest.mark.parametrize("change", [dict(slots=0), dict(max_tokens=0), dict(pages=0), dict(layers=0), dict(heads=0),
                                    dict(head_dim=12), dict(page=40)])
def test_caches_that_cannot_be(change):
    with pytest.raises(ValueError, match="invalid cache"):
        _cache(**change)


def test_the_memory_that_calls_read_stays_the_caches():
    cache = _cache()
    for name in ("pages", "table", "length", "refs"):
        with pytest.raises(AttributeError, match=f"{name} cannot be replaced"):
            setattr(cache, name, getattr(cache, name).clone())
        t = getattr(cache, name)
        t += 1
        assert getattr(cache._desc, name) == t.data_ptr()
    cache.length += 1
    assert cache.max_pages == 4 and cache.pages.shape == (20, 2 * 2 * 2 * 32 * 64) and cache.length.tolist() == [2] * 4


def test_tensors_refused():
    cache = _cache()
    q, k = torch.zeros(4, 8, 64, dtype=BF), torch.zeros(4, 2, 64, dtype=BF)
    four, on = torch.zeros(4, dtype=I32), torch.ones(4, dtype=torch.uint8)
    calls = [
        (lambda: fm.kv_resize(cache, four.long()), "delta must be"), (lambda: fm.kv_resize(cache, four[:3]), "delta must"),
        (lambda: fm.kv_resize(cache, four, out=four), "out must be"), (lambda: fm.kv_fork(cache, on), "parent must"),
        (lambda: fm.kv_compact(cache, out=four), "out must have"), (lambda: fm.kv_copy(cache, four, four[:2]), "dst must"),
        (lambda: fm.kv_write(cache, 0, k.float(), k), "k must be"), (lambda: fm.kv_write(cache, 0, k, k[:3]), "v must be"),
        (lambda: fm.kv_write(cache, 0, k, k[:3], offsets=torch.zeros(5, dtype=I32)), "as many rows"),
        (lambda: fm.kv_write(cache, 0, k, k, offsets=four), "offsets must"),
        (lambda: fm.kv_write(cache, 0, k.transpose(1, 2), k), "k must be"),
        (lambda: fm.kv_write(cache, 0, torch.zeros(4, 64, 2, dtype=BF).transpose(1, 2), k), "contiguous rows"),
        (lambda: fm.kv_write(cache, 0, k[:1].expand(4, 2, 64), k), "contiguous rows"),
        (lambda: fm.kv_write(cache, 0, k, k, active=four), "active must"),
        (lambda: fm.kv_read(cache, 0, offsets=torch.zeros(5, dtype=I32)), "offsets need T"),
        (lambda: fm.kv_read(cache, 0, T=3, out=(k, k)), "T=3 rows"),
        (lambda: fm.attn_decode(cache, 0, q.float()), "q must be"), (lambda: fm.attn_decode(cache, 0, q[:3]), "q must be"),
        (lambda: fm.attn_decode(cache, 0, torch.zeros(4, 7, 64, dtype=BF)), "not a multiple"),
        (lambda: fm.attn_decode(cache, 0, q, out=q), "out must not be q"),
        (lambda: fm.attn_decode(cache, 0, q, out=q[:, :4]), "out must have"),
        (lambda: fm.attn_decode(cache, 0, q, window=2 ** 32 + 5), "window=4294967301 does not fit"),
        (lambda: fm.attn_decode(cache, 2 ** 32, q), "layer=4294967296 does not fit"),
        (lambda: fm.kv_write(cache, -2 ** 40, k, k), "layer=-1099511627776 does not fit"),
        (lambda: fm.attn_decode(cache, 0, q, first=on), "first must"),
        (lambda: fm.attn_decode(cache, 0, q, active=four), "active must"),
        (lambda: fm.attn_decode(cache, 0, q, lse=torch.zeros(4, 7)), "lse must"),
        (lambda: fm.AttnWorkspace(cache, 7), "invalid workspace"),
        (lambda: fm.kv_resize(cache, four), "not on a GPU"), (lambda: fm.attn_decode(cache, 0, q), "not on a GPU")]
    for call, message in calls:
        with pytest.raises(ValueError, match=message):
            call()
    for call in (lambda: fm.attn_decode(cache, 0, None), lambda: fm.kv_write(cache, 0, k, [1])):
        with pytest.raises(TypeError, match="must be a torch.Tensor"):
            call()
    ws = fm.AttnWorkspace(cache, 8)
    ws.buf = ws.buf.to("meta")
    with pytest.raises(ValueError, match="workspace is on meta"):
        fm.attn_decode(cache, 0, q, workspace=ws)
    cache.flags = torch.zeros(2, dtype=I32)
    with pytest.raises(ValueError, match="flags"):
        fm.attn_decode(cache, 0, q)


def test_norm_tensors_refused():
    x, w, f = torch.zeros(4, 64, dtype=BF), torch.zeros(64, dtype=BF), torch.zeros(64)
    calls = [
        (lambda: fm.block_norm(x), "only the norm by pre"), (lambda: fm.block_norm(x, post=w, pre=w), "only the norm by pre"),
        (lambda: fm.block_norm(x, x.float(), pre=w), "y must"), (lambda: fm.block_norm(x, x, post=f), "post must"),
        (lambda: fm.block_norm(x, x, pre=w[:32]), "pre must"), (lambda: fm.block_norm(x, x, gate=w[:4]), "gate must have"),
        (lambda: fm.block_norm(x, x, gate=x.t()), "gate must have"), (lambda: fm.block_norm(x, x, gate=f), "gate must be"),
        (lambda: fm.block_norm(x.t(), x, pre=w), "x must be contiguous"),
        (lambda: fm.block_norm(x, x, out=(x, x)), "must be None without pre"),
        (lambda: fm.block_norm(x, pre=w, out=(x.clone(), x)), "must be None or x"),
        (lambda: fm.block_norm(x, x, pre=w, out=(x[:2], None)), "out\\[0\\]"),
        (lambda: fm.block_norm_grad(None, None, x, x), "dr or dh"),
        (lambda: fm.block_norm_grad(x, x, x, x), "exactly where pre"),
        (lambda: fm.block_norm_grad(x, None, x, x, pre=w), "exactly where pre"),
        (lambda: fm.block_norm_grad(x, x, x, post=w, pre=w), "need y"),
        (lambda: fm.block_norm_grad(x, None, x, x, post=w, accumulate=True), "accumulate needs out"),
        (lambda: fm.block_norm_grad(x, None, x, x, post=w, out=(x, x, w, None, None)), "dpost"),
        (lambda: fm.block_norm_grad(x, None, x, x, out=(x, x, f, None, None)), "must be None: its input"),
        (lambda: fm.block_norm_grad(x, None, x, x, gate=x[:, :1].contiguous(), out=(x, x, None, f, None)), "dgate"),
        (lambda: fm.BlockNormScratch(4, 60, "cpu"), "invalid scratch"),
        (lambda: fm.block_norm(x, x, pre=w), "not on a GPU"),
        (lambda: fm.block_norm_grad(x, None, x, x), "not on a GPU")]
    for call, message in calls:
        with pytest.raises(ValueError, match=message):
            call()
    with pytest.raises(TypeError, match="gate must be a torch.Tensor"):
        fm.block_norm(x, x, gate=0.5)
