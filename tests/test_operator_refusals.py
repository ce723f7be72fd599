"""What the model operators refuse, before anything reaches a GPU: the C ABI's
status codes for bad arguments, the sizes of scratch and workspace, and the
binding's checks of tensors (CPU only; no call enqueues anything)."""
import ctypes as C

import pytest
import torch

import paper_2502_05370_amd as fm
from paper_2502_05370_amd import _lib as L

P = 0x10000          # an aligned address; refused calls never follow it
lib = L.load()

LOOKUP = dict(table=P, V=10, d=8, dtype=1, tokens=P, T=4, scale=1.0, out=P, flags=None, stream=None)
POOL = dict(table=P, V=10, d=8, dtype=1, tokens=P, T=4, offsets=P, B=2, scale=1.0, out=P, flags=None, stream=None)
GRAD = dict(dout=P, dtype=1, tokens=P, T=4, V=10, d=8, scale=1.0, accumulate=0, dtable=P, grad_dtype=0, scratch=P,
            scratch_bytes=1 << 20, flags=None, stream=None)
ROUTE = dict(x=P, gate=P, dtype=1, T=4, d=64, E=8, K=2, renorm=0, active=None, probs=P, probs_dtype=0, stride=8, ids=P,
             weight=P, mask=None, stream=None)


@pytest.mark.parametrize("fn,base,change,status", [
    ("fm_embed_lookup", LOOKUP, dict(table=None), 1), ("fm_embed_lookup", LOOKUP, dict(tokens=None), 1),
    ("fm_embed_lookup", LOOKUP, dict(out=None), 1), ("fm_embed_lookup", LOOKUP, dict(V=0), 1),
    ("fm_embed_lookup", LOOKUP, dict(d=0), 1), ("fm_embed_lookup", LOOKUP, dict(d=16385), 1),
    ("fm_embed_lookup", LOOKUP, dict(T=-1), 1), ("fm_embed_lookup", LOOKUP, dict(T=(1 << 24) + 1), 1),
    ("fm_embed_lookup", LOOKUP, dict(dtype=2), 1), ("fm_embed_lookup", LOOKUP, dict(table=P + 1), 1),
    ("fm_embed_lookup", LOOKUP, dict(dtype=0, table=P + 2), 1), ("fm_embed_lookup", LOOKUP, dict(tokens=P + 2), 1),
    ("fm_embed_lookup", LOOKUP, dict(out=P + 1), 1), ("fm_embed_lookup", LOOKUP, dict(flags=P + 2), 1),
    ("fm_embed_lookup", LOOKUP, dict(T=0, table=None, tokens=None, out=None), 0),
    ("fm_embed_pool", POOL, dict(offsets=None), 1), ("fm_embed_pool", POOL, dict(out=None), 1),
    ("fm_embed_pool", POOL, dict(B=-1), 1), ("fm_embed_pool", POOL, dict(B=65537), 1),
    ("fm_embed_pool", POOL, dict(offsets=P + 1), 1), ("fm_embed_pool", POOL, dict(table=None), 1),
    ("fm_embed_pool", POOL, dict(B=0, offsets=None, out=None), 0),
    ("fm_embed_grad", GRAD, dict(dout=None), 1), ("fm_embed_grad", GRAD, dict(dtable=None), 1),
    ("fm_embed_grad", GRAD, dict(grad_dtype=9), 1), ("fm_embed_grad", GRAD, dict(dtype=-1), 1),
    ("fm_embed_grad", GRAD, dict(scratch=None), 1), ("fm_embed_grad", GRAD, dict(scratch=P + 16), 1),
    ("fm_embed_grad", GRAD, dict(scratch_bytes=1000), 1), ("fm_embed_grad", GRAD, dict(V=(1 << 24) + 1), 2),
    ("fm_embed_grad", GRAD, dict(dtable=P + 2), 1),
    ("fm_moe_route", ROUTE, dict(x=None), 1), ("fm_moe_route", ROUTE, dict(gate=None), 1),
    ("fm_moe_route", ROUTE, dict(probs=None), 1), ("fm_moe_route", ROUTE, dict(ids=None), 1),
    ("fm_moe_route", ROUTE, dict(weight=None), 1), ("fm_moe_route", ROUTE, dict(x=P + 8), 1),
    ("fm_moe_route", ROUTE, dict(E=0), 1), ("fm_moe_route", ROUTE, dict(E=65), 2), ("fm_moe_route", ROUTE, dict(K=0), 1),
    ("fm_moe_route", ROUTE, dict(K=9, E=16, stride=16), 1), ("fm_moe_route", ROUTE, dict(K=3, E=2), 1),
    ("fm_moe_route", ROUTE, dict(d=60), 2), ("fm_moe_route", ROUTE, dict(d=0), 1), ("fm_moe_route", ROUTE, dict(d=16392), 2),
    ("fm_moe_route", ROUTE, dict(stride=7), 1), ("fm_moe_route", ROUTE, dict(mask=P + 4), 1),
    ("fm_moe_route", ROUTE, dict(probs_dtype=3), 1), ("fm_moe_route", ROUTE, dict(T=0, x=None, ids=None), 0),
])
def test_refused(fn, base, change, status):
    assert getattr(lib, fn)(*{**base, **change}.values()) == status
    assert (lib.fm_last_error().decode() != "") == (status != 0)


CACHE = dict(E=8, n_slots=8, d=64, f=32, dtype=1, slots=P, slot_of=P)
EXPERTS = dict(x=P, ids=P, weight=P, T=4, K=2, residual=None, out=P, flags=None, workspace=P, workspace_bytes=1 << 24,
               stream=None)


@pytest.mark.parametrize("cache,call,status", [
    (dict(E=0), {}, 1), (dict(E=65), {}, 2), (dict(n_slots=0), {}, 1), (dict(d=0), {}, 1), (dict(d=60), {}, 2),
    (dict(f=33), {}, 2), (dict(f=65544), {}, 2), (dict(d=16384, f=65536), {}, 2), (dict(dtype=4), {}, 1),
    (dict(slots=None), {}, 1), (dict(slots=P + 8), {}, 1), (dict(slot_of=None), {}, 1), (dict(slot_of=P + 2), {}, 1),
    ({}, dict(x=None), 1), ({}, dict(ids=None), 1), ({}, dict(weight=None), 1), ({}, dict(out=None), 1),
    ({}, dict(K=0), 1), ({}, dict(K=9), 1), ({}, dict(T=-1), 1), ({}, dict(x=P + 2), 1), ({}, dict(residual=P + 8), 1),
    ({}, dict(workspace=None), 1), ({}, dict(workspace=P + 128), 1), ({}, dict(workspace_bytes=100), 1),
    ({}, dict(flags=P + 1), 1), ({}, dict(T=0, x=None, workspace=None), 0),
])
def test_experts_refused(cache, call, status):
    desc = L.ExpertCacheDesc(*{**CACHE, **cache}.values())
    assert lib.fm_moe_experts(C.byref(desc), *{**EXPERTS, **call}.values()) == status
    assert (lib.fm_last_error().decode() != "") == (status != 0)


def test_null_cache():
    assert lib.fm_moe_experts(None, *EXPERTS.values()) == L.FM_ERR_INVALID


def test_sizes():
    # n_freq, head and count of 100 rows, 10 positions, 1 frequent row, each 256-byte aligned
    assert fm.embed_grad_scratch_bytes(10, 100) == 256 + 2 * 512 + 256 + 256
    assert fm.embed_grad_scratch_bytes(0, 1) > 0
    assert fm.embed_grad_scratch_bytes(-1, 5) == fm.embed_grad_scratch_bytes(5, 0) == 0
    assert fm.embed_grad_scratch_bytes(5, (1 << 24) + 1) == 0
    ws = fm.moe_workspace_bytes
    assert ws(2048, 1408, "bf16", 1, 4) >= 4 * 1408 * 4
    assert ws(64, 32, "f32", 256, 8) == ws(64, 32, "f32", 5000, 8)    # launches of up to 256 tokens
    assert ws(64, 32, "bf16", 0, 8) == ws(64, 32, "bf16", 4, 9) == ws(60, 32, "bf16", 4, 2) == 0


def test_binding_checks(monkeypatch):
    bf = torch.bfloat16
    table, tok = torch.zeros(4, 8, dtype=bf), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="not on a GPU"):
        fm.embed_lookup(table, tok)
    with pytest.raises(ValueError, match="int32"):
        fm.embed_lookup(table, tok.long())
    with pytest.raises(ValueError, match="float32 or torch.bfloat16"):
        fm.embed_lookup(table.half(), tok)
    with pytest.raises(ValueError, match="contiguous"):
        fm.embed_lookup(torch.zeros(8, 4, dtype=bf).t(), tok)
    with pytest.raises(ValueError, match="out"):
        fm.embed_lookup(table, tok, out=torch.zeros(3, 8))
    with pytest.raises(TypeError):
        fm.embed_lookup([[1.0]], tok)
    with pytest.raises(ValueError, match="flags"):
        fm.embed_lookup(table, tok, flags=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError, match="offsets"):
        fm.embed_pool(table, tok, torch.zeros(2))
    with pytest.raises(ValueError, match="at least one"):
        fm.embed_pool(table, tok, tok[:0])
    with pytest.raises(ValueError, match="out"):
        fm.embed_pool(table, tok, tok, out=torch.zeros(2, 8))
    with pytest.raises(ValueError, match="tokens"):
        fm.embed_grad(table, tok, 5)
    with pytest.raises(ValueError, match="accumulate"):
        fm.embed_grad(table[:3], tok, 5, accumulate=True)
    with pytest.raises(ValueError, match="out"):
        fm.embed_grad(table[:3], tok, 5, out=torch.zeros(4, 8))
    with pytest.raises(ValueError, match="out"):
        fm.embed_grad(table[:3], tok, 5, grad_dtype=torch.float32, out=torch.zeros(5, 8, dtype=bf))
    with pytest.raises(ValueError, match="gate"):
        fm.moe_route(table, torch.zeros(5, 8), 2)
    with pytest.raises(ValueError, match="active"):
        fm.moe_route(table, table, 2, active=torch.zeros(4))
    maps = torch.zeros(4, 3, 4)
    ids, w = torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    with pytest.raises(ValueError, match="probs"):
        fm.moe_route(table, table, 2, out=(maps.transpose(1, 2)[:, 1], ids, w, None))
    with pytest.raises(ValueError, match="out\\[1\\]"):
        fm.moe_route(table, table, 2, out=(maps[:, 1], ids.long(), w, None))
    with pytest.raises(ValueError, match="not on a GPU"):
        fm.moe_route(table, table, 2, out=(maps[:, 1], ids, w, None))
    for kw in (dict(E=65), dict(d=12), dict(f=0), dict(slots=0)):
        with pytest.raises(ValueError, match="invalid expert cache"):
            fm.ExpertCache(**{**dict(slots=2, E=4, d=8, f=16, device="cpu"), **kw})
    cache = fm.ExpertCache(2, 4, 8, 16, device="cpu")
    with pytest.raises(ValueError, match="ids"):
        fm.moe_experts(cache, table, ids[:3], w)
    with pytest.raises(ValueError, match="weight"):
        fm.moe_experts(cache, table, ids, w[:, :1])
    with pytest.raises(ValueError, match="x must"):
        fm.moe_experts(cache, table.float(), ids, w)
    with pytest.raises(ValueError, match="residual"):
        fm.moe_experts(cache, table, ids, w, residual=table[:2])
    with pytest.raises(ValueError, match="workspace"):
        fm.MoeWorkspace(cache, 4, 9)
    with pytest.raises(ValueError, match="out of range"):
        cache.load(4, 0, *[None] * 3)
    with pytest.raises(ValueError, match="up must"):
        cache.load(0, 0, torch.zeros(16, 8, dtype=bf), torch.zeros(8, 16, dtype=bf), torch.zeros(8, 16, dtype=bf))
    with pytest.raises(ValueError, match="invalid scratch"):
        fm.EmbedGradScratch(5, 0, device="cpu")
