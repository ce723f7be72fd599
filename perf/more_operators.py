"""Performance cases of the attention half of a serving iteration.

Three operators around the experts' products:

* ``attn``    attention of one new token per slot over a paged key-value cache;
* the cache's pages: ``write`` (keys and values of new tokens), ``fork`` (slots
  that go on from other slots and grow), ``compact`` (live pages to the front);
* ``norm``    a block's output normed, gated, scaled and added to the residual
  stream, and the norm before the next block; ``norm_grad`` its gradient.

``own`` false computes them with elementary torch operations in float32,
rounded once at the end; ``own`` true calls the library.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
LANE = {"f32": 4, "bf16": 8}     # values of 16 bytes
IDLE_FRAC = 0.05                 # batch slots without a request, from 16 slots on
EPS = 1e-6


# ---------------------------------------------------------------- cases

def _case(kind, name=None, **sizes):
    c = {"kind": kind, **sizes}
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # three requests of the mean prompt length: launches and latency
        _case("attn", "attn_b3_len37_d128", B=3, length=37, q_heads=16, heads=16, D=128, page=64, layers=1, window=0,
              dtype="bf16"),
        # a decode iteration of a full batch, contexts from a few tokens to 8,192
        _case("attn", "attn_b64_len4k_d128", B=64, length=4096, q_heads=32, heads=8, D=128, page=64, layers=1,
              window=0, dtype="bf16"),
        # one request with a very long context: work only along its length
        _case("attn", "attn_b1_len128k_d128", B=1, length=131072, q_heads=32, heads=8, D=128, page=256, layers=1,
              window=0, dtype="bf16"),
        # float32, heads of 80, five queries per key head, small pages, a sliding window
        _case("attn", "attn_f32_b23_len3k_d80", B=23, length=3001, q_heads=20, heads=4, D=80, page=16, layers=2,
              window=1000, dtype="f32"),
        # the new tokens of a decode iteration of eight requests
        _case("write", "write_b8_t1_d128", B=8, before=300, new=1, heads=8, D=128, page=64, layers=2, dtype="bf16"),
        # prompts of mixed lengths, 8,192 tokens, some behind an earlier part
        _case("write", "write_b16_t512_d128", B=16, before=37, new=512, heads=8, D=128, page=64, layers=2,
              dtype="bf16"),
        # eight requests that each go on in four ways (a search over continuations)
        _case("fork", "fork_m8_w4_len500", M=8, width=4, length=500, grow=5, heads=8, D=128, page=16, layers=24,
              dtype="bf16"),
        # a cache half of whose requests have ended gives its upper half back
        _case("compact", "compact_b32_n1024", B=32, length=256, spare=2.0, heads=8, D=128, page=16, layers=24,
              dtype="bf16"),
        # one decoded token: launches and latency
        _case("norm", "norm_t1_d2048", T=1, d=2048, gate="channel", post=True, pre=True, dtype="bf16"),
        # a prefill of 8,192 tokens, a gate per token
        _case("norm", "norm_t8k_d4096", T=8192, d=4096, gate="token", post=True, pre=True, dtype="bf16"),
        # fine-tuning on a few short prompts, odd sizes, float32
        _case("norm_grad", "norm_grad_f32_t777_d1000", T=777, d=1000, gate="each", post=True, pre=True, dtype="f32"),
        # a training batch of 8,192 tokens
        _case("norm_grad", "norm_grad_t8k_d4096", T=8192, d=4096, gate="channel", post=True, pre=True, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "write", "fork", "compact", "norm", "norm", "norm_grad", "norm_grad"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    es = BYTES[dtype]
    if kind in ("norm", "norm_grad"):
        d = 8 * _log(rng, 8, 2048)
        T = _log(rng, 1, min(32768, 66_000_000 // (d * es)))
        post, pre = rng.choice([(True, True), (True, True), (True, False), (False, True)])
        return _case(kind, T=T, d=d, gate=rng.choice(["none", "channel", "token", "each"]), post=post, pre=pre,
                     dtype=dtype)
    heads = rng.choice([1, 2, 3, 4, 8, 8, 16, 32])
    D = rng.choice([64, 128, 128, 256, 8 * rng.randint(2, 32)])
    page = rng.choice([16, 32, 48, 64, 128, 256])
    token = 2 * heads * _width(D, dtype) * es   # bytes of a token's keys and values
    if kind == "attn":
        group = rng.choice([1, 1, 2, 4, 5, 7, 8, 16, 24])
        if heads * group > 128:
            group = 128 // heads
        layers = rng.randint(1, 2)
        total = min(1_000_000, 500_000_000 // (token * layers))
        B = _log(rng, 1, max(1, min(256, total // page)))
        length = _log(rng, 1, max(1, min(131072, total // B)))
        window = rng.choice([0, 0, 0, _log(rng, 1, 4096)])
        return _case(kind, B=B, length=length, q_heads=heads * group, heads=heads, D=D, page=page, layers=layers,
                     window=window, dtype=dtype)
    if kind == "write":
        layers = rng.randint(1, 2)
        B = _log(rng, 1, 128)
        room = max(1, min(16384, 60_000_000 // token) // B)   # tokens of a slot, on average
        new = rng.choice([1, _log(rng, 1, room)])
        return _case(kind, B=B, before=_log(rng, 1, max(1, room)), new=new, heads=heads, D=D, page=page,
                     layers=layers, dtype=dtype)
    layers = _log(rng, 1, 24)
    block = page * token * layers                 # bytes of a page
    if block > 8_000_000:
        layers = max(1, layers * 8_000_000 // block)
        block = page * token * layers
    pages = max(8, min(20_000, 600_000_000 // block))   # pages of the pool
    if kind == "fork":
        width = rng.randint(1, 4)
        M = _log(rng, 1, max(1, min(64, pages // (4 * width + 2))))
        length = _log(rng, 1, max(1, (pages - 2 * M * width) * page // (3 * M)))
        return _case(kind, M=M, width=width, length=length, grow=rng.randint(1, page), heads=heads, D=D, page=page,
                     layers=layers, dtype=dtype)
    spare = rng.uniform(1.05, 3.0)
    B = _log(rng, 1, min(256, max(1, int(pages / spare) // 2)))
    length = _log(rng, 1, max(1, int(pages / spare / B - 1) * page))
    return _case(kind, B=B, length=length, spare=spare, heads=heads, D=D, page=page, layers=layers, dtype=dtype)


# ---------------------------------------------------------------- inputs

def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + stream) & 0x7FFFFFFFFFFF)
    return g


def _randn(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device="cuda", dtype=dtype)


def _width(D, dtype):
    """Elements of a head's row in a page: D rounded up to 64 bytes."""
    step = 4 * LANE[dtype]
    return (D + step - 1) // step * step


def _spread(n, mean):
    """n lengths around a mean, from about 1 to about twice the mean."""
    if n == 1:
        return [mean]
    return [max(1, int((i + 0.5) / n * 2 * mean)) for i in range(n)]


def _idle(n):
    return int(n * IDLE_FRAC) if n >= 16 else 0


def _shuffled(values, g):
    order = torch.randperm(len(values), generator=g, device="cuda")
    return torch.tensor(values, device="cuda", dtype=torch.int32)[order]


def _pages_of(tokens, page):
    return (tokens + page - 1) // page


def _tables(length, W, n_pages, page, g):
    """Pages for slots of these lengths, at random places of the pool."""
    table = torch.full((len(length), W), -1, dtype=torch.int32, device="cuda")
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    used = torch.arange(W, device="cuda")[None, :] < _pages_of(length, page)[:, None]
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)[: int(used.sum())]
    table[used] = order
    refs[order.long()] = 1
    return table, refs


def _page_elems(c):
    return c["layers"] * 2 * c["heads"] * c["page"] * _width(c["D"], c["dtype"])


def _inputs(c, seed):
    g, dt = _gen(seed, 1), DTYPES[c["dtype"]]
    kind = c["kind"]
    if kind in ("norm", "norm_grad"):
        T, d = c["T"], c["d"]
        s = {"residual": (2.0 * _randn(g, T, d)).to(dt), "y": _randn(g, T, d).to(dt), "scale": 0.7}
        s["post"] = (1 + 0.2 * _randn(g, d)).to(dt) if c["post"] else None
        s["pre"] = (1 + 0.2 * _randn(g, d)).to(dt) if c["pre"] else None
        shape = {"none": None, "channel": (d,), "token": (T, 1), "each": (T, d)}[c["gate"]]
        s["gate"] = None if shape is None else (0.5 + 0.3 * _randn(g, *shape)).to(dt)
        if kind == "norm_grad":
            s["dout"] = _randn(g, T, d).to(dt)
            s["dh"] = _randn(g, T, d).to(dt) if c["pre"] else None
        return s
    page, H, D = c["page"], c["heads"], c["D"]
    if kind == "attn":
        B = c["B"]
        length = _shuffled(_spread(B, c["length"]), g)
        W = _pages_of(max(_spread(B, c["length"])), page)
        n_pages = int(1.1 * sum(_pages_of(n, page) for n in _spread(B, c["length"]))) + 1
        table, refs = _tables(length, W, n_pages, page, g)
        active = torch.ones(B, dtype=torch.uint8, device="cuda")
        active[torch.randperm(B, generator=g, device="cuda")[: _idle(B)]] = 0
        total = sum(_spread(B, c["length"]))
        return {"length": length, "table": table, "refs": refs, "active": active, "scale": 1.5 / math.sqrt(D),
                "q": _randn(g, B, c["q_heads"], D).to(dt), "k": _randn(g, total, H, D, dtype=dt),
                "v": _randn(g, total, H, D, dtype=dt)}
    if kind == "write":
        B = c["B"]
        # some slots start empty; the others have tokens before the new ones
        before = _shuffled([n if i % 3 else 0 for i, n in enumerate(_spread(B, c["before"]))], g)
        sizes = [1] * B if c["new"] == 1 else _spread(B, c["new"])
        new = _shuffled(sizes, g)
        length = before + new
        W = _pages_of(2 * (c["before"] + c["new"]) + 1, page)
        n_pages = int(1.1 * int(_pages_of(length, page).sum())) + 1
        table, refs = _tables(length, W, n_pages, page, g)
        # keys and values side by side, as one projection writes them
        kv = _randn(g, sum(sizes), 2 * H, D, dtype=dt)
        s = {"length": length, "table": table, "refs": refs, "k": kv[:, :H], "v": kv[:, H:],
             "offsets": None, "pages": torch.zeros(n_pages, _page_elems(c), dtype=dt, device="cuda")}
        if c["new"] != 1:
            s["offsets"] = torch.cat([new.new_zeros(1), new.cumsum(0).to(torch.int32)])
        return s
    if kind == "fork":
        M, width = c["M"], c["width"]
        spread = _spread(M, c["length"])
        length = torch.cat([_shuffled(spread, g), torch.zeros(M * width, dtype=torch.int32, device="cuda")])
        W = _pages_of(max(spread) + c["grow"], page)
        taken = sum(_pages_of(n, page) for n in spread)
        n_pages = int(1.2 * taken) + 2 * M * width + 2
        table, refs = _tables(length, W, n_pages, page, g)
        mains = torch.arange(M, dtype=torch.int32, device="cuda")
        none = torch.full((M,), -1, dtype=torch.int32, device="cuda")
        return {"length": length, "table": table, "refs": refs,
                "pages": _randn(g, n_pages, _page_elems(c), dtype=dt),
                "parent": torch.cat([none, mains.repeat_interleave(width)]),
                "delta": torch.cat([none * 0, torch.full((M * width,), c["grow"], dtype=torch.int32, device="cuda")])}
    B = c["B"]
    spread = _spread(B, c["length"])
    length = _shuffled(spread, g)
    n_pages = int(c["spare"] * sum(_pages_of(n, page) for n in spread)) + 1
    table, refs = _tables(length, _pages_of(max(spread), page), n_pages, page, g)
    return {"length": length, "table": table, "refs": refs, "pages": _randn(g, n_pages, _page_elems(c), dtype=dt)}


def _tokens(s):
    """Slot and position of every token of all slots, in order."""
    n = s["length"].long()
    slot = torch.repeat_interleave(torch.arange(len(n), device="cuda"), n)
    return slot, torch.arange(len(slot), device="cuda") - (n.cumsum(0) - n)[slot]


def prepare(case, seed):
    c = case
    s = {"case": c, **_inputs(c, seed)}
    if not own:
        if c["kind"] == "attn":
            # the keys and values in pages of [page tokens][head][D]
            slot, pos = _tokens(s)
            at = s["table"][slot, pos // c["page"]].long(), pos % c["page"]
            for name in ("k", "v"):
                rows = s.pop(name)
                s[name + "_pages"] = rows.new_zeros(len(s["refs"]), c["page"], c["heads"], c["D"])
                s[name + "_pages"][at] = rows
        if c["kind"] == "compact":
            s["now"] = {n: s[n].clone() for n in ("table", "refs")}
        return s
    import paper_2502_05370_amd as fm
    s["fm"] = fm
    if c["kind"] in ("norm", "norm_grad"):
        T, d = c["T"], c["d"]

        def like():
            return torch.empty_like(s["residual"])

        if c["kind"] == "norm":
            s["out"] = (like(), like() if c["pre"] else None)
        else:
            def vector(on):
                return torch.empty(d, device="cuda") if on else None
            dgate = {"none": None, "channel": vector(True), "token": torch.empty(T, 1, device="cuda"),
                     "each": like()}[c["gate"]]
            s["out"] = (like(), like(), vector(c["post"]), dgate, vector(c["pre"]))
            s["scratch"] = fm.BlockNormScratch(T, d)
        return s
    B, W = s["table"].shape
    cache = fm.KvCache(B, W * c["page"], len(s["refs"]), c["layers"], c["heads"], c["D"], c["dtype"], page=c["page"])
    for name in ("table", "length", "refs"):
        getattr(cache, name).copy_(s[name])
    s["cache"] = cache
    if c["kind"] == "attn":
        offsets = torch.cat([s["length"].new_zeros(1), s["length"].cumsum(0).to(torch.int32)])
        fm.kv_write(cache, c["layers"] - 1, s.pop("k"), s.pop("v"), offsets=offsets)
        s["out"] = torch.empty_like(s["q"])
        s["ws"] = fm.AttnWorkspace(cache, c["q_heads"])
    else:
        cache.pages.copy_(s.pop("pages"))
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    c = s["case"]
    if not own:
        return _PLAIN[c["kind"]](c, s)
    fm = s["fm"]
    if c["kind"] == "norm":
        return fm.block_norm(s["residual"], s["y"], post=s["post"], gate=s["gate"], scale=s["scale"], pre=s["pre"],
                             eps=EPS, out=s["out"])
    if c["kind"] == "norm_grad":
        return fm.block_norm_grad(s["dout"], s["dh"], s["residual"], s["y"], post=s["post"], gate=s["gate"],
                                  scale=s["scale"], pre=s["pre"], eps=EPS, out=s["out"], scratch=s["scratch"])
    cache = s["cache"]
    if c["kind"] == "attn":
        return fm.attn_decode(cache, c["layers"] - 1, s["q"], s["scale"], window=c["window"], active=s["active"],
                              out=s["out"], workspace=s["ws"])
    if c["kind"] == "write":
        fm.kv_write(cache, c["layers"] - 1, s["k"], s["v"], offsets=s["offsets"])
        return cache.pages
    if c["kind"] == "fork":
        fm.kv_fork(cache, s["parent"])
        granted = fm.kv_resize(cache, s["delta"])
        return granted, cache.table, cache.length, cache.refs, cache.pages
    # the tables of a fragmented cache, taken up again
    cache.table.copy_(s["table"])
    cache.refs.copy_(s["refs"])
    live = fm.kv_compact(cache)
    return live, cache.table, cache.refs, cache.pages


def _plain_attn(c, s):
    B, H, D = c["B"], c["heads"], c["D"]
    longest = max(_spread(B, c["length"]))
    q = s["q"].float().view(B, H, c["q_heads"] // H, D)
    pages = s["table"].long().clamp_min(0)

    def rows(pool):
        return pool[pages].view(B, -1, H, D)[:, :longest].float().transpose(1, 2)

    score = (q * s["scale"]) @ rows(s["k_pages"]).transpose(2, 3)
    pos, end = torch.arange(longest, device="cuda"), s["length"][:, None]
    seen = (pos < end) & (s["active"][:, None] != 0)
    if c["window"]:
        seen &= pos >= end - c["window"]
    score = score.masked_fill(~seen[:, None, None, :], -math.inf)
    p = torch.exp(score - score.amax(dim=3, keepdim=True)).nan_to_num_(0.0)
    out = (p @ rows(s["v_pages"])) / p.sum(dim=3, keepdim=True).clamp_min(1e-30)
    return out.view(B, c["q_heads"], D).to(s["q"].dtype)


def _plain_write(c, s):
    """Pages as the cache lays them out: per layer keys, then values; per head
    blocks of 16 tokens; of a block, pieces of 64 bytes of all 16 rows, each
    with 16 bytes of a row (keys) or of four tokens' columns (values) a lane."""
    page, H, layer, n = c["page"], c["heads"], c["layers"] - 1, LANE[c["dtype"]]
    if s["offsets"] is None:
        slot = torch.arange(c["B"], device="cuda")
        pos = s["length"].long() - 1
    else:
        new = s["offsets"].diff().long()
        slot = torch.repeat_interleave(torch.arange(c["B"], device="cuda"), new, output_size=len(s["k"]))
        pos = s["length"].long()[slot] - s["offsets"][1:].long()[slot] + torch.arange(len(slot), device="cuda")
    at = s["table"][slot, pos // page].long()
    block, row = pos % page // 16, pos % 16
    width = _width(c["D"], c["dtype"])
    pieces = width // (4 * n)
    k, v = (torch.nn.functional.pad(t, (0, width - c["D"])) for t in (s["k"], s["v"]))
    shape = len(s["refs"]), c["layers"], 2, H, page // 16, pieces
    to_k = s["pages"].view(*shape, 4, 16, n)
    to_k[at, layer, 0, :, block, :, :, row] = k.reshape(-1, H, pieces, 4, n)
    to_v = s["pages"].view(*shape, 4, 16, n // 4, 4)
    to_v[at, layer, 1, :, block, :, row // 4, :, :, row % 4] = v.reshape(-1, H, pieces, n // 4, 16).transpose(3, 4)
    return s["pages"]


def _add_refs(refs, table, used, by):
    """refs changed by ``by`` for every page of the used entries of the table."""
    more = torch.zeros(len(refs) + 1, dtype=torch.int32, device="cuda")
    dest = torch.where(used, table, len(refs)).long().view(-1)
    more.index_add_(0, dest, torch.full_like(dest, by, dtype=torch.int32))
    refs += more[:-1]


def _plain_fork(c, s):
    table, length, refs, pages, page = s["table"], s["length"], s["refs"], s["pages"], c["page"]
    B, W = table.shape
    col, slots = torch.arange(W, device="cuda")[None, :], torch.arange(B, device="cuda")
    # fork
    moved = (s["parent"] >= 0) & (s["parent"] != slots)
    parent = torch.where(moved, s["parent"].long(), slots)
    n = _pages_of(length, page)
    _add_refs(refs, table, (col < n[:, None]) & moved[:, None], -1)
    table.copy_(table[parent])
    length.copy_(length[parent])
    n = _pages_of(length, page)
    _add_refs(refs, table, (col < n[:, None]) & moved[:, None], 1)
    # grow: shared last pages are copied, then new ones follow
    end = length + s["delta"]
    last = (n - 1).clamp_min(0).long()
    tail = table[slots, last].clamp_min(0).long()
    copied = (s["delta"] > 0) & (length % page != 0) & (refs[tail] > 1)
    fresh = _pages_of(end, page) - n
    need = torch.where(s["delta"] > 0, fresh + copied, 0)
    upto = need.cumsum(0)
    free = torch.argsort(refs != 0, stable=True).to(torch.int32)
    granted = (s["delta"] > 0) & ((need == 0) | (upto <= (refs == 0).sum()))
    copied &= granted
    start = n - copied.to(n.dtype)       # first entry that takes a new page
    takes = (col >= start[:, None]) & (col < _pages_of(end, page)[:, None]) & granted[:, None]
    rank = (upto - need - start)[:, None] + col
    _add_refs(refs, tail[:, None], copied[:, None], -1)
    table.copy_(torch.where(takes, free[rank.clamp(0, len(free) - 1)], table))
    _add_refs(refs, table, takes, 1)
    length.copy_(torch.where(granted, end, length))
    who = copied.nonzero().squeeze(1)
    pages[table[who, last[who]].long()] = pages[tail[who]]
    return granted.to(torch.uint8), table, length, refs, pages


def _plain_compact(c, s):
    table, refs = s["now"]["table"], s["now"]["refs"]
    table.copy_(s["table"])
    refs.copy_(s["refs"])
    live = refs > 0
    count = live.sum(dtype=torch.int32)
    ids = torch.arange(len(refs), dtype=torch.int32, device="cuda")
    src = (live & (ids >= count)).nonzero().squeeze(1)
    dst = (~live & (ids < count)).nonzero().squeeze(1)
    s["pages"][dst] = s["pages"][src]
    name = ids.clone()
    name[src] = dst.to(torch.int32)
    refs[dst] = refs[src]
    refs[src] = 0
    table.copy_(torch.where(table >= 0, name[table.long().clamp_min(0)], -1))
    return count.view(1), table, refs, s["pages"]


def _rms(x):
    return torch.rsqrt((x * x).mean(dim=1, keepdim=True) + EPS)


def _plain_norm(c, s):
    n = s["y"].float()
    if c["post"]:
        n = n * _rms(n) * s["post"].float()
    if s["gate"] is not None:
        n = n * s["gate"].float()
    r = s["residual"].float() + s["scale"] * n
    dt = s["y"].dtype
    return r.to(dt), (r * _rms(r) * s["pre"].float()).to(dt) if c["pre"] else None


def _plain_norm_grad(c, s):
    y, dt = s["y"].float(), s["y"].dtype
    inv = _rms(y) if c["post"] else None
    hat = y * inv if c["post"] else y
    n = hat * s["post"].float() if c["post"] else hat
    gate = None if s["gate"] is None else s["gate"].float()
    r = s["residual"].float() + s["scale"] * (n if gate is None else n * gate)
    dr, dpre, dpost, dgate = s["dout"].float(), None, None, None
    if c["pre"]:
        dh, inv_r = s["dh"].float(), _rms(r)
        r_hat = r * inv_r
        dpre = (dh * r_hat).sum(dim=0)
        dz = dh * s["pre"].float()
        dr = dr + inv_r * (dz - r_hat * (dz * r_hat).mean(dim=1, keepdim=True))
    dn = s["scale"] * dr
    if gate is not None:
        dgate = dn * n
        dgate = {"channel": lambda t: t.sum(dim=0), "token": lambda t: t.sum(dim=1, keepdim=True),
                 "each": lambda t: t.to(dt)}[c["gate"]](dgate)
        dn = dn * gate
    dy = dn
    if c["post"]:
        dpost = (dn * hat).sum(dim=0)
        dz = dn * s["post"].float()
        dy = inv * (dz - hat * (dz * hat).mean(dim=1, keepdim=True))
    return dr.to(dt), dy.to(dt), dpost, dgate, dpre


_PLAIN = {"attn": _plain_attn, "write": _plain_write, "fork": _plain_fork, "compact": _plain_compact,
          "norm": _plain_norm, "norm_grad": _plain_norm_grad}


# ---------------------------------------------------------------- work, exact results

def work(case):
    c = case
    es = BYTES[c["dtype"]]
    if c["kind"] in ("norm", "norm_grad"):
        T, d = c["T"], c["d"]
        gate = {"none": 0, "channel": d, "token": T, "each": T * d}[c["gate"]]
        vectors = (c["post"] + c["pre"]) * d
        if c["kind"] == "norm":
            return {"bytes": es * ((3.0 + c["pre"]) * T * d + gate + vectors), "flops": 9.0 * T * d}
        # dout, dh, residual and y read, two gradients of their size written
        return {"bytes": es * ((5.0 + c["pre"]) * T * d + gate + vectors) + 4.0 * vectors
                + gate * (es if c["gate"] == "each" else 4.0), "flops": 25.0 * T * d}
    H, D, page = c["heads"], c["D"], c["page"]
    token = 2.0 * H * D * es
    block = float(_page_elems(c) * es)
    if c["kind"] == "attn":
        spread = _spread(c["B"], c["length"])
        seen = [min(n, c["window"]) if c["window"] else n for n in spread]
        tokens = sum(seen) * (1.0 - _idle(c["B"]) / c["B"])
        rows = c["B"] * c["q_heads"] * D
        return {"bytes": tokens * token + 2.0 * rows * es + 4.0 * sum(_pages_of(n, page) for n in seen),
                "flops": 4.0 * tokens * c["q_heads"] * D}
    if c["kind"] == "write":
        n = c["B"] if c["new"] == 1 else sum(_spread(c["B"], c["new"]))
        return {"bytes": 2.0 * n * token, "flops": 0.0}
    if c["kind"] == "fork":
        spread = _spread(c["M"], c["length"])
        copied = c["width"] * sum(n % page != 0 for n in spread)
        entries = c["width"] * sum(_pages_of(n + c["grow"], page) for n in spread)
        return {"bytes": 2.0 * copied * block + 16.0 * entries, "flops": 0.0}
    live = sum(_pages_of(n, page) for n in _spread(c["B"], c["length"]))
    n_pages = int(c["spare"] * live) + 1
    moved = live * (1.0 - live / n_pages)     # live pages of the upper part, on average
    return {"bytes": 2.0 * moved * block + 8.0 * (n_pages + live), "flops": 0.0}


def exact(case, seed):
    c = case
    if c["kind"] not in ("attn", "norm", "norm_grad"):
        return None   # copies
    s = _inputs(c, seed)
    if c["kind"] == "attn":
        H = c["heads"]
        out = torch.zeros(c["B"], c["q_heads"], c["D"], dtype=torch.float64, device="cuda")
        ends = [0] + s["length"].cumsum(0).tolist()
        for b in range(c["B"]):
            if not int(s["active"][b]):
                continue
            lo = max(ends[b], ends[b + 1] - c["window"]) if c["window"] else ends[b]
            for h in range(H):
                heads = slice(h * (c["q_heads"] // H), (h + 1) * (c["q_heads"] // H))
                k, v = s["k"][lo: ends[b + 1], h].double(), s["v"][lo: ends[b + 1], h].double()
                out[b, heads] = torch.softmax(s["q"][b, heads].double() @ k.t() * s["scale"], dim=1) @ v
        return out
    leaves = {n: s[n].double().requires_grad_() for n in ("residual", "y", "post", "gate", "pre") if s[n] is not None}

    def norm(x, w):
        return x / (x.square().mean(dim=1, keepdim=True) + EPS).sqrt() * w

    n = norm(leaves["y"], leaves["post"]) if c["post"] else leaves["y"]
    r = leaves["residual"] + s["scale"] * n * leaves.get("gate", 1.0)
    h = norm(r, leaves["pre"]) if c["pre"] else None
    if c["kind"] == "norm":
        return r.detach(), None if h is None else h.detach()
    loss = (r * s["dout"].double()).sum()
    if h is not None:
        loss = loss + (h * s["dh"].double()).sum()
    loss.backward()
    return tuple(leaves[n].grad if n in leaves else None for n in ("residual", "y", "post", "gate", "pre"))
