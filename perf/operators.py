"""Performance cases of the model operators around the expert-map search.

Five operators feed the search and use what it prefetches:

* ``lookup``  embedding rows of a batch of tokens, scaled;
* ``pool``    each request's mean embedding, the query of a semantic search;
* ``grad``    the embedding table's gradient from the gradients of its rows;
* ``route``   a layer's gate: probabilities of all experts, the chosen ones;
* ``moe``     the chosen experts' feed-forward products for a few tokens, on
              the experts that an expert cache holds.

``own`` false computes them with elementary torch operations in float32,
rounded once at the end; ``own`` true calls the library.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
PAD_FRAC = 0.01      # padding (-1) among the tokens of longer batches
IDLE_FRAC = 0.05     # batch slots without a request, from 16 tokens on
ZIPF_SHIFT = 2.7     # token frequencies fall as 1 / (rank + shift)
X_GRID, W_GRID = 64.0, 1024.0   # router inputs and weights lie on grids of 1/64 and 1/1024


# ---------------------------------------------------------------- cases

def _case(kind, name=None, **sizes):
    c = {"kind": kind, **sizes}
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one decode iteration of three requests: launches and latency
        _case("lookup", "lookup_t3_d2048", T=3, V=32000, d=2048, dtype="bf16"),
        # prefill of a large batch of prompts, a large vocabulary
        _case("lookup", "lookup_t64k_d4096", T=65536, V=128000, d=4096, dtype="bf16"),
        # eight prompts of the mean length of the search's workloads become queries
        _case("pool", "pool_b8_len37_d4096", B=8, length=37, V=32000, d=4096, dtype="bf16"),
        # a thousand prompts of mixed lengths, some empty
        _case("pool", "pool_b1024_len300_d2048", B=1024, length=300, V=128000, d=2048, dtype="bf16"),
        # fine-tuning on a few short prompts, an odd number of tokens; float32 gradients
        _case("grad", "grad_t777_v32k_d2048", T=777, V=32000, d=2048, dtype="bf16", grad="f32"),
        # a training batch of 64 sequences of 1,024 tokens, a large vocabulary; bfloat16 gradients
        _case("grad", "grad_t64k_v128k_d2048", T=65536, V=128000, d=2048, dtype="bf16", grad="bf16"),
        # the gate of one decoded token, 60 experts
        _case("route", "route_t1_e60_d2048", T=1, d=2048, E=60, K=4, renorm=False, dtype="bf16", probs="f32"),
        # the gate over a prefill, 16 experts, weights normalised over the chosen
        _case("route", "route_t8k_e16_d4096", T=8192, d=4096, E=16, K=2, renorm=True, dtype="bf16", probs="bf16"),
        # one decoded token through 4 of 60 small experts
        _case("moe", "moe_t1_e60_d2048", T=1, d=2048, f=1408, E=60, focus=60, K=4, dtype="bf16"),
        # eight requests through 2 of 16 experts each
        _case("moe", "moe_t8_e16_d4096", T=8, d=4096, f=6400, E=16, focus=16, K=2, dtype="bf16"),
        # a batch of 64 requests, every one of 8 large experts in use
        _case("moe", "moe_t64_e8_d4096", T=64, d=4096, f=14336, E=8, focus=8, K=2, dtype="bf16"),
        # float32 experts, ragged sizes, requests that share a few favourite experts
        _case("moe", "moe_f32_t23_e24_d1000", T=23, d=1000, f=2744, E=24, focus=11, K=3, dtype="f32"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["lookup", "pool", "grad", "grad", "route", "route", "moe", "moe", "moe"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    es = BYTES[dtype]
    if kind in ("lookup", "pool", "grad"):
        # any width: even or odd, a multiple of the vector width or not
        d = _log(rng, 64, 8192)
        d = d if rng.random() < 0.3 else (d + 7) // 8 * 8
        V = _log(rng, 1000, max(1000, min(128000, 1_000_000_000 // (d * es))))
    if kind == "lookup":
        return _case(kind, T=_log(rng, 1, min(65536, 500_000_000 // (d * es))), V=V, d=d, dtype=dtype)
    if kind == "pool":
        length = _log(rng, 1, 600)
        return _case(kind, B=_log(rng, 1, max(1, min(1024, 300_000 // length, 1_200_000_000 // (length * d * es)))),
                     length=length, V=V, d=d, dtype=dtype)
    if kind == "grad":
        grad = rng.choice(["f32", dtype])
        V = min(V, 520_000_000 // (d * BYTES[grad]))
        return _case(kind, T=_log(rng, 1, min(65536, 260_000_000 // (d * es))), V=V, d=d, dtype=dtype, grad=grad)
    E = rng.choice([4, 8, 16, 24, 40, 60, 64])
    K = rng.randint(1, min(8, E))
    if kind == "route":
        d = 8 * _log(rng, 32, 1024)
        return _case(kind, T=_log(rng, 1, min(16384, 64_000_000 // (d * es))), d=d, E=E, K=K,
                     renorm=rng.random() < 0.5, dtype=dtype, probs=rng.choice(["f32", "bf16"]))
    d = 8 * _log(rng, 32, 512)
    f = 8 * _log(rng, 32, max(32, min(1792, 2_400_000_000 // (3 * 8 * d * E * es))))
    # bounded so that no draw has more products than the largest listed case
    T = _log(rng, 1, max(1, min(256, 7_500_000_000 // (K * d * f))))
    return _case(kind, T=T, d=d, f=f, E=E, focus=rng.randint(K, E), K=K, dtype=dtype)


# ---------------------------------------------------------------- inputs

def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + stream) & 0x7FFFFFFFFFFF)
    return g


def _randn(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device="cuda", dtype=dtype)


def _zipf(V):
    p = 1.0 / (np.arange(V) + ZIPF_SHIFT)
    return p / p.sum()


def _tokens(c, n, g):
    """Token ids with the falling frequencies of text, a few of them padding."""
    cdf = torch.from_numpy(np.cumsum(_zipf(c["V"]))).cuda()
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    rank = torch.searchsorted(cdf, u).clamp_max(c["V"] - 1)
    tok = torch.randperm(c["V"], generator=g, device="cuda")[rank].to(torch.int32)
    if n >= 16:
        tok[torch.rand(n, generator=g, device="cuda") < PAD_FRAC] = -1
    return tok


def _grid(x, grid):
    return (x * grid).round().clamp(-255, 255) / grid


def _inputs(c, seed, experts=None):
    """The tensors of a case.  ``experts`` receives the expert weights of a
    ``moe`` case ([slots][3 d f]: gate and up [f][d], then down [d][f])."""
    g, dt = _gen(seed, 1), DTYPES[c["dtype"]]
    if c["kind"] in ("lookup", "pool", "grad"):
        s = {}
        if c["kind"] == "pool":
            # lengths from none to twice the mean
            n = torch.randint(0, 2 * c["length"] + 1, (c["B"],), generator=g, device="cuda")
            n[0] = max(1, c["length"])
            s["offsets"] = torch.cat([n.new_zeros(1), n.cumsum(0)]).to(torch.int32)
            s["tokens"] = _tokens(c, int(s["offsets"][-1]), g)
        else:
            s["tokens"] = _tokens(c, c["T"], g)
        if c["kind"] == "grad":
            s["dout"] = _randn(g, c["T"], c["d"]).to(dt)
            s["scale"] = math.sqrt(c["d"])
        else:
            s["table"] = (0.02 * _randn(g, c["V"], c["d"], dtype=dt)).contiguous()
            s["scale"] = math.sqrt(c["d"])
        return s
    T, d, E, K = c["T"], c["d"], c["E"], c["K"]
    idle = torch.rand(T, generator=g, device="cuda") < (IDLE_FRAC if T >= 16 else 0.0)
    if c["kind"] == "route":
        # On these grids every partial sum of a logit is exact in float32, so
        # logits that are equal are equal in every order of summation.
        x = _grid(_randn(g, T, d), X_GRID).to(dt)
        gate = _grid(_randn(g, E, d) * (1.5 / math.sqrt(d)), W_GRID).to(dt)
        return {"x": x, "gate": gate, "active": (~idle).to(torch.uint8)}
    f = c["f"]
    if experts is None:
        experts = torch.empty(E, 3 * d * f, dtype=dt, device="cuda")
    for e in range(E):
        experts[e].normal_(generator=g)
        experts[e, : 2 * d * f] *= 1.0 / math.sqrt(d)
        experts[e, 2 * d * f:] *= 1.0 / math.sqrt(f)
    x, residual = _randn(g, T, d).to(dt), _randn(g, T, d).to(dt)
    # every token takes K of the experts that the batch favours
    favoured = torch.randperm(E, generator=g, device="cuda")[: c["focus"]]
    z, pick = _randn(g, T, c["focus"]).topk(K, dim=1)
    ids = favoured[pick].to(torch.int32)
    ids[idle] = -1
    weight = torch.softmax(z, dim=1).masked_fill(idle[:, None], 0.0)
    slot_of = torch.randperm(E, generator=g, device="cuda").to(torch.int32)
    return {"experts": experts, "x": x, "residual": residual, "ids": ids.contiguous(), "weight": weight.contiguous(),
            "slot_of": slot_of}


def prepare(case, seed):
    c = case
    if not own:
        return {"case": c, **_inputs(c, seed)}
    import paper_2502_05370_amd as fm
    cache = None
    if c["kind"] == "moe":
        # an expert cache that holds the layer, filled once
        cache = fm.ExpertCache(c["E"], c["E"], c["d"], c["f"], c["dtype"])
    s = {"case": c, "fm": fm, **_inputs(c, seed, None if cache is None else cache.weights)}

    def empty(dtype, *shape):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    dt = DTYPES[c["dtype"]]
    if c["kind"] == "lookup":
        s["out"] = empty(dt, c["T"], c["d"])
    elif c["kind"] == "pool":
        s["out"] = empty(torch.bfloat16, c["B"], c["d"])
    elif c["kind"] == "grad":
        s["out"] = empty(DTYPES[c["grad"]], c["V"], c["d"])
        s["scratch"] = fm.EmbedGradScratch(c["T"], c["V"])
    elif c["kind"] == "route":
        s["out"] = (empty(DTYPES[c["probs"]], c["T"], c["E"]), empty(torch.int32, c["T"], c["K"]),
                    empty(torch.float32, c["T"], c["K"]), empty(torch.int64, c["T"]))
    else:
        cache.slot_of.copy_(s["slot_of"])
        s["cache"], s["out"] = cache, empty(dt, c["T"], c["d"])
        s["ws"] = fm.MoeWorkspace(cache, c["T"], c["K"])
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    c = s["case"]
    if not own:
        return _PLAIN[c["kind"]](c, s)
    fm = s["fm"]
    if c["kind"] == "lookup":
        return fm.embed_lookup(s["table"], s["tokens"], s["scale"], out=s["out"])
    if c["kind"] == "pool":
        return fm.embed_pool(s["table"], s["tokens"], s["offsets"], s["scale"], out=s["out"])
    if c["kind"] == "grad":
        return fm.embed_grad(s["dout"], s["tokens"], c["V"], s["scale"], out=s["out"], scratch=s["scratch"])
    if c["kind"] == "route":
        return fm.moe_route(s["x"], s["gate"], c["K"], renorm=c["renorm"], active=s["active"], out=s["out"])
    return fm.moe_experts(s["cache"], s["x"], s["ids"], s["weight"], residual=s["residual"], out=s["out"],
                          workspace=s["ws"])


def _rows(s):
    """The float32 rows that the tokens select, zero for padding."""
    tok = s["tokens"].long()
    return s["table"][tok.clamp_min(0)].float() * (tok >= 0)[:, None]


def _plain_lookup(c, s):
    return (_rows(s) * s["scale"]).to(s["table"].dtype)


def _plain_pool(c, s):
    tok, end = s["tokens"], s["offsets"][1:].long()
    req = torch.bucketize(torch.arange(len(tok), device="cuda"), end, right=True)
    total = torch.zeros(c["B"], c["d"], device="cuda").index_add_(0, req, _rows(s))
    count = torch.zeros(c["B"], device="cuda").index_add_(0, req, (tok >= 0).float())
    return (total * (s["scale"] / count.clamp_min(1))[:, None]).to(torch.bfloat16)


def _plain_grad(c, s):
    tok = s["tokens"].long()
    dest = torch.where(tok >= 0, tok, c["V"])   # padding adds to a row past the table
    total = torch.zeros(c["V"] + 1, c["d"], device="cuda").index_add_(0, dest, s["dout"].float())
    return (total[: c["V"]] * s["scale"]).to(DTYPES[c["grad"]])


def _plain_route(c, s):
    on = s["active"] != 0
    logits = s["x"].float() @ s["gate"].float().t()
    p = torch.exp(logits - logits.amax(dim=1, keepdim=True))
    p = p / p.sum(dim=1, keepdim=True)
    ids = logits.sort(dim=1, descending=True, stable=True).indices[:, : c["K"]]
    weight = p.gather(1, ids)
    if c["renorm"]:
        weight = weight / weight.sum(dim=1, keepdim=True)
    mask = (torch.ones_like(ids) << ids).sum(dim=1)
    return ((p * on[:, None]).to(DTYPES[c["probs"]]), torch.where(on[:, None], ids, -1).to(torch.int32),
            weight * on[:, None], mask * on)


def _ffn(c, x, block):
    """One expert's products for the rows of x; block [..., 3 d f] float32."""
    d, f = c["d"], c["f"]
    gate, up = block[: d * f].view(f, d), block[d * f: 2 * d * f].view(f, d)
    h = x @ gate.t()
    h = h / (1 + torch.exp(-h)) * (x @ up.t())
    return h @ block[2 * d * f:].view(d, f).t()


def _plain_moe(c, s):
    x, ids, w, out = s["x"].float(), s["ids"].long(), s["weight"], s["residual"].float()
    if c["T"] * c["K"] < c["E"]:
        # fewer choices than experts: only the chosen experts are read
        slots = s["slot_of"].long()[ids.clamp_min(0)].view(-1)
        for p in range(c["T"] * c["K"]):
            t = p // c["K"]
            y = _ffn(c, x[t: t + 1], s["experts"].index_select(0, slots[p: p + 1])[0].float())
            out[t] += w.view(-1)[p] * y[0]
    else:
        for e in range(c["E"]):
            block = s["experts"].index_select(0, s["slot_of"][e: e + 1].long())[0].float()
            out = out + (w * (ids == e)).sum(dim=1, keepdim=True) * _ffn(c, x, block)
    return out.to(s["x"].dtype)


_PLAIN = {"lookup": _plain_lookup, "pool": _plain_pool, "grad": _plain_grad, "route": _plain_route, "moe": _plain_moe}


# ---------------------------------------------------------------- work, exact results

def _distinct_tokens(c, n):
    return float((1.0 - (1.0 - _zipf(c["V"])) ** n).sum())


def work(case):
    c = case
    es = BYTES[c["dtype"]]
    if c["kind"] == "lookup":
        return {"bytes": _distinct_tokens(c, c["T"]) * c["d"] * es + c["T"] * (c["d"] * es + 4.0),
                "flops": 1.0 * c["T"] * c["d"]}
    if c["kind"] == "pool":
        n = c["B"] * c["length"]
        return {"bytes": _distinct_tokens(c, n) * c["d"] * es + 4.0 * n + c["B"] * (2.0 * c["d"] + 4),
                "flops": 1.0 * n * c["d"]}
    if c["kind"] == "grad":
        # the gradients of the rows read, the dense gradient of the table written
        return {"bytes": c["T"] * (c["d"] * es + 4.0) + c["V"] * c["d"] * BYTES[c["grad"]],
                "flops": 2.0 * c["T"] * c["d"]}
    T, d, E, K = c["T"], c["d"], c["E"], c["K"]
    if c["kind"] == "route":
        return {"bytes": (T + E) * d * es + T * (E * BYTES[c["probs"]] + 8.0 * K + 9), "flops": 2.0 * T * d * E}
    used = c["focus"] * (1.0 - (1.0 - K / c["focus"]) ** T)   # experts that some token takes
    return {"bytes": used * 3.0 * d * c["f"] * es + 3.0 * T * d * es + 8.0 * T * K, "flops": 6.0 * T * K * d * c["f"]}


def exact(case, seed):
    c = case
    s = _inputs(c, seed)
    if c["kind"] == "lookup":
        out = torch.zeros(c["T"], c["d"], dtype=torch.float64, device="cuda")
        live = s["tokens"] >= 0
        out[live] = s["table"][s["tokens"][live].long()].double() * s["scale"]
        return out
    if c["kind"] == "pool":
        out = torch.zeros(c["B"], c["d"], dtype=torch.float64, device="cuda")
        ends = s["offsets"].tolist()
        for b in range(c["B"]):
            tok = s["tokens"][ends[b]: ends[b + 1]]
            tok = tok[tok >= 0].long()
            if len(tok):
                out[b] = s["table"][tok].double().mean(dim=0) * s["scale"]
        return out
    if c["kind"] == "grad":
        out = torch.zeros(c["V"], c["d"], dtype=torch.float64, device="cuda")
        live = s["tokens"] >= 0
        out.index_put_((s["tokens"][live].long(),), s["dout"][live].double(), accumulate=True)
        return out.mul_(s["scale"])
    if c["kind"] == "route":
        p = torch.softmax(s["x"].double() @ s["gate"].double().t(), dim=1) * (s["active"] != 0)[:, None]
        weight = p.topk(c["K"], dim=1).values
        if c["renorm"]:
            weight = weight / weight.sum(dim=1, keepdim=True).clamp_min(1e-300)
        return p, None, weight, None
    d, f = c["d"], c["f"]
    out = s["residual"].double()
    for e in range(c["E"]):
        t, k = torch.nonzero(s["ids"] == e, as_tuple=True)
        if len(t):
            block = s["experts"][int(s["slot_of"][e])].double()
            x = s["x"][t].double()
            h = torch.nn.functional.silu(x @ block[: d * f].view(f, d).t()) * (x @ block[d * f: 2 * d * f].view(f, d).t())
            out.index_add_(0, t, s["weight"][t, k].double()[:, None] * (h @ block[2 * d * f:].view(d, f).t()))
    return out
