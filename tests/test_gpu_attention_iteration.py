"""The attention operators and norms together, as a server calls them: the example's
iterations with attention (examples/moe_iteration.py), token by token, against the
same layers in float64 over all tokens, with requests that come, branch, end and
come again while pages are shared, copied and moved."""
import numpy as np
import pytest
import torch

from test_gpu_moe_iteration import _example

pytestmark = pytest.mark.gpu


def _norm(x, w):
    return x * torch.rsqrt(x.square().mean(dim=1, keepdim=True) + 1e-6) * w


def _plain(model, tokens):
    """Hidden state of a request's last token: every layer over all of its tokens, in float64, rounded to bfloat16 where
    the model rounds."""
    c = model.c
    bf = lambda t: t.to(torch.bfloat16).double()
    wide = lambda t: t.cpu().double()
    x = bf(wide(model.table)[tokens] * c.d ** 0.5)
    T = len(tokens)
    seen = torch.ones(T, T, dtype=torch.bool).tril()
    if c.window:
        seen &= ~torch.ones(T, T, dtype=torch.bool).tril(-c.window)
    for layer in model.layers:
        rows = bf(bf(_norm(x, wide(layer.first))) @ wide(layer.qkv)).view(T, -1, c.head_dim).transpose(0, 1)
        q, k, v = rows[: c.heads], rows[c.heads: c.heads + c.kv_heads], rows[c.heads + c.kv_heads:]
        k, v = (t.repeat_interleave(c.heads // c.kv_heads, dim=0) for t in (k, v))
        p = torch.softmax((q @ k.transpose(1, 2) * c.head_dim ** -0.5).masked_fill(~seen, -torch.inf), dim=2)
        y = bf(bf((p @ v).transpose(0, 1).reshape(T, -1)) @ wide(layer.back))
        r = x + wide(layer.gain) * _norm(y, wide(layer.post))
        x, h = bf(r), bf(_norm(r, wide(layer.pre)))
        p = torch.softmax(h @ wide(layer.gate).t(), dim=1)      # every expert is taken: their order does not matter
        out = x.clone()
        for e in range(c.E):
            g, u, dn = (m.double() for m in layer.host[e])
            out += p[:, e: e + 1] * ((torch.nn.functional.silu(h @ g.t()) * (h @ u.t())) @ dn.t())
        x = bf(out)
    return x[-1]


def _check(model, x, requests):
    for s, tokens in enumerate(requests):
        if not tokens:
            assert (x[s] == 0).all()
            continue
        want = _plain(model, tokens)
        err = float((x[s].cpu().double() - want).abs().max() / want.abs().max())
        # Six roundings of half a unit (2^-8) per layer at most show in full: the norms, the projections, attention and
        # both streams; the layers' maps stretch them by little, since their inputs are normed and their weights are of
        # unit gain.
        assert err < 6 * model.c.L * 2.0 ** -8, (s, len(tokens), err)


@pytest.mark.parametrize("window", [0, 9])
def test_requests_come_branch_and_end(window):
    m = _example()
    c = m.Config(d=128, f=64, L=2, E=2, K=2, slots=2, heads=4, kv_heads=2, head_dim=32, batch=4, tokens=96, pages=14,
                 page=16, window=window)
    model = m.Model(c, seed=9)
    rng = np.random.default_rng(1)
    word = lambda n: [int(t) for t in rng.integers(0, c.V, n)]
    requests = [word(21), [], word(3), word(40)]
    x, *_ = model.iteration(requests)
    _check(model, x, requests)
    requests = [r + word(1) if r else r for r in requests]      # an iteration of one token each
    x, *_ = model.iteration(requests)
    _check(model, x, requests)
    model.branch([-1, 0, 0, -1])                                # two go on from request 0
    assert int((model.kv.refs > 1).sum()) == 2
    requests = [requests[0] + word(2), requests[0] + word(1), requests[0] + word(3), requests[3]]
    x, *_ = model.iteration([r if s < 3 else [] for s, r in enumerate(requests)])
    _check(model, x, [r if s < 3 else [] for s, r in enumerate(requests)])
    held = model.end([0, 3])
    assert held == int((model.kv.refs > 0).sum()) and (model.kv.refs[held:] == 0).all()
    requests = [word(30), requests[1] + word(5), requests[2] + word(1), word(2)]
    x, *_ = model.iteration(requests)
    _check(model, x, requests)
    assert model.kv.check() == 0 and model.kv.length.tolist() == [len(r) for r in requests]


def test_a_cache_that_is_full_is_said():
    m = _example()
    model = m.Model(m.Config(d=128, f=64, L=1, E=2, K=2, slots=2, heads=2, kv_heads=1, head_dim=32, batch=2, tokens=96,
                             pages=2, page=16), seed=9)
    with pytest.raises(AssertionError, match="no page left"):
        model.iteration([[1] * 20, [2] * 20])


def test_tuning_the_norms():
    """The example's descent runs, and its steps go along the gradients of the loss that it returns."""
    m = _example()
    model = m.Model(m.Config(L=1, heads=2), seed=2)
    layer, d = model.layers[0], model.c.d
    g = torch.Generator().manual_seed(3)
    x, y = ((torch.randn(9, d, generator=g)).to(torch.bfloat16).cuda() for _ in range(2))
    wanted = torch.randn(9, d, generator=g).cuda()
    before = [w.clone() for w in (layer.post, layer.gain, layer.pre)]
    rate = 2.0 ** -6
    first = model.tune_norms(layer, x, y, wanted, rate)

    def loss(weights):
        post, gain, pre = (w.double().requires_grad_() for w in weights)
        n = y.double() / (y.double().square().mean(dim=1, keepdim=True) + 1e-6).sqrt() * post
        r = x.double() + gain * n
        h = r / (r.square().mean(dim=1, keepdim=True) + 1e-6).sqrt() * pre
        off = h - wanted.double()
        (0.5 * off.square().sum()).backward()
        return 0.5 * float(off.detach().square().sum()), (post.grad, gain.grad, pre.grad), float(off.detach().abs().max())

    want, grads, largest = loss(before)
    # h and the distance to what is wanted are bfloat16: half a unit each, relative to values of up to `largest` + 4
    assert abs(first - want) <= 9 * d * (largest + 4) ** 2 * 2.0 ** -8
    for w, b, gr in zip((layer.post, layer.gain, layer.pre), before, grads):
        step = (b.double() - w.double()) / rate
        # the step's own rounding (half a unit of weights below 2), and two roundings of each of nine terms
        limit = 2.0 ** -7 / rate + 9 * 2 * 2.0 ** -8 * (largest + 4) * 8
        assert (step - gr).abs().max() < limit
