"""The float64 definitions of the paged attention and the norms (oracle.layer)
against closed forms, differences and torch's autograd on the CPU."""
import numpy as np
import pytest
import torch

from oracle import layer as ref


def _pages(B=5, W=4, n=16, page=16, seed=0):
    rng = np.random.default_rng(seed)
    return ref.Pages(np.full((B, W), -1), np.zeros(B), np.zeros(n), rng.standard_normal((n, 3)), page)


def test_pages_are_shared_copied_and_released():
    p = _pages()
    granted, refused = p.resize([20, 0, 33, 0, 0])
    assert granted.tolist() == [1, 0, 1, 0, 0] and not refused
    assert p.held(0) == [0, 1] and p.held(2) == [2, 3, 4]
    p.fork([-1, 0, -1, 2, 0])
    assert p.held(1) == [0, 1] and p.held(4) == [0, 1] and p.refs[1] == 3
    p.check()
    p.resize([1, 1, 0, 0, 0])             # both get a copy of page 1, which slot 4 keeps
    assert p.held(0) == [0, 5] and p.held(1) == [0, 6] and p.held(4) == [0, 1] and p.refs[1] == 1
    assert (p.content[5] == p.content[1]).all() and (p.content[6] == p.content[1]).all()
    p.resize([-100, -5, 0, -2 ** 31, 0])
    assert p.held(0) == [] and p.length.tolist() == [0, 16, 33, 0, 20] and p.held(1) == [0]
    p.check()


def test_refusals_in_order():
    p = _pages(B=4, W=3, n=4)
    granted, refused = p.resize([16, 49, 64, 0])      # 1 page; past the table; past the table
    assert granted.tolist() == [1, 0, 0, 0] and refused
    granted, refused = p.resize([3, 48, 16, 1])
    assert granted.tolist() == [1, 0, 0, 0] and refused      # 2 used; 3 wanted of 2; later ones that need a page too
    granted, refused = p.resize([13, 32, 0, 0])
    assert granted.tolist() == [1, 1, 0, 0] and not refused  # slot 0's tokens fit its page
    p.check()


def test_forks_chain_and_cycle():
    p = _pages()
    p.resize([5, 17, 40, 0, 0])
    rows = [p.held(s) for s in range(5)]
    assert p.fork([1, 2, 0, 7, 3])
    assert [p.held(s) for s in range(5)] == [rows[1], rows[2], rows[0], rows[3], rows[3]]
    p.check()


def test_compaction_and_copies():
    p = _pages()
    p.resize([16, 48, 33, 16, 0])
    p.fork([-1, -1, -1, -1, 2])
    p.resize([-16, 0, 0, -16, 0])
    content = [p.content[p.held(s)].copy() for s in range(5)]
    n = p.compact()
    assert n == 6 and (p.refs[:6] > 0).all() and (p.refs[6:] == 0).all() and p.refs.sum() == 9
    for s in range(5):
        assert (p.content[p.held(s)] == content[s]).all()
    p.check()
    before = p.content.copy()
    assert p.copy([0, 1, 2, 9, 3, -1], [8, 9, 10, 11, 10, 12])   # 9 is a source too, 10 twice, no page -1
    assert (p.content[8] == before[0]).all() and (p.content[[9, 10, 12]] == before[[9, 10, 12]]).all()
    assert (p.content[11] == before[9]).all()


@pytest.mark.parametrize("size", [2, 4])
def test_places_are_a_permutation(size):
    c = dict(page=32, layers=2, heads=3, head_dim=40, size=size)
    at = [ref.place(c, l, kv, h, t, d) for l in range(2) for kv in (False, True) for h in range(3) for t in range(32)
          for d in range(40)]
    row = -(-40 * size // 64) * 64 // size
    assert len(set(at)) == len(at) and max(at) < 2 * 2 * 3 * 32 * row
    # keys: 16 bytes of one row; values: four tokens of a column
    n = 16 // size
    assert ref.place(c, 1, False, 2, 17, n + 1) - ref.place(c, 1, False, 2, 17, n) == 1
    assert ref.place(c, 1, True, 2, 18, 5) - ref.place(c, 1, True, 2, 17, 5) == 1


def test_attention_closed_forms():
    rng = np.random.default_rng(1)
    k, v, q = rng.standard_normal((9, 8)), rng.standard_normal((9, 8)), rng.standard_normal(8)
    out, bound, lse, _ = ref.attention(q * 0, k, v, 1.0, "f32")
    assert np.allclose(out, v.mean(axis=0)) and np.isclose(lse, np.log(9)) and (bound < 1e-3).all()
    out, *_ = ref.attention(q, k[:1], v[:1], 3.0, "f32")
    assert np.allclose(out, v[0])
    want = torch.nn.functional.scaled_dot_product_attention(*(torch.from_numpy(a)[None, None] for a in (q[None], k, v)),
                                                            scale=0.3)
    assert np.allclose(ref.attention(q, k, v, 0.3, "f32")[0], want.numpy()[0, 0, 0], rtol=1e-12)
    assert ref.attention(q, k[:0], v[:0], 1.0, "f32")[2] == -np.inf
    k[:, 0], q[0] = -np.inf, 1.0
    assert (ref.attention(q, k, v, 1.0, "f32")[0] == 0).all()


@pytest.mark.parametrize("kind", [None, "channel", "token", "each"])
@pytest.mark.parametrize("post,pre", [(True, True), (False, True), (True, False), (False, False)])
def test_norm_gradient_is_autograds_and_differences(kind, post, pre):
    rng = np.random.default_rng(3)
    T, d, scale, eps = 5, 8, 0.7, 1e-3
    shape = {None: None, "channel": (d,), "token": (T, 1), "each": (T, d)}[kind]
    leaves = dict(x=rng.standard_normal((T, d)), y=rng.standard_normal((T, d)),
                  post=rng.standard_normal(d) if post else None,
                  gate=None if shape is None else rng.standard_normal(shape), pre=rng.standard_normal(d) if pre else None)
    dr, dh = rng.standard_normal((T, d)), rng.standard_normal((T, d)) if pre else None

    def loss(a):
        r, h = ref.block_norm(a["x"], a["y"], a["post"], a["gate"], scale, a["pre"], eps)
        return (r.v * dr).sum() + (0.0 if h is None else (h.v * dh).sum())

    got = ref.block_norm_grad(dr, dh, leaves["x"], leaves["y"], leaves["post"], leaves["gate"], scale, leaves["pre"], eps,
                              kind)
    for name, g in zip(("x", "y", "post", "gate", "pre"), got):
        if leaves[name] is None:
            assert g is None
            continue
        g = g.v.reshape(leaves[name].shape)
        for at in np.ndindex(*leaves[name].shape):
            step = []
            for by in (1e-5, -1e-5):
                moved = {n: None if a is None else a.copy() for n, a in leaves.items()}
                moved[name][at] += by
                step.append(loss(moved))
            assert abs((step[0] - step[1]) / 2e-5 - g[at]) < 1e-6 * (1 + abs(g[at])), (name, at)
    t = {n: torch.from_numpy(a).requires_grad_() for n, a in leaves.items() if a is not None}

    def norm(z, w):
        return z / (z.square().mean(dim=1, keepdim=True) + eps).sqrt() * w

    r = t["x"] + scale * (norm(t["y"], t["post"]) if post else t["y"]) * t.get("gate", 1.0)
    total = (r * torch.from_numpy(dr)).sum()
    if pre:
        total = total + (norm(r, t["pre"]) * torch.from_numpy(dh)).sum()
    total.backward()
    for name, g in zip(("x", "y", "post", "gate", "pre"), got):
        if g is not None:
            assert np.allclose(g.v.reshape(t[name].shape), t[name].grad.numpy(), rtol=1e-10, atol=1e-12)


def test_bounds_cover_float32():
    """A float32 computation of the norms in NumPy stays within the carried bounds, and those are not wide."""
    rng = np.random.default_rng(4)
    T, d = 7, 200
    x, y = (rng.standard_normal((T, d)).astype(np.float32) for _ in range(2))
    w, g = (rng.standard_normal(d).astype(np.float32) for _ in range(2))
    r, h = ref.block_norm(x, y, w, g, 0.5, w, 1e-6)
    f = np.float32
    n = y * (f(1) / np.sqrt((y * y).mean(axis=1, keepdims=True) + f(1e-6))) * w
    r32 = x + f(0.5) * g * n
    h32 = r32 * (f(1) / np.sqrt((r32 * r32).mean(axis=1, keepdims=True) + f(1e-6))) * w
    assert (np.abs(r32 - r.v) <= r.e).all() and (np.abs(h32 - h.v) <= h.e).all()
    assert (h.e < 1e-3 * (np.abs(h.v) + 1)).all()
