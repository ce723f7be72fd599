"""Pins of the model operators' float64 definitions (oracle.operators): closed
forms, adjointness of lookup and gradient, torch's float64 softmax, SiLU and
products.  CPU only."""
import numpy as np
import torch

from oracle import operators as ref


def test_lookup_and_gradient_are_adjoint():
    """<dout, lookup(table)> = <gradient(dout), table> for any table and dout."""
    rng = np.random.default_rng(0)
    table, dout = rng.standard_normal((7, 5)), rng.standard_normal((30, 5))
    tok = rng.integers(-2, 9, 30)          # some padding, some past the table
    grad, bound = ref.embed_grad(dout, tok, 7, 1.5)
    assert np.isclose((dout * ref.embed_lookup(table, tok, 1.5)).sum(), (grad * table).sum(), rtol=1e-13)
    base = rng.standard_normal((7, 5))
    assert np.allclose(ref.embed_grad(dout, tok, 7, 1.5, base=base)[0], grad + base)
    assert (bound >= 0).all() and (bound[np.setdiff1d(np.arange(7), tok)] == 0).all()
    assert (ref.embed_lookup(table, [-1, 7], 1.0) == 0).all()
    assert (ref.embed_lookup(table, [3], 2.0) == 2 * table[3]).all()


def test_pool_closed_forms():
    table = np.arange(12.0).reshape(4, 3)
    out, _ = ref.embed_pool(table, [0, 3, -1, 2, 4], [0, 3, 3, 5, 4], 2.0)
    assert np.allclose(out[0], table[0] + table[3])      # 2 * mean of two rows, padding not counted
    assert (out[1] == 0).all()                           # no tokens
    assert np.allclose(out[2], 2 * table[2])             # a token past the table is not counted
    assert (out[3] == 0).all()                           # an end before its start


def test_route_against_torch():
    rng = np.random.default_rng(1)
    x, g = rng.standard_normal((6, 9)), rng.standard_normal((11, 9))
    g[4] = g[2]                                          # an equal logit: lower index first
    p, ids, w, mask = ref.moe_route(x, g, 4, True, [1, 1, 0, 1, 1, 1])
    want = torch.softmax(torch.from_numpy(x @ g.T), dim=1).numpy()
    on = [0, 1, 3, 4, 5]
    assert np.allclose(p[on], want[on], rtol=1e-12) and np.allclose(w[on].sum(axis=1), 1)
    assert (p[2] == 0).all() and (ids[2] == -1).all() and (w[2] == 0).all() and mask[2] == 0
    for t in on:
        assert (np.diff(p[t, ids[t]]) <= 0).all() and mask[t] == sum(1 << int(j) for j in ids[t])
        for first, second in zip(ids[t], ids[t][1:]):
            assert p[t, first] > p[t, second] or first < second
    x[0, 0] = np.nan
    assert ref.moe_route(x, g, 3, False)[1][0].tolist() == [0, 1, 2]


def test_experts_against_torch():
    rng = np.random.default_rng(2)
    T, d, f, S = 5, 6, 4, 3
    x, slots = rng.standard_normal((T, d)), rng.standard_normal((S, 3 * d * f))
    ids = np.array([[0, 1], [1, 1], [3, 0], [-1, 2], [2, 0]])   # expert 1 twice, 3 held nowhere
    wt, slot_of, res = rng.random((T, 2)), [2, 0, 1, -1], rng.standard_normal((T, d))
    out, bound = ref.moe_experts(x, ids, wt, slots, slot_of, d, f, res)
    for t in range(T):
        want = torch.from_numpy(res[t])
        for k in range(2):
            if ids[t, k] < 0 or slot_of[ids[t, k]] < 0:
                continue
            b = torch.from_numpy(slots[slot_of[ids[t, k]]])
            v = torch.from_numpy(x[t])
            h = torch.nn.functional.silu(b[:d * f].view(f, d) @ v) * (b[d * f:2 * d * f].view(f, d) @ v)
            want = want + wt[t, k] * (b[2 * d * f:].view(d, f) @ h)
        assert np.allclose(out[t], want.numpy(), rtol=1e-12)
    assert (bound > 0).all() and (bound < 1e-3).all()
