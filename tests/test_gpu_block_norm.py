"""The norms around a block and their gradient on the GPU, against oracle.layer
within the carried bounds and one rounding of each output's type, and against
differences of the kernel's own forward pass."""
import numpy as np
import pytest
import torch

from oracle import layer as ref
from oracle.operators import EPS32, rounding
from test_gpu_kv_pages import DT, _fm

pytestmark = pytest.mark.gpu


def drawn(rng, shape, dtype, scale=1.0):
    t = torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).cuda().to(DT[dtype])
    return t, t.float().cpu().numpy().astype(np.float64)


def close(got, want, dtype, what=""):
    if want is None:
        assert got is None, what
        return
    g = got.float().cpu().numpy().astype(np.float64).reshape(want.v.shape)
    limit = want.e + rounding(dtype) * (np.abs(want.v) + want.e) * (1 + 2.0 ** -8) + 2.0 ** -126
    bad = ~(np.abs(g - want.v) <= limit)
    assert not bad.any(), (what, np.argwhere(bad)[:4], g[bad][:4], want.v[bad][:4], limit[bad][:4])


def inputs(rng, T, d, kind, post, pre, dtype):
    """-> tensors and their float64 values by name."""
    shape = {None: None, "channel": (d,), "token": (T, 1), "each": (T, d)}[kind]
    t, n = {}, {}
    for name, s in (("x", (T, d)), ("y", (T, d)), ("post", (d,) if post else None), ("gate", shape),
                    ("pre", (d,) if pre else None), ("dr", (T, d)), ("dh", (T, d) if pre else None)):
        t[name], n[name] = (None, None) if s is None else drawn(rng, s, dtype)
    return t, n


SIZES = [(1, 8), (3, 64), (5, 512), (1, 520), (9, 1000), (2, 1024), (7, 1032), (4, 2048), (2, 2056), (3, 4096), (2, 4104),
         (1, 8192), (3, 8200), (2, 16384), (600, 136), (1100, 1032), (2100, 64),
         (9, 1536), (1100, 1536), (5, 1544), (3, 2600), (3, 6144), (2, 6152), (2, 9768), (3, 12288), (2, 12296),
         (3, 12296), (300, 4104), (300, 9768), (300, 12296)]


@pytest.mark.parametrize("T,d", [(4 * 65536 + 5, 8), (65536 + 3, 2056), (65536 + 2, 8200)])
def test_more_workgroups_than_a_row_of_the_grid(T, d):
    """Rows on either side of the border, against the same rows in a call of their own."""
    fm = _fm()
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn(T, d, generator=g, device="cuda", dtype=torch.bfloat16)
    w = torch.randn(d, generator=g, device="cuda", dtype=torch.bfloat16)
    y = x.flip(0)
    r, h = fm.block_norm(x, y, post=w, pre=w)
    for at in (0, 65530, T - 9):
        rows = slice(at, at + 9)
        for got, want in zip((r, h), fm.block_norm(x[rows], y[rows], post=w, pre=w)):
            assert torch.equal(got[rows], want)
    assert torch.isfinite(r).all() and torch.isfinite(h).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", SIZES)
def test_norm_and_gradient(T, d, dtype):
    fm = _fm()
    rng = np.random.default_rng(T + d)
    kinds = [None, "channel", "token", "each"]
    for i, (post, pre) in enumerate([(True, True), (False, True), (True, False), (False, False)]):
        for kind in (kinds if T * d < 10000 else [kinds[(i + T) % 4]]):
            print(f"T={T} d={d} {dtype} post={post} pre={pre} gate={kind}", flush=True)
            t, n = inputs(rng, T, d, kind, post, pre, dtype)
            common = dict(post=t["post"], gate=t["gate"], scale=0.7, pre=t["pre"], eps=1e-5)
            values = [n[k] for k in ("x", "y", "post", "gate")] + [float(np.float32(0.7)), n["pre"],
                                                                   float(np.float32(1e-5))]
            r, h = fm.block_norm(t["x"], t["y"], **common)
            want = ref.block_norm(*values)
            close(r, want[0], dtype, "r")
            close(h, want[1], dtype, "h")
            got = fm.block_norm_grad(t["dr"], t["dh"], t["x"], t["y"], **common)
            want = ref.block_norm_grad(n["dr"], n["dh"], *values, kind)
            for name, g, w in zip(("dx", "dy", "dpost", "dgate", "dpre"), got, want):
                whole = name in ("dx", "dy") or (name == "dgate" and kind == "each")
                assert w is None or g.dtype == (DT[dtype] if whole else torch.float32)
                close(g, w, dtype if whole else "f32", (name, kind, post, pre))
            again = fm.block_norm_grad(t["dr"], t["dh"], t["x"], t["y"], **common)
            assert all(a is None or torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_first_norm_and_missing_gradients(dtype):
    """The norm before a first block (no y); gradients of which one is missing."""
    fm = _fm()
    rng = np.random.default_rng(1)
    T, d = 5, 264
    t, n = inputs(rng, T, d, "channel", True, True, dtype)
    r, h = fm.block_norm(t["x"], pre=t["pre"])
    assert r is t["x"]
    eps = float(np.float32(1e-6))
    close(h, ref.block_norm(n["x"], None, None, None, 1.0, n["pre"], eps)[1], dtype)
    for dr in (None, "dr"):
        got = fm.block_norm_grad(t.get(dr), t["dh"], t["x"], pre=t["pre"])
        want = ref.block_norm_grad(n.get(dr), n["dh"], n["x"], None, None, None, 1.0, n["pre"], eps, None)
        close(got[0], want[0], dtype)
        close(got[4], want[4], "f32")
        assert got[1] is got[2] is got[3] is None
    got = fm.block_norm_grad(None, t["dh"], t["x"], t["y"], post=t["post"], gate=t["gate"], pre=t["pre"])
    want = ref.block_norm_grad(None, n["dh"], n["x"], n["y"], n["post"], n["gate"], 1.0, n["pre"], eps, "channel")
    for g, w, whole in zip(got, want, (True, True, False, False, False)):
        close(g, w, dtype if whole else "f32")


@pytest.mark.parametrize("T,d", [(4, 64), (3, 4096), (2, 16384)])
def test_outputs_over_inputs(T, d):
    """The overlaps that the documentation allows."""
    fm = _fm()
    rng = np.random.default_rng(d)
    t, _ = inputs(rng, T, d, "each", True, True, "bf16")
    common = dict(post=t["post"], gate=t["gate"], pre=t["pre"])
    r, h = fm.block_norm(t["x"], t["y"], **common)
    x, y = t["x"].clone(), t["y"].clone()
    fm.block_norm(x, y, out=(x, y), **common)
    assert torch.equal(x, r) and torch.equal(y, h)
    y = t["y"].clone()
    fm.block_norm(t["x"], y, out=(y, torch.empty_like(h)), **common)
    assert torch.equal(y, r)
    want = fm.block_norm_grad(t["dr"], t["dh"], t["x"], t["y"], **common)
    for over in ("y", "dh"):
        c = {k: None if v is None else v.clone() for k, v in t.items()}
        out = (c["dr"], c[over], torch.empty(d, device="cuda"), c["gate"], torch.empty(d, device="cuda"))
        got = fm.block_norm_grad(c["dr"], c["dh"], c["x"], c["y"], post=c["post"], gate=c["gate"], pre=c["pre"], out=out)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_accumulated_and_empty_gradients():
    fm = _fm()
    rng = np.random.default_rng(2)
    t, _ = inputs(rng, 37, 200, "channel", True, True, "bf16")
    common = dict(post=t["post"], gate=t["gate"], pre=t["pre"])
    want = fm.block_norm_grad(t["dr"], t["dh"], t["x"], t["y"], **common)
    base = [torch.full((200,), 3.0, device="cuda") for _ in range(3)]
    out = torch.empty_like(t["x"]), torch.empty_like(t["x"]), base[0].clone(), base[1].clone(), base[2].clone()
    scratch = fm.BlockNormScratch(100, 200)
    got = fm.block_norm_grad(t["dr"], t["dh"], t["x"], t["y"], accumulate=True, out=out, scratch=scratch, **common)
    for i in (2, 3, 4):
        # one more sum than the plain call's, of another order: 17 terms of their magnitudes
        size = want[i].abs() + 3
        assert ((got[i] - want[i] - 3).abs() <= 32 * EPS32 * size * 8).all()
    none = {k: v if k in ("post", "gate", "pre") else v[:0].contiguous() for k, v in t.items()}
    out = none["x"], none["y"].clone(), base[0].clone(), base[1].clone(), base[2].clone()
    fm.block_norm_grad(none["dr"], none["dh"], none["x"], none["y"], accumulate=True, out=out, **common)
    assert all((o == 3).all() for o in out[2:])
    got = fm.block_norm_grad(none["dr"], none["dh"], none["x"], none["y"], **common)
    assert all((o == 0).all() for o in got[2:]) and got[0].shape == (0, 200)
    r, h = fm.block_norm(none["x"], none["y"], **common)
    assert r.shape == h.shape == (0, 200)


def test_special_rows():
    """Zeros, infinities and NaN stay in their rows and follow the formula; rows of zeros have no direction."""
    fm = _fm()
    T, d = 5, 128
    x, y = torch.ones(T, d, device="cuda"), torch.ones(T, d, device="cuda")
    w = torch.ones(d, device="cuda")
    y[1], x[2], x[2, 3], y[3, 5] = 0, 0, float("inf"), float("nan")
    x[4], y[4] = 0, 0
    r, h = fm.block_norm(x, y, post=w, pre=w, eps=1e-6)
    assert (r[1] == 1).all() and (r[0] - 2).abs().max() < 1e-6
    assert torch.isinf(r[2, 3]) and torch.isnan(h[2, 3]) and (h[2, :3] == 0).all()
    assert torch.isnan(r[3]).all() and torch.isnan(h[3]).all()
    assert (r[4] == 0).all() and (h[4] == 0).all()
    got = fm.block_norm_grad(torch.ones_like(x), torch.ones_like(x), x, y, post=w, pre=w, eps=1e-6)
    assert torch.isfinite(got[0][[0, 1, 4]]).all() and torch.isfinite(got[1][[0, 1, 4]]).all()
    r, h = fm.block_norm(x, y, post=w, pre=w, eps=0.0)
    assert torch.isnan(r[4]).all() and torch.isnan(r[1]).all()       # 0 times 1 / 0


@pytest.mark.parametrize("kind", [None, "channel", "token", "each"])
def test_gradient_against_differences(kind):
    """Central differences of the float32 kernel along random directions.  Off by at most: the forward's rounding
    bounds over the step, the difference's own error (known from the float64 definition at the same step), and the
    gradient's bound along the direction."""
    fm = _fm()
    rng = np.random.default_rng(3)
    T, d, step = 6, 96, 2.0 ** -5
    t, n = inputs(rng, T, d, kind, True, True, "f32")
    scale, eps = 0.5, float(np.float32(1e-4))

    def kernel(a):
        f32 = {k: None if v is None else torch.from_numpy(v.astype(np.float32)).cuda() for k, v in a.items()}
        r, h = fm.block_norm(f32["x"], f32["y"], post=f32["post"], gate=f32["gate"], scale=scale, pre=f32["pre"], eps=eps)
        return (r.cpu().double().numpy() * n["dr"]).sum() + (h.cpu().double().numpy() * n["dh"]).sum()

    def exact(a):
        r, h = ref.block_norm(a["x"], a["y"], a["post"], a["gate"], scale, a["pre"], eps)
        # the outputs round once more
        err = sum((np.abs(g) * (o.e + EPS32 * (np.abs(o.v) + o.e))).sum() for g, o in ((n["dr"], r), (n["dh"], h)))
        return (r.v * n["dr"]).sum() + (h.v * n["dh"]).sum(), err

    got = fm.block_norm_grad(t["dr"], t["dh"], t["x"], t["y"], post=t["post"], gate=t["gate"], scale=scale, pre=t["pre"],
                             eps=eps)
    want = ref.block_norm_grad(n["dr"], n["dh"], n["x"], n["y"], n["post"], n["gate"], scale, n["pre"], eps, kind)
    for i, name in enumerate(("x", "y", "post", "gate", "pre")):
        if n[name] is None:
            continue
        for _ in range(3):
            u = rng.choice([-1.0, 1.0], n[name].shape)
            sides = []
            for sign in (1, -1):
                a = dict(n)
                a[name] = (n[name] + sign * step * u).astype(np.float32).astype(np.float64)
                sides.append((a[name], kernel(a), *exact(a)))
            move = sides[0][0] - sides[1][0]        # as it was rounded
            quotient, true = sides[0][1] - sides[1][1], sides[0][2] - sides[1][2]
            along = (got[i].cpu().double().numpy().reshape(move.shape) * move).sum()
            exactly = (want[i].v.reshape(move.shape) * move).sum()
            slack = sides[0][3] + sides[1][3] + abs(true - exactly) + \
                ((want[i].e + EPS32 * np.abs(want[i].v)).reshape(move.shape) * np.abs(move)).sum()
            assert abs(quotient - along) <= slack, (name, quotient, along, slack)
            assert slack < 0.05 * abs(exactly) + 0.05 * np.abs(want[i].v.reshape(move.shape) * move).sum(), (name, slack)
