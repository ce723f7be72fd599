"""Gradients of a block that is not normed, where its output holds infinities and
NaN: dy = scale gate dr' has no y in it."""
import numpy as np
import pytest
import torch

from oracle import layer as ref
from test_gpu_block_norm import close, inputs
from test_gpu_kv_pages import DT, _fm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", [(4, 64), (5, 264), (4, 2056), (4, 12296), (700, 72)])
@pytest.mark.parametrize("kind", [None, "channel", "token", "each"])
def test_outputs_of_a_block_that_are_not_finite(kind, T, d, dtype):
    fm = _fm()
    print(f"T={T} d={d} {dtype} gate={kind}", flush=True)
    rng = np.random.default_rng(d)
    t, n = inputs(rng, T, d, kind, False, False, dtype)
    for row, value in ((0, np.inf), (1, -np.inf), (T - 1, np.nan)):
        t["y"][row, d // 3] = float(value)
        n["y"][row, d // 3] = value
    t["y"][1] = n["y"][1] = float("inf")
    scale = float(np.float32(0.7))
    dx, dy, dpost, dgate, dpre = fm.block_norm_grad(t["dr"], None, t["x"], t["y"], gate=t["gate"], scale=0.7)
    with np.errstate(invalid="ignore"):
        want = ref.block_norm_grad(n["dr"], None, n["x"], n["y"], None, n["gate"], scale, None, 1e-6, kind)
    assert np.isfinite(want[0].v).all() and np.isfinite(want[1].v).all()
    close(dx, want[0], dtype, "dx")
    close(dy, want[1], dtype, "dy")
    assert dpost is None and dpre is None
    if kind is None:
        assert dgate is None
        return
    # the gate's gradient has y in it: what is finite is within its bound, what is not follows the formula
    got, exact = dgate.float().cpu().numpy().astype(np.float64).reshape(want[3].v.shape), want[3].v
    finite = np.isfinite(exact)
    assert (np.isnan(got) == np.isnan(exact)).all() and (got[np.isinf(exact)] == exact[np.isinf(exact)]).all()
    limit = (want[3].e + 2.0 ** (-8 if kind == "each" and dtype == "bf16" else -24) * (np.abs(exact) + want[3].e) * 1.01)[finite]
    assert (np.abs(got[finite] - exact[finite]) <= limit + 2.0 ** -126).all()


def test_the_same_rows_with_a_norm_follow_the_formula():
    """With post, a row that holds an infinity has a norm of infinity: NaN in all of its dy, and in no other row's."""
    fm = _fm()
    rng = np.random.default_rng(1)
    t, n = inputs(rng, 3, 264, "channel", True, False, "f32")
    t["y"][1, 7] = float("inf")
    _, dy, dpost, *_ = fm.block_norm_grad(t["dr"], None, t["x"], t["y"], post=t["post"], gate=t["gate"])
    assert torch.isnan(dy[1]).all() and torch.isfinite(dy[[0, 2]]).all()
    assert torch.isnan(dpost[7]) and torch.isfinite(dpost[torch.arange(264) != 7]).all()
