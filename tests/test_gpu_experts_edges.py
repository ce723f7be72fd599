"""The experts' products of bf16 models at the ends of the number range, in every
class of batch lengths, against the float64 definition of oracle.operators."""
import numpy as np
import pytest
import torch

from oracle import operators as ref
from test_gpu_operators import _fm, _layer, close, dev, drawn

pytestmark = pytest.mark.gpu

LENGTHS = [1, 9, 40, 100, 200]


def _single(T, d, f, gate, up, down, weight, x=1.0):
    """T equal tokens on one expert with one path: input 0, place 0, then output 0
    by `down` and output 1 by its half.  -> (kernel's output, oracle's output, its bound)"""
    fm = _fm()
    cache = fm.ExpertCache(1, 1, d, f, "bf16")
    w = np.zeros((1, 3 * d * f), np.float32)
    w[0, 0], w[0, d * f], w[0, 2 * d * f], w[0, 2 * d * f + f] = gate, up, down, down / 2
    cache.weights.copy_(dev(w))
    cache.slot_of.zero_()
    xs = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
    xs[:, 0] = x
    ids, wt = np.zeros((T, 1), np.int32), np.full((T, 1), weight, np.float32)
    with np.errstate(all="ignore"):
        want, bound = ref.moe_experts(xs.float().cpu().numpy(), ids, wt, cache.weights.float().cpu().numpy(), [0], d, f,
                                      None, "bf16")
    return fm.moe_experts(cache, xs, dev(ids), dev(wt)), want, bound


@pytest.mark.parametrize("T", LENGTHS)
def test_products_beyond_the_largest_bfloat16(T):
    """silu(128) is 128, so that h is the largest bf16 times 1 + 1.5 2^-9: a float32
    number that lies nearer to the bf16 after the largest (there is none) than to it."""
    top = float(torch.finfo(torch.bfloat16).max)
    for sign in (1, -1):
        got, want, bound = _single(T, 8, 8, 128.0, sign * top / 128, 2.0 ** -20, 1 + 1.5 * 2.0 ** -9)
        assert np.isfinite(want).all() and (np.abs(want[:, 0]) > 1e32).all()
        close(got, want, bound, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", LENGTHS)
def test_infinite_weights_of_a_down_projection(T, dtype):
    """Outputs that meet one are infinite, of the sign of its product, and the other rows as they were."""
    fm = _fm()
    rng = np.random.default_rng(T)
    d, f, E, K = 72, 136, 3, 2
    cache, slots = _layer(rng, E, E, d, f, dtype)
    cache.slot_of.copy_(torch.arange(E, device="cuda", dtype=torch.int32))
    x, xn = drawn(rng, (T, d), dtype)
    ids = np.stack([rng.permutation(E)[:K] for _ in range(T)]).astype(np.int32)
    wt = (rng.random((T, K)) + 0.1).astype(np.float32)
    at = {5: (0, 3, np.inf), 20: (1, 70, -np.inf), 71: (2, 135, np.inf)}   # row: expert, place, weight
    want, bound = ref.moe_experts(xn, ids, wt, slots, np.arange(E), d, f, None, dtype)
    for row, (e, place, v) in at.items():
        cache.weights[e, (2 * d + row) * f + place] = v
        alone = slots.copy()
        alone[:, 2 * d * f:] = 0
        alone[e, (2 * d + row) * f + place] = np.sign(v)
        product = ref.moe_experts(xn, ids, wt, alone, np.arange(E), d, f, None, dtype)[0][:, row]
        takes = (ids == e).any(axis=1)
        assert (product[takes] != 0).all()
        want[takes, row] = np.copysign(np.inf, product[takes])
    got = fm.moe_experts(cache, x, dev(ids), dev(wt))
    infinite = np.isinf(want)
    assert infinite.any() and np.array_equal(got.float().cpu().numpy()[infinite], want[infinite])
    close(got, want, bound, dtype)


@pytest.mark.parametrize("T", LENGTHS)
def test_infinite_weights_meet_products_of_few_bits(T):
    """h is a bf16 itself (its rest is zero), or infinite (the up projection overflows), or zero."""
    inf, nan = np.inf, np.nan
    for up, down, x, want, others in ((2.0, inf, 1.0, inf, 0.0), (-2.0, inf, 1.0, -inf, 0.0), (2.0, -inf, 1.0, -inf, 0.0),
                                      (3e38, inf, 2.0, inf, nan), (3e38, 1.0, 2.0, inf, nan), (-3e38, 0.5, 2.0, -inf, nan),
                                      (0.0, inf, 1.0, nan, 0.0)):
        got = _single(T, 8, 8, 128.0, up, down, 1.0, x)[0].float().cpu().numpy()
        row = np.array([want, want] + [others] * 6, np.float32)   # 0 times an infinite h is NaN
        assert np.array_equal(got, np.tile(row, (T, 1)), equal_nan=True), (up, down, x, got[0])
