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
