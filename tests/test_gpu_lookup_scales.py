"""Embedding rows and their means under scales that are no ordinary numbers."""
import pytest
import torch

from test_gpu_operators import _fm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("scale", [float("inf"), float("-inf"), float("nan")])
def test_padding_is_zeros_under_any_scale(scale, dtype):
    fm = _fm()
    for d in (5, 64):
        table = torch.ones(3, d, dtype=dtype, device="cuda")
        tok = torch.tensor([1, -1, 3, 2, -5], dtype=torch.int32, device="cuda")
        got = fm.embed_lookup(table, tok, scale).float().cpu()
        assert (got[[1, 2, 4]] == 0).all()
        assert torch.equal(got[[0, 3]], torch.full((2, d), scale)) or (scale != scale and got[[0, 3]].isnan().all())
        off = torch.tensor([0, 1, 2, 3], dtype=torch.int32, device="cuda")
        got = fm.embed_pool(table, tok, off, scale).float().cpu()
        assert (got[1:] == 0).all() and not torch.isfinite(got[0]).any()
        into = fm.embed_grad(torch.ones(5, d, dtype=dtype, device="cuda"), tok, 4, scale).cpu()
        assert (into[0] == 0).all() and not torch.isfinite(into[[1, 2, 3]]).any()
