"""Counts that do not fit 32 bits are refused by the binding of the paged cache, its
attention and the norms, before they are cut (CPU only)."""
import pytest
import torch

import paper_2502_05370_amd as fm

BIG = 2 ** 32
SIZES = dict(slots=2, max_tokens=100, pages=4, layers=1, heads=1, head_dim=8, page=16)


@pytest.mark.parametrize("name,by", [("slots", 2), ("pages", 4), ("layers", 1), ("heads", 1), ("head_dim", 8), ("page", 16),
                                     ("max_tokens", 100 + 15 * BIG)])
@pytest.mark.parametrize("sign", [1, -1])
def test_a_caches_sizes(name, by, sign):
    with pytest.raises(ValueError, match="does not fit 32 bits|invalid cache"):
        fm.KvCache(**{**SIZES, name: by + sign * BIG}, device="cpu")


def test_the_size_that_was_cut_to_a_small_page():
    with pytest.raises(ValueError, match=f"page={BIG + 16} does not fit 32 bits"):
        fm.KvCache(2, 100, 4, 1, 1, 8, page=BIG + 16, device="cpu")


@pytest.mark.parametrize("at", range(4))
def test_sizes_of_pages_and_scratch(at):
    sizes = [1, 1, 8, 16]
    assert fm.kv_page_bytes(*sizes) == 2 * 16 * 64
    sizes[at] += BIG
    with pytest.raises(ValueError, match="does not fit 32 bits"):
        fm.kv_page_bytes(*sizes)
    if at < 2:
        of = [1, 8]
        of[at] += BIG
        with pytest.raises(ValueError, match="does not fit 32 bits"):
            fm.block_norm_scratch_bytes(*of)
        with pytest.raises(ValueError, match="does not fit 32 bits"):
            fm.BlockNormScratch(*of, device="cpu")


def test_query_heads():
    cache = fm.KvCache(**SIZES, device="cpu")
    for call in (lambda: fm.attn_workspace_bytes(cache, BIG + 4), lambda: fm.AttnWorkspace(cache, BIG + 4),
                 lambda: cache.ensure_workspace(BIG + 4)):
        with pytest.raises(ValueError, match=f"q_heads={BIG + 4} does not fit 32 bits"):
            call()
    cache = fm.KvCache(**SIZES, device="meta")
    q = torch.empty(2, BIG + 4, 8, dtype=torch.bfloat16, device="meta")
    with pytest.raises(ValueError, match=f"q_heads={BIG + 4} does not fit 32 bits"):
        fm.attn_decode(cache, 0, q, workspace=fm.AttnWorkspace(cache, 4))


def test_rows():
    """Tensors of more than 2^31 rows: none is taken for its count's lower half."""
    n = BIG + 4
    x = torch.empty(n, 8, dtype=torch.bfloat16, device="meta")
    for call in (lambda: fm.block_norm(x, x), lambda: fm.block_norm_grad(x, None, x, out=(x, *[None] * 4),
                                                                        scratch=fm.BlockNormScratch(4, 8, "meta"))):
        with pytest.raises(ValueError, match=f"T={n} does not fit 32 bits"):
            call()
    cache = fm.KvCache(**{**SIZES, "heads": 1}, device="meta")
    rows = x.view(n, 1, 8)
    offsets = torch.empty(3, dtype=torch.int32, device="meta")
    for call in (lambda: fm.kv_write(cache, 0, rows, rows, offsets=offsets),
                 lambda: fm.kv_read(cache, 0, offsets=offsets, out=(rows, rows))):
        with pytest.raises(ValueError, match=f"T={n} does not fit 32 bits"):
            call()
    pages = torch.empty(n, dtype=torch.int32, device="meta")
    with pytest.raises(ValueError, match=f"n={n} does not fit 32 bits"):
        fm.kv_copy(cache, pages, pages)
