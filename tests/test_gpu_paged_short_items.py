"""Attention of many short blocks behind few keys: runs of items with one tile each, of differing heights, whose queries follow one another through the
kernel's ring as closely as they can."""
import pytest
import torch

from paper_2502_08923_b200 import binding as cs
from paged_helpers import Case, check_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("H,Hkv,most", [(32, 8, 7), (8, 8, 16)])
def test_items_of_one_tile_each(D, H, Hkv, most):
    g = torch.Generator().manual_seed(D)
    n = 300
    lens = torch.randint(0, most + 1, (n,), generator=g).tolist()
    lens = [min(x, 4) if i % 3 else x for i, x in enumerate(lens)] if most == 7 else lens
    cached = torch.randint(0, 101, (n,), generator=g).tolist()
    case = Case(lens, cached, H, Hkv, D, seed=D + most)
    assert case.rows * (H // Hkv) <= 16 * n               # the kernel for few rows
    cache = cs.PagedCache(case.kp, case.vp)
    first = cache.cs_paged_attention(case.q, *case.blocks(), with_lse=True)
    for _ in range(30):
        again = cache.cs_paged_attention(case.q, *case.blocks(), with_lse=True)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    assert cache.cs_paged_status() == cs.CS_OK
    check_attention(case, *first, *case.attention())


@pytest.mark.parametrize("D", [32, 64, 128])
def test_tall_items_between_items_of_one_tile(D):
    """On the tensor cores: after an item whose rows fill both slots, items of one tile that one slot has to itself."""
    g = torch.Generator().manual_seed(D)
    lens = [60 if b % 4 == 0 else int(torch.randint(1, 6, (1,), generator=g)) for b in range(240)]
    cached = torch.randint(0, 60, (len(lens),), generator=g).tolist()
    case = Case(lens, cached, 32, 8, D, seed=D)
    assert case.rows * 4 > 16 * len(lens)                 # the kernel for tall blocks
    cache = cs.PagedCache(case.kp, case.vp)
    first = cache.cs_paged_attention(case.q, *case.blocks(), with_lse=True)
    for _ in range(30):
        again = cache.cs_paged_attention(case.q, *case.blocks(), with_lse=True)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    assert cache.cs_paged_status() == cs.CS_OK
    check_attention(case, *first, *case.attention())
