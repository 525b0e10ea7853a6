"""Attention of tall blocks over the cache of 4 bits whose waits run out in the middle of their runs, behind tiles enough for every ring and every packed place to have gone round: what was not finished stays as it was, what was
is right, and so is the next call.  (Nothing faults: the warps that write tiles out leave one unannounced, or its copy is left out; every wait has a limit of 2 ms.)"""
import pytest
import torch

from paper_2502_08923_b200 import binding as cs
from quant_helpers import QuantCase, check_attention, is_tall

pytestmark = pytest.mark.gpu


def tiles_of(case):
    """Tiles that all items of the call have between them, at least (items are of up to 256 query rows of a KV head; rows of a block see all that was cached before it)."""
    return case.Hkv * sum(-(-n * (case.H // case.Hkv) // 256) * (c // 128) for n, c in zip(case.lens, case.cached))


def items_of(case):
    """Items, at most."""
    tokens = 2 * (128 // (case.H // case.Hkv))
    return case.Hkv * sum(-(-n // tokens) for n in case.lens)


def give_up(case, tile, monkeypatch):
    """A call whose CTAs never get their tile-th K tile, after one that has left finished pieces in the workspace; rows and heads that were not written."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    # (a CTA's run is at least tile + 1 tiles and the two places that each of its items takes besides)
    assert is_tall(case) and (tiles_of(case) + 2 * items_of(case)) // sms - 2 * (items_of(case) // sms + 2) > tile + 1
    monkeypatch.setenv("CS_WAIT_LIMIT_US", "2000")
    cache = cs.QuantCache(case.kd, case.vd, case.ks, case.vs, tall_positions=case.cache.tall_positions)
    want = case.attention()
    case.q = -case.q
    check_attention(case, *cache.cs_quant_attention(case.q, *case.blocks(), with_lse=True), *case.attention(), tall=True)
    case.q = -case.q
    out, lse = torch.full_like(case.q, 7.0), torch.full(case.q.shape[:2], 7.0, device="cuda")
    cache.cs_quant_debug_drop_tile(tile)
    cache.cs_quant_attention(case.q, *case.blocks(), out=out, lse=lse)
    assert cache.cs_quant_status() == cs.CS_ERR_TIMEOUT and cache.cs_quant_status() == cs.CS_OK
    left = (out == 7.0).all(dim=-1) & (lse == 7.0)
    check_attention(case, torch.where(left[..., None], want[0].to(out.dtype), out), torch.where(left, want[1].float(), lse), *want, tall=True)
    for _ in range(2):
        check_attention(case, *cache.cs_quant_attention(case.q, *case.blocks(), with_lse=True), *want, tall=True)
        assert cache.cs_quant_status() == cs.CS_OK
    return left


@pytest.mark.parametrize("D,dtype", [(32, torch.bfloat16), (64, torch.float16), (128, torch.bfloat16), (128, torch.float16)])
@pytest.mark.parametrize("tile", [1, 5, 10])
@pytest.mark.parametrize("lens,cached,Hkv", [([200], [12000], 16), ([70, 1, 300, 33], [12000, 500, 4000, 9000], 16)])
def test_in_the_middle_of_a_run(D, dtype, tile, lens, cached, Hkv, monkeypatch):
    left = give_up(QuantCase(lens, cached, 2 * Hkv, Hkv, D, dtype, page=16 if tile & 1 else 64, seed=tile), tile, monkeypatch)
    assert bool(left.any())
    if lens == [200]:                                     # items of 94 tiles and more: all have several CTAs, and none of those is done
        assert bool(left.all())


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("tile", [2, 9])
def test_from_copies(D, tile, monkeypatch):
    """Chunks by way of copies in 16 bits (3,200 query rows per KV head)."""
    case = QuantCase([100], [9000], 128, 4, D, seed=tile, tall=1 << 14)
    assert case.rows * 32 > 2560
    assert bool(give_up(case, tile, monkeypatch).any())


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("tile", [3, 6])
def test_with_a_second_pass_to_come(D, tile, monkeypatch):
    """CTAs that give up after results that are not finite, which would have them go through those items again: they do not, and nobody waits."""
    monkeypatch.setenv("CS_WAIT_LIMIT_US", "2000")
    case = QuantCase([20] * 200, [(29 * b) % 300 for b in range(200)], 32, 8, D, seed=tile)      # items of one to three tiles: some are done before the tile that does not come
    for b in range(0, 200, 3):
        pos = case.cached[b] + 10
        case.vs[case.table[b, pos // case.page].long(), :, pos % case.page] = float("nan")
    cache = cs.QuantCache(case.kd, case.vd, case.ks, case.vs)
    assert is_tall(case)
    good = cache.cs_quant_attention(case.q, *case.blocks(), with_lse=True)
    assert cache.cs_quant_status() == cs.CS_OK
    out, lse = torch.full_like(case.q, 7.0), torch.full(case.q.shape[:2], 7.0, device="cuda")
    cache.cs_quant_debug_drop_tile(tile)
    cache.cs_quant_attention(case.q, *case.blocks(), out=out, lse=lse)
    assert cache.cs_quant_status() == cs.CS_ERR_TIMEOUT and cache.cs_quant_status() == cs.CS_OK
    # rows of sequences without such values are as they should be, or as they were
    clean = torch.tensor([r for b in range(200) if b % 3 for r in range(case.starts[b], case.starts[b] + 20)], device="cuda")
    left = (out == 7.0).all(dim=-1) & (lse == 7.0)
    assert bool(left.any()) and bool((left | ((out == good[0]).all(dim=-1) & (lse == good[1])))[clean].all())
    again = cache.cs_quant_attention(case.q, *case.blocks(), with_lse=True)
    assert cache.cs_quant_status() == cs.CS_OK
    assert torch.equal(again[0].view(torch.int16), good[0].view(torch.int16)) and torch.equal(again[1], good[1])
