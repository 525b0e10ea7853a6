"""Attention of tall blocks whose waits run out in the middle of their runs: what was not finished stays as it was - rows that several CTAs share too, whichever of them
gave up - and what was is right.  (Nothing faults: the producer leaves a copy out, every wait has a limit of 2 ms.)"""
import pytest
import torch

from paper_2502_08923_b200 import binding as cs
from paged_helpers import Case, check_attention

pytestmark = pytest.mark.gpu


def give_up(case, tile, monkeypatch):
    """A call whose CTAs never get their tile-th K tile, after one that has left finished pieces in the workspace; (rows and heads that were not written, want)."""
    monkeypatch.setenv("CS_WAIT_LIMIT_US", "2000")
    cache = cs.PagedCache(case.kp, case.vp)
    want = case.attention()
    check_attention(case, *cache.cs_paged_attention(-case.q, *case.blocks(), with_lse=True), *negated(case))
    out, lse = torch.full_like(case.q, 7.0), torch.full(case.q.shape[:2], 7.0, device="cuda")
    cache.cs_paged_debug_drop_tile(tile)
    cache.cs_paged_attention(case.q, *case.blocks(), out=out, lse=lse)
    assert cache.cs_paged_status() == cs.CS_ERR_TIMEOUT and cache.cs_paged_status() == cs.CS_OK
    left = (out == 7.0).all(dim=-1) & (lse == 7.0)
    check_attention(case, torch.where(left[..., None], want[0].to(out.dtype), out), torch.where(left, want[1].float(), lse), *want)
    check_attention(case, *cache.cs_paged_attention(case.q, *case.blocks(), with_lse=True), *want)
    assert cache.cs_paged_status() == cs.CS_OK
    return left


def negated(case):
    case.q = -case.q
    want = case.attention()
    case.q = -case.q
    return want


@pytest.mark.parametrize("D", [32, 64, 128])
def test_the_first_of_an_items_ctas_is_done_and_others_are_not(D, monkeypatch):
    """Two items, four places of the line for each CTA: the CTAs that an item begins in have two tiles of it (two places are its own cost), the others four.  Without
    the fourth tile the former finish, and announce the item."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    case = Case([40], [(2 * sms - 2) * 128 - 40], 4, 2, D, seed=D)
    assert bool(give_up(case, 3, monkeypatch).all())


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("tile", [1, 2, 5])
@pytest.mark.parametrize("lens,cached,Hkv", [([200], [9000], 16), ([70, 1, 300, 33], [12000, 500, 3000, 7000], 8)])
def test_in_the_middle_of_a_run(D, tile, lens, cached, Hkv, monkeypatch):
    """At least tile + 3 tiles a CTA: all of them give up."""
    case = Case(lens, cached, 2 * Hkv, Hkv, D, seed=tile)
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    tiles = Hkv * sum(-(-2 * n // 256) * (c // 128) for n, c in zip(lens, cached))      # (fewer than there are)
    assert tiles >= sms * (tile + 3)
    left = give_up(case, tile, monkeypatch)
    assert bool(left.any())
    if lens == [200] and tile < 3:                        # items of 71 tiles and more, no CTA gets as far as the end of one
        assert bool(left.all())


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("tile", [1, 3, 6])
def test_with_a_second_pass_to_come(D, tile, monkeypatch):
    """CTAs that give up after results that are not finite, which would have them go through those items again: they do not, and nobody waits."""
    monkeypatch.setenv("CS_WAIT_LIMIT_US", "2000")
    lens = [20] * 200                                     # items of one to three tiles: some are done before the tile that does not come
    case = Case(lens, [(29 * b) % 300 for b in range(200)], 32, 8, D, seed=tile)
    for b in range(0, 200, 3):
        case.v[b][case.cached[b] + 10, :, 1] = float("nan")
        case.put(b)
    cache = cs.PagedCache(case.kp, case.vp)
    good = cache.cs_paged_attention(case.q, *case.blocks(), with_lse=True)
    assert cache.cs_paged_status() == cs.CS_OK
    out, lse = torch.full_like(case.q, 7.0), torch.full(case.q.shape[:2], 7.0, device="cuda")
    cache.cs_paged_debug_drop_tile(tile)
    cache.cs_paged_attention(case.q, *case.blocks(), out=out, lse=lse)
    assert cache.cs_paged_status() == cs.CS_ERR_TIMEOUT and cache.cs_paged_status() == cs.CS_OK
    # rows of sequences without such values are as they should be, or as they were
    clean = torch.tensor([r for b in range(200) if b % 3 for r in range(case.starts[b], case.starts[b] + 20)], device="cuda")
    left = (out == 7.0).all(dim=-1) & (lse == 7.0)
    assert bool(left.any()) and bool((left | ((out == good[0]).all(dim=-1) & (lse == good[1])))[clean].all())
    again = cache.cs_paged_attention(case.q, *case.blocks(), with_lse=True)
    assert cache.cs_paged_status() == cs.CS_OK
    assert torch.equal(again[0].view(torch.int16), good[0].view(torch.int16)) and torch.equal(again[1], good[1])
