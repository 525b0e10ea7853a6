"""A K tile that never comes: the waits of the attention of tall blocks run out, the call gives up without writing anything, the status says so once, and the next
call is right.  (Nothing faults: the producer leaves the copy out, every wait has a limit of 2 ms.)"""
import pytest
import torch

from paper_2502_08923_b200 import binding as cs
from paged_helpers import Case, check_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("lens,cached,tile", [([40], [300], 0), ([40], [1500], 2), ([300, 1, 70], [900, 40, 500], 1), ([200], [2000], 5)])
def test_gives_up_and_recovers(D, lens, cached, tile, monkeypatch):
    monkeypatch.setenv("CS_WAIT_LIMIT_US", "2000")
    case = Case(lens, cached, 8, 2, D, seed=tile)
    cache = cs.PagedCache(case.kp, case.vp)
    want = case.attention()
    out, lse = torch.full_like(case.q, 7.0), torch.full((case.rows, 8), 7.0, device="cuda")
    cache.cs_paged_debug_drop_tile(tile)
    cache.cs_paged_attention(case.q, *case.blocks(), out=out, lse=lse)
    status = cache.cs_paged_status()
    # CTAs whose runs have fewer tiles are not concerned
    assert status in (cs.CS_ERR_TIMEOUT, cs.CS_OK) and (tile > 0 or status == cs.CS_ERR_TIMEOUT)
    if tile == 0:
        assert bool((out == 7.0).all()) and bool((lse == 7.0).all())
    assert cache.cs_paged_status() == cs.CS_OK
    for _ in range(3):
        cache.cs_paged_attention(case.q, *case.blocks(), out=out, lse=lse)
        assert cache.cs_paged_status() == cs.CS_OK
        check_attention(case, out, lse, *want)


def test_hook_is_cleared_and_few_rows_do_without():
    case = Case([1], [300], 8, 2, 128, seed=3)
    cache = cs.PagedCache(case.kp, case.vp)
    cache.cs_paged_debug_drop_tile(0)
    out, lse = cache.cs_paged_attention(case.q, *case.blocks(), with_lse=True)      # (kept for the next tall call)
    check_attention(case, out, lse, *case.attention())
    cache.cs_paged_debug_drop_tile(-1)
    tall = Case([60], [300], 8, 2, 128, seed=4)
    other = cs.PagedCache(tall.kp, tall.vp, workspace=cache)
    out, lse = other.cs_paged_attention(tall.q, *tall.blocks(), with_lse=True)
    assert cache.cs_paged_status() == cs.CS_OK
    check_attention(tall, out, lse, *tall.attention())
