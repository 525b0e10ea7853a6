"""A K tile that never comes, over the cache of 4 bits: the waits of the attention of tall blocks run out, the call gives up, the status says so once, and the next call is right.  (Nothing faults: the warps that
write tiles out leave one unannounced, or its copy is left out; every wait has a limit of 2 ms.)"""
import pytest
import torch

from paper_2502_08923_b200 import binding as cs
from quant_helpers import QuantCase, check_attention, is_tall

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("lens,cached,H,tile,room", [([40], [300], 16, 0, 0), ([40], [1500], 16, 2, 0), ([300, 1, 70], [900, 40, 500], 8, 1, 0), ([200], [2000], 8, 5, 0), ([100], [300], 64, 0, 1 << 10)])
def test_gives_up_and_recovers(D, lens, cached, H, tile, room, monkeypatch):
    monkeypatch.setenv("CS_WAIT_LIMIT_US", "2000")
    case = QuantCase(lens, cached, H, 2, D, seed=tile, tall=room)
    assert is_tall(case)
    want = case.attention()
    out, lse = torch.full_like(case.q, 7.0), torch.full((case.rows, H), 7.0, device="cuda")
    case.cache.cs_quant_debug_drop_tile(tile)
    case.cache.cs_quant_attention(case.q, *case.blocks(), out=out, lse=lse)
    status = case.cache.cs_quant_status()
    # CTAs whose runs have fewer tiles are not concerned
    assert status in (cs.CS_ERR_TIMEOUT, cs.CS_OK) and (tile > 0 or status == cs.CS_ERR_TIMEOUT)
    if tile == 0:
        assert bool((out == 7.0).all()) and bool((lse == 7.0).all())
    assert case.cache.cs_quant_status() == cs.CS_OK
    for _ in range(3):
        case.cache.cs_quant_attention(case.q, *case.blocks(), out=out, lse=lse)
        assert case.cache.cs_quant_status() == cs.CS_OK
        check_attention(case, out, lse, *want, tall=True)
