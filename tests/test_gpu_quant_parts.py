"""Calls of more sequences than a launch has: each launch deals with its own as a call of them alone does."""
import pytest
import torch

from paper_2502_08923_b200 import binding as cs
from quant_helpers import QuantCase, check_attention, is_tall

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("rows", [1, 3])
def test_parts_of_a_call_are_calls_of_their_own(D, rows):
    """Bit by bit: how rows are put together and where contexts are cut goes by a sequence's rows on the average, and these all have as many."""
    n, part = 384, 128
    case = QuantCase([rows] * n, [100 + 11 * b % 1900 for b in range(n)], 8, 2, D, torch.float16, page=64, seed=D)
    assert not is_tall(case)
    got, lse = case.cache.cs_quant_attention(case.q, *case.blocks(), with_lse=True)
    for b in range(0, n, part):
        at = slice(b * rows, (b + part) * rows)
        some, some_lse = case.cache.cs_quant_attention(case.q[at], case.start[:part], case.len[b:b + part], case.kv_len[b:b + part], case.table[b:b + part], with_lse=True)
        assert torch.equal(some, got[at]) and torch.equal(some_lse, lse[at])
    assert case.cache.cs_quant_status() == cs.CS_OK
    check_attention(case, got, lse, *case.attention())
