"""Attention over the paged cache of 4 bits where slots that no row attends to hold any scale: finite ones so large that a kernel's own products with them are not, negative ones, infinities, NaN."""
import pytest
import torch

from paper_2502_08923_b200 import binding as cs
from quant_helpers import QuantCase, check_attention, is_tall

pytestmark = pytest.mark.gpu

# the largest scale of the format, the last one that 24 times it is finite for, the first that it is not, others beyond, with signs, what is not finite
SCALES = [0x7D00, 0x7D2A, 0x7D2B, 0x7F00, 0x7F7F, 0xFD2B, 0xFE80, 0xFF7F, 0x7F80, 0xFF80, 0x7FC1, 0xFFFF]


def bits(pattern):
    return pattern - (1 << 16) if pattern & 0x8000 else pattern


def poison(case, pattern, mask, window):
    """That scale in every slot that no position lies in, and at every position that no row of its sequence's block attends to."""
    raw = case.scales.view(torch.int16)
    raw[torch.isnan(case.scales)] = bits(pattern)
    for b, (n, c) in enumerate(zip(case.lens, case.cached)):
        hi = c if mask == cs.MASK_PREFIX else c + n
        for pos in [*range(max(0, c + 1 - window) if window else 0), *range(hi, c + n)] if n else range(c):
            for scales in (case.ks, case.vs):
                scales.view(torch.int16)[case.table[b, pos // case.page].long(), :, pos % case.page] = bits(pattern)


@pytest.mark.parametrize("pattern", SCALES)
@pytest.mark.parametrize("mask,window", [(cs.MASK_CAUSAL, 0), (cs.MASK_PREFIX, 0), (cs.MASK_FULL, 0), (cs.MASK_CAUSAL, 5), (cs.MASK_PREFIX, 40), (cs.MASK_FULL, 1), (cs.MASK_CAUSAL, 300)])
@pytest.mark.parametrize("lens,cached,H,D,page", [([1, 5, 2, 7], [0, 1, 333, 129], 8, 128, 16), ([9, 1, 30], [20, 515, 0], 8, 64, 32), ([3, 17, 0], [0, 260, 50], 8, 32, 16),
                                                  ([40, 1], [300, 90], 32, 128, 64), ([150, 140], [300, 40], 8, 64, 16), ([70], [511], 32, 32, 128)])
def test_slots_that_no_row_attends_to(pattern, mask, window, lens, cached, H, D, page):
    case = QuantCase(lens, cached, H, 2, D, torch.float16 if pattern & 1 else torch.bfloat16, page=page, seed=window + D, gaps=1)
    poison(case, pattern, mask, window)
    got, lse = case.cache.cs_quant_attention(case.q, *case.blocks(), mask=mask, window=window, with_lse=True)
    assert case.cache.cs_quant_status() == cs.CS_OK
    check_attention(case, got, lse, *case.attention(mask, window), tall=is_tall(case, window))


@pytest.mark.parametrize("pattern", SCALES)
@pytest.mark.parametrize("D", [32, 64, 128])
def test_copies_of_such_slots(pattern, D):
    """Prompts' chunks by way of copies in 16 bits."""
    for mask, window in ((cs.MASK_CAUSAL, 0), (cs.MASK_PREFIX, 0), (cs.MASK_CAUSAL, 70)):
        case = QuantCase([50, 45], [300, 40], 128, 2, D, torch.float16 if pattern & 1 else torch.bfloat16, seed=D, tall=1 << 12)
        poison(case, pattern, mask, window)
        got, lse = case.cache.cs_quant_attention(case.q, *case.blocks(), mask=mask, window=window, with_lse=True)
        assert case.cache.cs_quant_status() == cs.CS_OK
        check_attention(case, got, lse, *case.attention(mask, window), tall=True)


@pytest.mark.parametrize("pattern", SCALES[2:])
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("lens,H", [([6, 3], 8), ([150, 140], 8)])
def test_positions_that_some_rows_attend_to(pattern, D, lens, H):
    """Beyond the format's largest scale: rows that attend to such a key get nothing that means anything, rows ahead of it all that they should, in every column."""
    cached, at = [300, 40], 2
    case = QuantCase(lens, cached, H, 2, D, torch.bfloat16, seed=5)
    want, want_lse, size = case.attention()
    raw = case.vs.view(torch.int16)
    for b in range(2):
        pos = cached[b] + at
        raw[case.table[b, pos // case.page].long(), 1, pos % case.page, (D // 32 - 1) * b] = bits(pattern)
    got, lse = case.cache.cs_quant_attention(case.q, *case.blocks(), with_lse=True)
    assert case.cache.cs_quant_status() == cs.CS_OK
    for b, (s, n) in enumerate(zip(case.starts, lens)):
        group = 32 * (D // 32 - 1) * b
        got[s + at:s + n, H // 2:, group:group + 32] = want[s + at:s + n, H // 2:, group:group + 32].to(got.dtype)
    check_attention(case, got, lse, want, want_lse, size, tall=is_tall(case))
