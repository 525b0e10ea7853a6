"""Groups whose scales lie below 2^-126, where bf16 has fewer bits: multiples of 2^-133.  Reading back is exact."""
import pytest
import torch

from paper_2502_08923_b200 import binding as cs
from quant_helpers import QuantCase, held, pack

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [32, 64, 128])
def test_every_small_scale_reads_back(D):
    """All scales of up to five significant bits from 2^-133 to 2^-125, all sixteen numbers at all places of a word."""
    # (up to there a bf16 pattern counts multiples of 2^-133)
    patterns = [p for p in range(1, 0x100) if len(bin(p).rstrip("0")) - 2 <= 5]
    case = QuantCase([len(patterns) * 16], [0], 1, 1, D)
    T = case.rows
    n = torch.stack([(torch.arange(D) * 7 + r) % 16 for r in range(T)]) - 8
    bits = torch.tensor([patterns[r // 16] for r in range(T)], dtype=torch.int16)
    s = (bits.double() * 2.0 ** -133)[:, None].expand(T, D // 32)
    pos = torch.arange(T)
    page, slot = case.table[0].long().cpu()[pos // case.page].cuda(), (pos % case.page).cuda()
    for data, scales in ((case.kd, case.ks), (case.vd, case.vs)):
        data[page, 0, slot] = pack(n).cuda()
        scales.view(torch.int16)[page, 0, slot] = bits.cuda()[:, None].expand(T, D // 32)
    want = held(n.double(), s)[:, None]
    for dtype in (torch.bfloat16, torch.float32, torch.float16):
        for x in case.cache.cs_quant_read(*case.blocks(), rows=T, dtype=dtype):
            # (five bits times three: exact in bf16; in fp16 all of it is below half of the smallest number)
            assert torch.equal(x.double().cpu(), want if dtype is not torch.float16 else torch.zeros_like(want))
