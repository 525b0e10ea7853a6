"""Groups whose scales lie below 2^-126, where bf16 has fewer bits: multiples of 2^-133.  Reading back is exact, and their scales and numbers are the format's whichever way a row comes in."""
import pytest
import torch

from paper_2502_08923_b200 import binding as cs
from quant_helpers import QuantCase, held, pack, round5, unpack

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


def small_rows(T, D, dtype, seed):
    """Rows of groups from 2^-149 to 2^-100 in size, some of zeros."""
    g = torch.Generator().manual_seed(seed)
    size = torch.randint(-149, -99, (T, D // 32), generator=g).double()
    x = torch.randn(T, D // 32, 32, generator=g).double() * (2.0 ** size)[..., None]
    x[:: 7, 0] = 0
    return x.flatten(1).to(dtype)


def small_groups(x):
    """(numbers, scales) in 64 bits: s = max / 7 to five significant bits, and to a multiple of 2^-133; n = x / s of that."""
    g = x.double().unflatten(-1, (-1, 32))
    s = round5(g.abs().amax(dim=-1) / 7)
    s = torch.where(s < 2.0 ** -126, torch.round(s * 2.0 ** 133) * 2.0 ** -133, s)
    n = torch.round(g / torch.where(s > 0, s, torch.ones_like(s))[..., None]).clamp(-7, 7)
    return torch.where(s[..., None] > 0, n, torch.zeros_like(n)).flatten(-2), s


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rotated", [False, True])
def test_small_rows_appended(D, dtype, rotated):
    """The same rows as keys and as values.  (Rotated by nothing, at position 0 of sequences of a row each, keys are worked out in 64 bits; else in 32, as values are.)"""
    T = 300
    case = QuantCase([1] * T, [0] * T, 1, 1, D)
    x = small_rows(T, D, dtype, D)
    rows = x.cuda()[:, None]
    case.cache.cs_quant_append(rows, rows.clone(), *case.blocks(), cs.cs_rope_table(1, D) if rotated else None)
    assert case.cache.cs_quant_status() == cs.CS_OK
    want_n, want_s = small_groups(x)
    page = case.table[:, 0].long()
    for data, scales in ((case.kd, case.ks), (case.vd, case.vs)):
        s = scales[page, 0, 0].cpu().view(torch.int16)
        # (bf16 patterns of positive numbers are in their order, and those below 2^-126 count multiples of 2^-133)
        assert torch.equal(s, want_s.float().to(torch.bfloat16).view(torch.int16))
        assert torch.equal(unpack(data[page, 0, 0]).cpu(), want_n)
    got = case.cache.cs_quant_read(*case.blocks(), rows=T, dtype=torch.float32)
    for y in got:
        assert torch.equal(y[:, 0].double().cpu(), held(want_n, want_s))
