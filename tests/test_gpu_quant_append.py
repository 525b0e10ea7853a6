"""Rows quantised into the paged cache of 4 bits and read back, against the format's definition in 64 bits: numbers and scales are compared bit by bit."""
import math

import pytest
import torch

from paper_2502_08923_b200 import binding as cs
from paged_helpers import check_rows
from quant_helpers import GROUP, QuantCase, U, held, i32, norm_rope, pack, quantise, unpack

pytestmark = pytest.mark.gpu


def rows_for(case, dtype, seed=7, views=True):
    """q, k, v of the case's rows: views of one projection's output, or tensors of their own."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    H, Hkv, D = case.H, case.Hkv, case.D
    x = torch.randn(case.rows, H + 2 * Hkv, D, generator=g, device="cuda").to(dtype)
    q, k, v = x.split([H, Hkv, Hkv], dim=1)
    return (q, k, v) if views else (q.contiguous(), k.contiguous(), v.contiguous())


def positions(case):
    """(rows, their positions, pages, slots) of all blocks."""
    rows, pos, page = [], [], []
    for b, (s, n, c) in enumerate(zip(case.starts, case.lens, case.cached)):
        p = torch.arange(c, c + n, device="cuda")
        rows.append(torch.arange(s, s + n, device="cuda"))
        pos.append(p)
        page.append(case.table[b].long()[p // case.page])
    rows, pos, page = (torch.cat(x) for x in (rows, pos, page))
    return rows, pos, page, pos % case.page


def check_pages(case, which, want, before, exact):
    """The blocks' positions hold `want` [rows][Hkv][D] (64 bits; `exact`: without a rounding) quantised, all others what they held before."""
    data, scales = (case.kd, case.ks) if which == "k" else (case.vd, case.vs)
    rows, _, page, slot = positions(case)
    n, s = quantise(want[rows])
    got_n, got_s = unpack(data[page, :, slot]), scales[page, :, slot].double()
    assert torch.equal(got_s.nan_to_num(-1.0), s.to(torch.bfloat16).double().nan_to_num(-1.0))
    off = got_n != n
    assert not exact or not bool(off.any())
    if bool(off.any()):
        # (a number may be the other one only where 64 bits of another order cannot tell)
        q = want[rows].unflatten(-1, (-1, GROUP)) / s[..., None]
        near = ((q - torch.floor(q) - 0.5).abs() < 1e-9).flatten(-2)
        assert bool(near[off].all()), f"{int((off & ~near).sum())} of {off.numel()} numbers are others, first {torch.nonzero(off & ~near)[0].tolist()}"
    i = 0 if which == "k" else 1
    whole = torch.ones(case.data.shape[1:4], dtype=torch.bool, device="cuda")
    whole[page, :case.Hkv, slot] = False
    assert torch.equal(case.data[i][whole], before[0][i][whole]) and torch.equal(case.scales[i].view(torch.int16)[whole], before[1][i].view(torch.int16)[whole])


SHAPES = [([1], [0], 4, 1, 128), ([11], [4096], 32, 8, 128), ([1] * 9, [0, 1, 15, 16, 17, 100, 31, 32, 63], 32, 8, 64), ([5, 0, 21, 3], [7, 9, 250, 0], 8, 8, 32), ([300, 77], [3, 500], 6, 3, 64),
          ([33, 2], [1, 40], 5, 5, 128), ([130], [0], 20, 10, 32)]


@pytest.mark.parametrize("lens,cached,H,Hkv,D", SHAPES)
@pytest.mark.parametrize("source,dtype", [(torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16), (torch.float32, torch.bfloat16), (torch.float32, torch.float16)])
@pytest.mark.parametrize("norm,rotate", [(False, 0), (False, 1), (True, 1), (True, 0.5), (False, 0.5)])
def test_append(lens, cached, H, Hkv, D, source, dtype, norm, rotate):
    case = QuantCase(lens, cached, H, Hkv, D, dtype, page=16 if D != 64 else 32, gaps=2, apart=1 if D == 32 else 0)
    q, k, v = rows_for(case, source)
    rot = int(D * rotate) // 16 * 16
    rope = cs.cs_rope_table(max(n + c for n, c in zip(lens, cached)), rot) if rot else None
    gain = lambda seed: (1 + 0.2 * torch.randn(D, generator=torch.Generator().manual_seed(seed))).to(dtype).cuda()
    qg, kg = (gain(1), gain(2)) if norm else (None, None)
    before = case.data.clone(), case.scales.clone()
    got = case.cache.cs_quant_append(k, v, *case.blocks(), rope, kg, q, qg, dtype=dtype)
    assert case.cache.cs_quant_status() == cs.CS_OK
    rows, pos, _, _ = positions(case)
    at = torch.zeros(case.rows, dtype=torch.int64, device="cuda")
    at[rows] = pos
    want, size = norm_rope(q, qg, rope, at)
    assert got.dtype == dtype
    check_rows(got[rows], want[rows], size[rows], dtype)
    check_pages(case, "k", norm_rope(k, kg, rope, at)[0], before, exact=not norm and not rot)
    check_pages(case, "v", v.double(), before, exact=True)


def test_format():
    """Hand-made groups: halves, the largest elements, zeros, a tie of the scale, what is not finite."""
    case = QuantCase([8], [0], 1, 1, 32)
    x = torch.zeros(8, 1, 32, device="cuda")
    x[0, 0] = torch.arange(32) - 16.0                                     # a = 16: 16 / 7 = 2.2857 -> 2.25
    x[1, 0, :4] = torch.tensor([7.0, 0.5, 1.5, -2.5])                     # s = 1: halves go to even
    x[2, 0, 0] = 1e-30
    x[3, 0, 5] = math.inf
    x[4, 0, 31] = math.nan
    x[5, 0, :2] = torch.tensor([-7 * 2.0 ** 100, 2.0 ** 100])
    x[6, 0, :3] = torch.tensor([7 * 1.03125, 1.0, -1.03125])              # a / 7 halfway between 1 and 1.0625: to even
    case.cache.cs_quant_append(x, x.clone(), *case.blocks())
    n, s = unpack(case.kd[case.table[0, 0].long()])[0, :8], case.ks[case.table[0, 0].long()][0, :8, 0].double()
    assert s.nan_to_num(-1.0).tolist() == [2.25, 1.0, float(round5_of(1e-30 / 7)), -1.0, -1.0, 2.0 ** 100, 1.0, 0.0]
    assert n[0].tolist() == [max(-7.0, float(round((i - 16) / 2.25))) for i in range(32)]
    assert n[1, :5].tolist() == [7.0, 0.0, 2.0, -2.0, 0.0] and n[5, :3].tolist() == [-7.0, 1.0, 0.0] and n[6, :3].tolist() == [7.0, 1.0, -1.0]
    assert bool((n[7] == 0).all()) and torch.equal(case.kd, case.vd) and torch.equal(case.ks.view(torch.int16), case.vs.view(torch.int16))
    k, v = case.cache.cs_quant_read(*case.blocks(), rows=8, dtype=torch.float32)
    assert torch.equal(torch.isnan(k), torch.isnan(s)[:, None, None].expand(8, 1, 32)) and torch.equal(k.nan_to_num(5.0), v.nan_to_num(5.0))
    fine = ~torch.isnan(s)
    assert torch.equal(k[fine, 0].double(), (n * s[:, None])[fine])


def round5_of(x):
    from quant_helpers import round5
    return torch.tensor(float(round5(torch.tensor(x, dtype=torch.float64)))).to(torch.bfloat16).item()


def test_every_number_and_scale_reads_back():
    """All sixteen numbers at all places of a word, scales of five bits from 2^-126 to 2^120: exact in bf16 and fp32, rounded and saturated in fp16."""
    exponents = list(range(-126, 121, 6))
    case = QuantCase([len(exponents) * 16], [0], 1, 1, 128, page=16)
    T = case.rows
    n = torch.stack([(torch.arange(128) * 7 + r) % 16 for r in range(T)]).cuda() - 8
    mantissa = torch.tensor([16 + r % 16 for r in range(T)], dtype=torch.float64)
    s = torch.ldexp(mantissa / 16, torch.tensor([float(exponents[r // 16]) for r in range(T)], dtype=torch.float64)).cuda()[:, None].expand(T, 4)
    _, pos, page, slot = positions(case)
    for data, scales in ((case.kd, case.ks), (case.vd, case.vs)):
        data[page, 0, slot] = pack(n)
        scales[page, 0, slot] = s.to(torch.bfloat16)
    want = held(n.double(), s)[:, None]
    for dtype in (torch.bfloat16, torch.float32, torch.float16):
        for x in case.cache.cs_quant_read(*case.blocks(), rows=T, dtype=dtype):
            assert torch.equal(x, want.clamp(-65504, 65504).to(dtype) if dtype is torch.float16 else want.to(dtype))


@pytest.mark.parametrize("lens,cached,H,Hkv,D", SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("page", [16, 64])
def test_read(lens, cached, H, Hkv, D, dtype, page):
    case = QuantCase(lens, cached, H, Hkv, D, page=page, gaps=1)
    out = tuple(torch.full((case.rows, 2 * Hkv, D), 7.0, dtype=dtype, device="cuda")[:, Hkv * i:Hkv * i + Hkv] for i in range(2))
    case.cache.cs_quant_read(*case.blocks(), out=out)
    fresh = case.cache.cs_quant_read(*case.blocks(), rows=case.rows, dtype=dtype)
    assert case.cache.cs_quant_status() == cs.CS_OK
    live = case.live()
    for got, again, rows in zip(out, fresh, (case.k, case.v)):
        want = torch.cat([x[c:] for x, c in zip(rows, cached)]).to(dtype)
        assert torch.equal(got[live], want) and torch.equal(again[live], want) and bool((got[~live] == 7.0).all())


def test_appended_rows_read_back_whole():
    """Blocks one after the other, then whole sequences read back: no element is off by more than half a step."""
    lens, D, Hkv = [40, 3, 17], 128, 2
    case = QuantCase(lens, [0, 0, 0], 2, Hkv, D, page=16, n_pages=40)
    wide = -(-3 * max(lens) // case.page)
    table = torch.arange(3 * wide, device="cuda", dtype=torch.int32).view(3, wide)
    kv = torch.zeros(3, dtype=torch.int32, device="cuda")
    ks, vs = [[] for _ in lens], [[] for _ in lens]
    for step in range(3):
        q, k, v = rows_for(case, torch.bfloat16, seed=step)
        case.cache.cs_quant_append(k, v, case.start, case.len, kv, table)
        for b, (s, n) in enumerate(zip(case.starts, lens)):
            ks[b].append(k[s:s + n])
            vs[b].append(v[s:s + n])
        kv += case.len
    assert case.cache.cs_quant_status() == cs.CS_OK
    total = [3 * n for n in lens]
    start = i32([0, total[0], total[0] + total[1]])
    got = case.cache.cs_quant_read(start, i32(total), torch.zeros_like(kv), table, rows=sum(total), dtype=torch.float32)
    for x, rows in zip(got, (ks, vs)):
        want = torch.cat([torch.cat(r) for r in rows]).double()
        n, s = quantise(want)
        assert torch.equal(x.double(), held(n, s))
        assert bool(((x.double() - want).abs() <= s.repeat_interleave(GROUP, dim=-1) / 2).all())


def test_what_the_device_finds_wrong():
    case = QuantCase([3, 4, 5], [10, 20, 30], 4, 2, 64)
    q, k, v = rows_for(case, torch.bfloat16)
    before = case.data.clone(), case.scales.clone()
    for start, length, kv, code in (([0, 3, 7], [3, -1, 5], [10, 20, 30], cs.CS_ERR_ARG), ([0, 3, 9], [0, 0, 5], [10, 20, 30], cs.CS_ERR_ARG), ([0, 3, 7], [0, 4, 0], [10, 2000, 30], cs.CS_ERR_CAPACITY),
                                    ([0, 3, 7], [0, 0, 5], [10, 20, -3], cs.CS_ERR_ARG)):
        args = i32(start), i32(length), i32(kv), case.table
        if length[0]:
            args = args[0], i32([0, -1, 0]), *args[2:]
        case.cache.cs_quant_append(k, v, *args, None, None, q)
        assert case.cache.cs_quant_status() == code and case.cache.cs_quant_status() == cs.CS_OK
        out = tuple(torch.full((12, 2, 64), 3.0, device="cuda") for _ in range(2))
        case.cache.cs_quant_read(*args, out=out)
        assert case.cache.cs_quant_status() == code and all(bool((x == 3.0).all()) for x in out)
    assert torch.equal(case.data, before[0]) and torch.equal(case.scales.view(torch.int16), before[1].view(torch.int16))
    # positions behind the rotation table, a page that does not exist: the others' rows are there
    table = case.table.clone()
    table[1, 1] = case.data.shape[1]
    case.cache.cs_quant_append(k, v, *case.blocks()[:3], table, cs.cs_rope_table(32, 64), None, q)
    assert case.cache.cs_quant_status() == cs.CS_ERR_CAPACITY
    case.cache.cs_quant_append(k, v, *case.blocks()[:3], table)
    assert case.cache.cs_quant_status() == cs.CS_ERR_ARG
    got = case.cache.cs_quant_read(*case.blocks()[:3], table, rows=case.rows, dtype=torch.float32)
    assert case.cache.cs_quant_status() == cs.CS_ERR_ARG
    for x, rows in zip(got, (k, v)):
        want = held(*quantise(rows))
        assert torch.equal(x[:3].double(), want[:3]) and torch.equal(x[7:].double(), want[7:]) and bool((x[3:7] == 0).all())


def test_empty_calls():
    case = QuantCase([3], [5], 4, 2, 64)
    none = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    case.cache.cs_quant_append(none, none, *case.blocks())
    k, v = case.cache.cs_quant_read(*case.blocks(), rows=0)
    assert k.shape == v.shape == (0, 2, 64)
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    q, k, v = rows_for(case, torch.bfloat16)
    case.cache.cs_quant_append(k, v, e, e, e, torch.empty(0, 3, dtype=torch.int32, device="cuda"))
    case.cache.cs_quant_append(k, v, case.start, torch.zeros_like(case.len), case.kv_len, case.table)
    assert case.cache.cs_quant_status() == cs.CS_OK
