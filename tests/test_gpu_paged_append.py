"""Norms and rotation of queries and keys, and rows appended to a paged KV cache, against the formulas in 64 bits."""
import math

import pytest
import torch

from paper_2502_08923_b200 import binding as cs
from paged_helpers import Case, check_rows, i32, norm_rope

pytestmark = pytest.mark.gpu
BF, FP, F32 = torch.bfloat16, torch.float16, torch.float32
TYPES = [(BF, BF), (FP, FP), (F32, BF), (F32, FP), (F32, F32)]


def gains(D, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(1 + 0.2 * torch.randn(D, generator=g, device="cuda")).to(dtype) for _ in range(2)]


@pytest.mark.parametrize("D", [32, 64, 128])
def test_table(D):
    got = cs.cs_rope_table(1000, D, 500000.0)
    inv = 500000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D)
    angle = torch.arange(1000, dtype=torch.float64, device="cuda")[:, None] * inv
    want = torch.cat([angle.cos(), angle.sin()], 1)
    assert float((got.double() - want).abs().max()) <= 2.0 ** -24          # one rounding of values up to 1
    far = cs.cs_rope_table(131073, 32, 10000.0)[131072]
    angle = 131072 * 10000.0 ** (-torch.arange(0, 32, 2, dtype=torch.float64, device="cuda") / 32)
    assert float((far.double() - torch.cat([angle.cos(), angle.sin()])).abs().max()) <= 2.0 ** -24


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("src,dst", TYPES)
@pytest.mark.parametrize("rows,H,Hkv", [(1, 32, 8), (11, 8, 8), (3, 7, 1), (70, 5, 3), (2, 200, 3)])
@pytest.mark.parametrize("norm", [True, False])
def test_norm_rope(D, src, dst, rows, H, Hkv, norm):
    g = torch.Generator(device="cuda").manual_seed(rows + H)
    qkv = (torch.randn(rows, (H + 2 * Hkv) * D, generator=g, device="cuda") * 3).to(src)
    q, k = qkv[:, :H * D].unflatten(1, (H, D)), qkv[:, H * D:(H + Hkv) * D].unflatten(1, (Hkv, D))
    rope = cs.cs_rope_table(500, D, 10000.0)
    pos = torch.randint(0, 500, (rows,), generator=g, device="cuda", dtype=torch.int32)
    qg, kg = gains(D, dst) if norm else (None, None)
    got = cs.cs_qk_norm_rope(q, k, pos, rope, qg, kg, dtype=dst)
    for x, y, gain in ((q, got[0], qg), (k, got[1], kg)):
        assert y.dtype == dst and y.is_contiguous()
        check_rows(y, *norm_rope(x, gain, rope, pos), dst)


@pytest.mark.parametrize("rot", [0, 16, 48, 96, 128])
def test_part_of_a_head_rotated(rot):
    q = torch.randn(5, 4, 128, device="cuda").to(BF)
    pos = i32([0, 1, 99, 7, 50])
    rope = cs.cs_rope_table(100, rot, 10000.0) if rot else None
    qg = gains(128, BF)[0]
    for gain in (None, qg):
        got, none = cs.cs_qk_norm_rope(q, None, pos if rot else None, rope, gain)
        assert none is None
        check_rows(got, *norm_rope(q, gain, rope, pos), BF)


@pytest.mark.parametrize("src,dst", TYPES)
@pytest.mark.parametrize("rows", [200, 297, 741, 1481])          # shared by 8, 4, 2 warps, with a warp each
def test_many_rows_part_rotated(src, dst, rows):
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = (2 * torch.randn(rows, 23, 128, generator=g, device="cuda")).to(src)
    rope = cs.cs_rope_table(2000, 96, 10000.0)
    pos = torch.randint(0, 2000, (rows,), generator=g, device="cuda", dtype=torch.int32)
    qg, kg = gains(128, dst)
    got = cs.cs_qk_norm_rope(x[:, :20], x[:, 20:], pos, rope, qg, kg, dtype=dst)
    check_rows(got[0], *norm_rope(x[:, :20], qg, rope, pos), dst)
    check_rows(got[1], *norm_rope(x[:, 20:], kg, rope, pos), dst)


@pytest.mark.parametrize("dt", [BF, FP, F32])
@pytest.mark.parametrize("rows,rot", [(5, 128), (1700, 64)])
def test_in_place(dt, rows, rot):
    x = torch.randn(rows, 10, 128, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(dt)
    rope, pos = cs.cs_rope_table(rows, rot), torch.arange(rows, device="cuda", dtype=torch.int32)
    qg, kg = gains(128, dt)
    want = [norm_rope(x[:, :7], qg, rope, pos), norm_rope(x[:, 7:9], kg, rope, pos)]
    rest = x[:, 9].clone()
    cs.cs_qk_norm_rope(x[:, :7], x[:, 7:9], pos, rope, qg, kg, out=(x[:, :7], x[:, 7:9]))
    check_rows(x[:, :7], *want[0], dt)
    check_rows(x[:, 7:9], *want[1], dt)
    assert torch.equal(x[:, 9], rest)


def test_in_place_and_extremes():
    x = torch.randn(9, 12, 64, device="cuda").to(BF)
    x[3, 2] = 0.0                                        # a head of zeros: eps keeps the norm finite
    x[4, 1] = 1e18                                       # squares beyond 16 bits' range, within 32's
    q, k = x[:, :8], x[:, 8:]
    rope, pos = cs.cs_rope_table(64, 64), torch.arange(9, device="cuda", dtype=torch.int32)
    qg, kg = gains(64, BF)
    want = [norm_rope(q, qg, rope, pos), norm_rope(k, kg, rope, pos)]
    got = cs.cs_qk_norm_rope(q, k, pos, rope, qg, kg, out=(q, k))
    assert got[0].data_ptr() == x.data_ptr()
    check_rows(x[:, :8], *want[0], BF)
    check_rows(x[:, 8:], *want[1], BF)


def test_positions_outside_the_table():
    q = torch.randn(4, 2, 64, device="cuda").to(BF)
    got = cs.cs_qk_norm_rope(q, None, i32([3, 10, -1, 9]), cs.cs_rope_table(10, 32))[0].float()
    assert torch.isnan(got[1, :, :32]).all() and torch.isnan(got[2, :, :32]).all() and torch.isfinite(got[[0, 3]]).all()
    assert torch.equal(got[..., 32:], q[..., 32:].float())


def append(case, src, norm, H, seed=0, rope=None, gaps=0):
    """Runs an append of all the case's blocks, checks it and returns the cache."""
    D, Hkv, dt = case.D, case.Hkv, case.dtype
    g = torch.Generator(device="cuda").manual_seed(seed)
    qkv = (2 * torch.randn(case.rows, (H + 2 * Hkv) * D, generator=g, device="cuda")).to(src)
    q, k, v = qkv[:, :H * D].unflatten(1, (H, D)), qkv[:, H * D:(H + Hkv) * D].unflatten(1, (Hkv, D)), qkv[:, (H + Hkv) * D:].unflatten(1, (Hkv, D))
    rope = rope if rope is not None else cs.cs_rope_table(max(n + c for n, c in zip(case.lens, case.cached)) + 1, D, 500000.0)
    qg, kg = gains(D, dt) if norm else (None, None)
    before = case.kp.clone(), case.vp.clone()
    cache = cs.PagedCache(case.kp, case.vp)
    q_out = torch.full((case.rows, H, D), 7.0, dtype=dt, device="cuda") if H else None
    got = cache.cs_paged_append(k, v, *case.blocks(), rope, kg, q if H else None, qg if H else None, q_out=q_out)
    assert got is q_out and cache.cs_paged_status() == cs.CS_OK
    written = torch.zeros(case.kp.shape[0], case.page, dtype=torch.bool, device="cuda")
    live = torch.zeros(case.rows, dtype=torch.bool, device="cuda")
    for b, (n, c) in enumerate(zip(case.lens, case.cached)):
        if n == 0:
            continue
        rows, pos = slice(case.starts[b], case.starts[b] + n), torch.arange(c, c + n, device="cuda")
        live[rows] = True
        at = case.table[b].long()[pos // case.page]
        written[at, pos % case.page] = True
        check_rows(case.kp[at, :, pos % case.page], *norm_rope(k[rows], kg, rope, pos), dt)
        assert torch.equal(case.vp[at, :, pos % case.page], v[rows].to(dt))
        if H:
            check_rows(q_out[rows], *norm_rope(q[rows], qg, rope, pos), dt)
    if H:
        assert bool((q_out[~live] == 7.0).all())
    kept = ~written[:, None, :, None].expand_as(case.kp)
    for now, was in zip((case.kp, case.vp), before):     # (bits: the rest holds NaN)
        assert torch.equal(now.view(torch.int16)[kept], was.view(torch.int16)[kept])
    return cache


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("dt,src", [(BF, BF), (FP, FP), (BF, F32), (FP, F32)])
@pytest.mark.parametrize("lens,cached", [([1], [0]), ([1], [16]), ([11], [4090]), ([3, 0, 1, 40], [15, 9, 0, 31]), ([200, 17], [1, 500])])
@pytest.mark.parametrize("norm", [True, False])
def test_append(D, dt, src, lens, cached, norm):
    append(Case(lens, cached, 8, 2, D, dt, seed=1), src, norm, 8)


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("src", [BF, F32])
@pytest.mark.parametrize("lens", [[250, 1, 90], [900, 2, 600]])
def test_append_of_chunks(D, src, lens):
    append(Case(lens, [30, 0, 601], 32, 8, D, seed=10, gaps=1), src, True, 32)


@pytest.mark.parametrize("page", [16, 64, 512])
@pytest.mark.parametrize("layout", ["head", "token"])
@pytest.mark.parametrize("H,Hkv", [(0, 1), (0, 8), (7, 1), (32, 8), (40, 20)])
def test_append_layouts(page, layout, H, Hkv):
    append(Case([5, 1, 33], [page - 2, 0, 2 * page + 3], max(H, Hkv), Hkv, 128, page=page, layout=layout, seed=2, gaps=3), BF, True, H)


def test_append_part_rotated_and_many_sequences():
    append(Case([5, 30], [7, 100], 4, 2, 128, seed=3), BF, True, 4, rope=cs.cs_rope_table(131, 64))
    n = 700
    append(Case([b % 3 for b in range(n)], [(b * 31) % 70 for b in range(n)], 2, 1, 64, FP, seed=4), FP, False, 2)


def test_append_offsets_beyond_32_bits():
    n_pages = (1 << 31) // (16 * 8 * 128) + 100
    case = Case([3], [40], 8, 8, 128, seed=5, first_page=n_pages - 50, n_pages=n_pages)
    k, v = (torch.randn(3, 8, 128, device="cuda").to(BF) for _ in range(2))
    cache = cs.PagedCache(case.kp, case.vp)
    cache.cs_paged_append(k, v, *case.blocks())
    assert cache.cs_paged_status() == cs.CS_OK
    pos = torch.arange(40, 43, device="cuda")
    at = case.table[0].long()[pos // 16]
    assert torch.equal(case.kp[at, :, pos % 16], k) and torch.equal(case.vp[at, :, pos % 16], v)


def test_then_attention():
    """Append and attention as a decoding step calls them: appended rows are attended to in the same stream."""
    case = Case([4, 1], [30, 130], 8, 2, 64, seed=6)
    qkv = torch.randn(case.rows, 12, 64, device="cuda")
    rope = cs.cs_rope_table(200, 64)
    cache = cs.PagedCache(case.kp, case.vp)
    case.q = cache.cs_paged_append(qkv[:, 8:10], qkv[:, 10:], *case.blocks(), rope, q=qkv[:, :8])
    out, lse = cache.cs_paged_attention(case.q, *case.blocks(), with_lse=True)
    assert cache.cs_paged_status() == cs.CS_OK
    for b, (n, c) in enumerate(zip(case.lens, case.cached)):
        pos = torch.arange(n + c, device="cuda")
        at = case.table[b].long()[pos // 16]
        case.k[b], case.v[b] = case.kp[at, :, pos % 16], case.vp[at, :, pos % 16]
    from paged_helpers import check_attention
    check_attention(case, out, lse, *case.attention())


def test_append_conditions_of_the_device():
    def fresh():
        case = Case([3, 2], [20, 40], 4, 2, 64, seed=7)
        k = torch.randn(5, 2, 64, device="cuda").to(BF)
        return case, k, cs.PagedCache(case.kp, case.vp), case.kp.clone()

    same = lambda a, b: torch.equal(a.view(torch.int16), b.view(torch.int16))
    for field, value, code in (("kv_len", 10 ** 6, cs.CS_ERR_CAPACITY), ("kv_len", -3, cs.CS_ERR_ARG), ("len", -1, cs.CS_ERR_ARG), ("start", 4, cs.CS_ERR_ARG), ("len", 2 ** 31 - 1, cs.CS_ERR_ARG)):
        case, k, cache, before = fresh()
        getattr(case, field)[1] = value
        cache.cs_paged_append(k, k, *case.blocks())
        assert cache.cs_paged_status() == code and cache.cs_paged_status() == cs.CS_OK
        pages = case.table[1][case.table[1] >= 0].long()
        assert same(case.kp[pages], before[pages])       # the other sequence's rows are there
        at = case.table[0].long()[torch.arange(20, 23, device="cuda") // 16]
        assert torch.equal(case.kp[at, :, torch.arange(20, 23, device="cuda") % 16], k[:3])
    for page in (-1, 10 ** 7):
        case, k, cache, before = fresh()
        case.table[0, 1] = page
        cache.cs_paged_append(k, k, *case.blocks())
        assert cache.cs_paged_status() == cs.CS_ERR_ARG
        assert torch.equal(case.kp[case.table[1, 2].long(), :, 8:10], k[3:].transpose(0, 1))
    case, k, cache, before = fresh()
    cache.cs_paged_append(k, k, *case.blocks(), cs.cs_rope_table(22, 64))      # positions 22, 40 and 41 lie behind the table
    assert cache.cs_paged_status() == cs.CS_ERR_CAPACITY
    at = case.table[0, 1].long()
    assert not same(case.kp[at, :, 5], before[at, :, 5]) and same(case.kp[at, :, 6], before[at, :, 6])


def test_on_another_stream():
    case = Case([30], [100], 8, 2, 128, seed=9)
    k = torch.randn(30, 2, 128, device="cuda").to(BF)
    cache = cs.PagedCache(case.kp, case.vp)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        case.q = cache.cs_paged_append(k, k, *case.blocks(), q=case.q)
        out, lse = cache.cs_paged_attention(case.q, *case.blocks(), with_lse=True)
        assert cache.cs_paged_status() == cs.CS_OK
    torch.cuda.current_stream().wait_stream(side)
    case.k[0][100:], case.v[0][100:] = k, k
    from paged_helpers import check_attention
    check_attention(case, out, lse, *case.attention())


def test_without_the_native_side(monkeypatch):
    """The calls' general path, which stands in where the native module does not load, gives the same bits."""
    case = Case([4, 60], [30, 130], 8, 2, 64, seed=16)
    qkv = torch.randn(case.rows, 12, 64, device="cuda").to(BF)
    rope, pos, (qg, kg) = cs.cs_rope_table(200, 64), torch.arange(case.rows, device="cuda", dtype=torch.int32), gains(64, BF)
    got = []
    for native in (True, False):
        if not native:
            monkeypatch.setattr(cs, "_native", None)
        cache = cs.PagedCache(case.kp, case.vp)
        q = cache.cs_paged_append(qkv[:, 8:10], qkv[:, 10:], *case.blocks(), rope, kg, q=qkv[:, :8], q_gain=qg)
        out, lse = cache.cs_paged_attention(q, *case.blocks(), with_lse=True)
        got.append([q, out, lse, case.kp.clone(), *cs.cs_qk_norm_rope(qkv[:, :8], qkv[:, 8:10], pos, rope, qg, kg), cs.cs_qk_norm_rope(None, qkv[:, 8:10].float(), pos, rope, None, kg, dtype=BF)[1]])
        assert cache.cs_paged_append(qkv[:, 8:10], qkv[:, 10:], *case.blocks()) is None and cache.cs_paged_status() == cs.CS_OK
    for a, b in zip(*got):
        assert torch.equal(a.view(torch.int16) if a.dtype is BF else a, b.view(torch.int16) if b.dtype is BF else b)


def test_refusals():
    case = Case([2], [20], 4, 2, 64, seed=1)
    cache = cs.PagedCache(case.kp, case.vp)
    k, q = torch.zeros(2, 2, 64, dtype=BF, device="cuda"), torch.zeros(2, 4, 64, dtype=BF, device="cuda")
    rope = cs.cs_rope_table(30, 64)

    def code(call):
        with pytest.raises((cs.CsError, ValueError)) as e:
            call()
        return e.value.code if isinstance(e.value, cs.CsError) else "value"

    app = lambda k=k, v=k, **kw: code(lambda: cache.cs_paged_append(k, v, *case.blocks(), **kw))
    assert app(k.to(FP), k.to(FP)) == cs.CS_ERR_ARG                    # neither the cache's type nor 32 bits
    assert app(k[:, :1], k[:, :1]) == cs.CS_ERR_SHAPE
    assert app(rope=rope[:, :24].contiguous()) == cs.CS_ERR_SHAPE and app(rope=cs.cs_rope_table(30, 128)) == cs.CS_ERR_SHAPE
    assert app(eps=-1.0) == cs.CS_ERR_ARG and app(eps=math.nan) == cs.CS_ERR_ARG
    off = torch.zeros(2 * 2 * 64 + 4, dtype=BF, device="cuda")[4:].view(2, 2, 64)
    assert app(off, k) == cs.CS_ERR_ARG and app(k, off) == cs.CS_ERR_ARG
    assert app(k, k.float()) == "value" and app(q=q.float()) == "value" and app(q=q, q_out=q.float()) == "value" and app(k_gain=torch.ones(64, device="cuda")) == "value"
    assert app(rope=rope.double()) == "value"
    nr = lambda *a, **kw: code(lambda: cs.cs_qk_norm_rope(*a, **kw))
    pos = i32([0, 1])
    assert nr(q, k, pos, rope, dtype=FP) == cs.CS_ERR_ARG and nr(q[..., :40], None, pos, rope) == cs.CS_ERR_SHAPE
    assert nr(q, k.float(), pos, rope) == "value" and nr(q, k, pos[:1], rope) == "value" and nr(None, None, pos, rope) == "value" and nr(q.cpu(), None, pos, rope) == "value"
    for make in (lambda: cs.PagedCache(torch.zeros(4, 2, 24, 64, dtype=BF, device="cuda"), torch.zeros(4, 2, 24, 64, dtype=BF, device="cuda")),
                 lambda: cs.PagedCache(torch.zeros(4, 2, 16, 48, dtype=BF, device="cuda"), torch.zeros(4, 2, 16, 48, dtype=BF, device="cuda"))):
        assert code(make) == cs.CS_ERR_SHAPE
    assert code(lambda: cs.PagedCache(case.kp, case.vp.float())) == "value" and code(lambda: cs.PagedCache(case.kp, case.vp.transpose(1, 2))) == "value"
    assert cache.cs_paged_status() == cs.CS_OK
    other = cs.PagedCache(case.vp, case.kp, workspace=cache)            # a second layer's, same workspace
    other.cs_paged_append(k, k, *case.blocks())
    assert other.cs_paged_status() == cs.CS_OK
