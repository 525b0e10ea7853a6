"""Attention of blocks over a paged KV cache against softmax(scale q k^T) v in 64 bits: head sizes, group sizes, types, page sizes and
layouts, block heights from none to a prompt's chunk, lengths around tiles and pages, masks and windows that leave rows without a key."""
import math

import pytest
import torch

from paper_2502_08923_b200 import binding as cs
from paged_helpers import Case, check_attention, i32

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16


def run(case, cache=None, **kw):
    cache = cache or cs.PagedCache(case.kp, case.vp)
    out, lse = cache.cs_paged_attention(case.q, *case.blocks(), with_lse=True, **kw)
    assert cache.cs_paged_status() == cs.CS_OK
    want = case.attention(kw.get("mask", cs.MASK_CAUSAL), kw.get("window", 0), kw.get("scale"))
    check_attention(case, out, lse, *want)
    return out, lse


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("lens,cached", [([1], [0]), ([1], [1]), ([1], [15]), ([1], [16]), ([1], [127]), ([1], [128]), ([1], [129]), ([1], [1000]),
                                         ([11], [0]), ([11], [512]), ([2, 1, 11, 0, 5], [300, 1, 117, 40, 0]), ([21, 33], [1531, 95]), ([70], [190]), ([150, 3], [0, 700])])
def test_lengths(D, dtype, lens, cached):
    run(Case(lens, cached, 8, 2, D, dtype, seed=len(lens) + sum(cached)))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,Hkv", [(1, 1), (8, 8), (3, 1), (6, 2), (7, 1), (20, 4), (16, 1), (17, 1), (40, 1), (128, 1)])
def test_groups(D, H, Hkv):
    for lens, cached in (([1, 1], [200, 33]), ([9, 2], [100, 260]), ([45], [77])):
        run(Case(lens, cached, H, Hkv, D, seed=H))


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256, 1024])
@pytest.mark.parametrize("layout", ["head", "token"])
def test_pages(D, page, layout):
    run(Case([1, 11, 60], [page - 1, 3 * page + 5, 17], 8, 2, D, page=page, layout=layout, seed=page))


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("mask", [cs.MASK_CAUSAL, cs.MASK_PREFIX, cs.MASK_FULL])
@pytest.mark.parametrize("window", [0, 1, 2, 16, 100, 129, 5000])
def test_masks(D, mask, window):
    for lens, cached in (([1, 1], [0, 400]), ([12, 3], [0, 257]), ([130, 40], [140, 0])):
        run(Case(lens, cached, 4, 2, D, seed=window), mask=mask, window=window)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,cached", [([300], [700]), ([512, 257], [0, 1300]), ([1, 400, 1, 1, 33], [900, 128, 5, 2000, 640])])
@pytest.mark.parametrize("mask,window", [(cs.MASK_CAUSAL, 0), (cs.MASK_CAUSAL, 150), (cs.MASK_FULL, 0), (cs.MASK_PREFIX, 300)])
def test_chunks(D, lens, cached, mask, window):
    run(Case(lens, cached, 8, 2, D, FP if D == 64 else BF, page=32, seed=sum(lens)), mask=mask, window=window)


@pytest.mark.parametrize("scale", [1e-3, 0.5, 1.0])
@pytest.mark.parametrize("lens,cached", [([1, 1], [300, 50]), ([40], [200])])
def test_scale(scale, lens, cached):
    case = Case(lens, cached, 8, 2, 128, seed=3)
    case.q = (case.q.float() / (8.0 * scale)).clamp(-3e4, 3e4).to(BF) if scale >= 0.5 else case.q
    run(case, scale=scale)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,cached", [([1], [5000]), ([30], [3000]), ([260], [2000])])
def test_scores_that_rise(D, lens, cached):
    """Every tile's scores beat those before it: the running maximum moves all the time, by far more than weights can hold."""
    case = Case(lens, cached, 4, 1, D, seed=9)
    case.q = torch.ones_like(case.q)
    n = lens[0] + cached[0]
    step = torch.linspace(-40.0, 40.0, n, device="cuda")[:, None, None] * D ** -0.5
    case.k[0] = (step + 0.01 * torch.randn(n, 1, D, device="cuda")).to(BF)
    case.put(0)
    run(case)
    case.k[0] = case.k[0].flip(0)
    case.put(0)
    run(case)


def test_rows_of_projections():
    """Queries as a view of wider rows, and rows that no block has, which stay as they are."""
    case = Case([3, 20, 1], [40, 100, 250], 8, 2, 128, seed=5, gaps=2)
    wide = torch.randn(case.rows, 12 * 128, device="cuda").to(BF)
    case.q = wide[:, 2 * 128:10 * 128].unflatten(1, (8, 128))
    cache = cs.PagedCache(case.kp, case.vp)
    out, lse = torch.full((case.rows, 8, 128), 7.0, dtype=BF, device="cuda"), torch.full((case.rows, 8), 7.0, device="cuda")
    got = cache.cs_paged_attention(case.q, *case.blocks(), out=out, lse=lse)
    assert got[0] is out and got[1] is lse and cache.cs_paged_status() == cs.CS_OK
    check_attention(case, out, lse, *case.attention())
    for s, n in zip(case.starts, case.lens):
        assert bool((out[s + n:s + n + 2] == 7.0).all()) and bool((lse[s + n:s + n + 2] == 7.0).all())
    only = cache.cs_paged_attention(case.q, *case.blocks())
    assert torch.equal(only[:3], out[:3])


@pytest.mark.parametrize("lens", [[1], [3], [90]])
def test_one_page_one_head_one_row_repeated(lens):
    """Strides that nothing uses may be anything, and queries may be one row for all."""
    case = Case(lens, [100], 4, 1, 64, page=256, seed=7, spare=0)
    assert case.kp.shape[:2] == (1, 1)
    strange = [torch.as_strided(p, p.shape, (3, 5, p.stride(2), 1)) for p in (case.kp, case.vp)]
    run(case, cs.PagedCache(*strange))
    case.q = case.q[:1].expand(case.rows, 4, 64)
    run(case, cs.PagedCache(*strange))
    case.q = case.q[:, :1].expand(case.rows, 4, 64)
    run(case, cs.PagedCache(*strange))


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("lens", [[11], [150]])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_values_that_are_not_finite_reach_only_rows_that_see_them(D, lens, bad):
    case = Case(lens, [100], 4, 2, D, seed=11)
    at = 100 + lens[0] - 4                               # a position inside the block: rows before it must not notice
    case.k[0][at], case.v[0][at] = bad, bad
    case.v[0][at - 1, 0, 3] = bad
    case.put(0)
    cache = cs.PagedCache(case.kp, case.vp)
    out, lse = cache.cs_paged_attention(case.q, *case.blocks(), with_lse=True)
    assert cache.cs_paged_status() == cs.CS_OK
    want, want_lse, size = case.attention()
    first = lens[0] - 5                                  # the first row that sees a value that is not finite
    assert bool(torch.isfinite(out[:first].float()).all())
    case.lens = [first]
    check_attention(case, out, lse, want, want_lse, size)
    row = out[first].float()                             # it sees V[at - 1][head 0][3], and a key of its own
    assert not torch.isfinite(row[:2, 3]).any() and torch.isfinite(row[2:]).all() and torch.isfinite(torch.cat([row[:2, :3], row[:2, 4:]], 1)).all()


@pytest.mark.parametrize("D", [32, 128])
def test_nan_keys_make_nan_rows(D):
    case = Case([1, 1], [50, 60], 4, 2, D, seed=2)
    case.k[0][7, 0, 5] = math.nan
    case.put(0)
    out, lse = cs.PagedCache(case.kp, case.vp).cs_paged_attention(case.q, *case.blocks(), with_lse=True)
    assert torch.isnan(out[0, :2].float()).all() and torch.isnan(lse[0, :2]).all() and torch.isfinite(out[0, 2:].float()).all() and torch.isfinite(out[1].float()).all()


@pytest.mark.parametrize("lens", [[1], [40]])
def test_pages_behind_the_window_may_be_gone(lens):
    case = Case(lens, [1000], 8, 2, 128, page=16, seed=4)
    want = case.attention(window=100)
    gone = (1000 + 1 - 100) // 16                        # pages wholly to the left of every row's window
    case.kp[case.table[0, :gone].long()] = math.nan
    case.vp[case.table[0, :gone].long()] = math.nan
    case.table[0, :gone] = 1 << 30
    cache = cs.PagedCache(case.kp, case.vp)
    out, lse = cache.cs_paged_attention(case.q, *case.blocks(), window=100, with_lse=True)
    assert cache.cs_paged_status() == cs.CS_OK
    check_attention(case, out, lse, *want)


def test_many_sequences():
    """More than one launch's plan holds."""
    n = 1100
    case = Case([1 + b % 3 for b in range(n)], [(b * 37) % 90 for b in range(n)], 2, 1, 64, seed=8)
    run(case)


def test_offsets_beyond_32_bits():
    """Pages whose elements lie beyond 2^31 of the pool."""
    n_pages = (1 << 31) // (16 * 8 * 128) + 200
    for lens in ([1, 2], [130]):
        run(Case(lens, [300] * len(lens), 8, 8, 128, seed=6, first_page=n_pages - 150, n_pages=n_pages))


@pytest.mark.parametrize("lens", [[1] * 5, [30, 200]])
def test_reproducible_and_on_another_stream(lens):
    case = Case(lens, [700 + 90 * b for b in range(len(lens))], 8, 2, 128, seed=13)
    cache = cs.PagedCache(case.kp, case.vp)
    first = cache.cs_paged_attention(case.q, *case.blocks(), with_lse=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(20):
            again = cache.cs_paged_attention(case.q, *case.blocks(), with_lse=True)
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
        assert cache.cs_paged_status() == cs.CS_OK
    torch.cuda.current_stream().wait_stream(side)


@pytest.mark.parametrize("lens", [[1, 1], [40, 100]])
def test_captured_in_a_graph(lens):
    """Lengths and pages are read on the device when the call runs."""
    case = Case(lens, [200, 330], 8, 2, 128, seed=14)
    cache = cs.PagedCache(case.kp, case.vp)
    out, lse = cache.cs_paged_attention(case.q, *case.blocks(), with_lse=True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.cs_paged_attention(case.q, *case.blocks(), out=out, lse=lse)
    for cached in ([199, 12], [60, 330]):
        case.cached = cached
        case.kv_len.copy_(i32(cached))
        graph.replay()
        check_attention(case, out, lse, *case.attention())
    assert cache.cs_paged_status() == cs.CS_OK


def test_sequences_that_do_not_fit_are_left_out():
    for lens in ([4, 1, 2, 3, 1], [64, 60, 70, 61, 40]):
        case = Case(lens, [50, 60, 70, 80, 90], 4, 2, 64, seed=15)
        cache = cs.PagedCache(case.kp, case.vp)
        want = case.attention()
        for field, b, value, code in (("kv_len", 1, case.table.shape[1] * 16 - lens[1] + 1, cs.CS_ERR_CAPACITY), ("kv_len", 2, -1, cs.CS_ERR_ARG), ("len", 3, -1, cs.CS_ERR_ARG),
                                      ("start", 4, case.rows, cs.CS_ERR_ARG), ("start", 0, -1, cs.CS_ERR_ARG), ("kv_len", 3, 2 ** 31 - 1, cs.CS_ERR_CAPACITY)):
            t = getattr(case, field)
            old = int(t[b])
            t[b] = value
            out, lse = torch.full_like(case.q, 7.0), torch.full((case.rows, 4), 7.0, device="cuda")
            cache.cs_paged_attention(case.q, *case.blocks(), out=out, lse=lse)
            assert cache.cs_paged_status() == code and cache.cs_paged_status() == cs.CS_OK
            t[b] = old
            s = slice(case.starts[b], case.starts[b] + lens[b])
            assert bool((out[s] == 7.0).all()) and bool((lse[s] == 7.0).all())
            rest = want[0].clone(), want[1].clone(), want[2].clone()
            keep, case.lens = case.lens, [0 if i == b else n for i, n in enumerate(case.lens)]
            check_attention(case, out, lse, *rest)
            case.lens = keep


@pytest.mark.parametrize("lens", [[2, 1], [80, 70]])
@pytest.mark.parametrize("page", [-1, 10 ** 6])
def test_a_page_that_does_not_exist_is_reported(lens, page):
    case = Case(lens, [100, 100], 4, 2, 128, seed=16)
    case.table[0, 3] = page
    cache = cs.PagedCache(case.kp, case.vp)
    out, lse = cache.cs_paged_attention(case.q, *case.blocks(), with_lse=True)
    assert cache.cs_paged_status() == cs.CS_ERR_ARG
    case.k[0][48:64], case.v[0][48:64] = 0.0, 0.0        # its keys and values are taken for zeros
    check_attention(case, out, lse, *case.attention())


def test_nothing_to_do():
    case = Case([0, 0], [10, 0], 4, 2, 64, seed=1)
    cache = cs.PagedCache(case.kp, case.vp)
    assert cache.cs_paged_attention(case.q, *case.blocks()).shape == (0, 4, 64)
    q = torch.randn(3, 4, 64, device="cuda").to(BF)
    out = torch.full_like(q, 7.0)
    cache.cs_paged_attention(q, *case.blocks(), out=out)
    none = i32([])
    cache.cs_paged_attention(q, none, none, none, case.table[:0], out=out)
    assert bool((out == 7.0).all()) and cache.cs_paged_status() == cs.CS_OK


def test_refusals():
    case = Case([2], [20], 4, 2, 64, seed=1)
    cache = cs.PagedCache(case.kp, case.vp)

    def code(q=case.q, **kw):
        with pytest.raises((cs.CsError, ValueError)) as e:
            cache.cs_paged_attention(q, *case.blocks(), **kw)
        return e.value.code if isinstance(e.value, cs.CsError) else "value"

    assert code(mask=3) == cs.CS_ERR_ARG and code(mask=-1) == cs.CS_ERR_ARG and code(window=-1) == cs.CS_ERR_ARG
    assert code(scale=0.0) == cs.CS_ERR_ARG and code(scale=-1.0) == cs.CS_ERR_ARG and code(scale=math.nan) == cs.CS_ERR_ARG and code(scale=math.inf) == cs.CS_ERR_ARG
    assert code(torch.zeros(2, 3, 64, dtype=BF, device="cuda")) == cs.CS_ERR_SHAPE        # heads: no multiple
    assert code(torch.zeros(2, 512, 64, dtype=BF, device="cuda")) == cs.CS_ERR_SHAPE      # 256 per KV head
    assert code(torch.zeros(2 * 4 * 64 + 4, dtype=BF, device="cuda")[4:].view(2, 4, 64)) == cs.CS_ERR_ARG       # 8 bytes off
    assert code(torch.zeros(2, 4, 68, dtype=BF, device="cuda")[..., :64]) == cs.CS_ERR_ARG                        # strides of 136 bytes
    assert code(case.q.to(FP)) == "value" and code(case.q[..., :32]) == "value" and code(case.q.cpu()) == "value"
    assert code(out=torch.zeros(2, 4, 64, device="cuda")) == "value" and code(lse=torch.zeros(2, 3, device="cuda")) == "value"
    assert cache.cs_paged_status() == cs.CS_OK
