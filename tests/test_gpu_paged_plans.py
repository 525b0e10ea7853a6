"""How the attention over pages deals its work out, where the other tests do not come by: many sequences some of which have many row groups, more KV heads than a warp has
lanes, tens of thousands of keys, prompts' chunks beside single tokens; and that the kernel for few rows is as exact as its two terms of every weight."""
import pytest
import torch

from paper_2502_08923_b200 import binding as cs
from paged_helpers import U, Case, check_attention

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16


def run(case, **kw):
    cache = cs.PagedCache(case.kp, case.vp)
    out, lse = cache.cs_paged_attention(case.q, *case.blocks(), with_lse=True, **kw)
    assert cache.cs_paged_status() == cs.CS_OK
    check_attention(case, out, lse, *case.attention(kw.get("mask", cs.MASK_CAUSAL), kw.get("window", 0)))
    return out, lse


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("n", [33, 100, 520])
@pytest.mark.parametrize("window", [0, 40])
def test_many_sequences_with_many_row_groups(D, n, window):
    g = torch.Generator().manual_seed(n)
    cached = torch.randint(0, 150, (n,), generator=g).tolist()
    # every thirteenth has 9 to 60 rows: up to 15 groups of 16 query rows; the average leaves them to the kernel for few rows
    lens = [9 + (7 * b) % 52 if b % 13 == 0 else b % 2 for b in range(n)]
    case = Case(lens, cached, 8, 2, D, seed=n)
    assert case.rows * 4 <= 16 * n
    run(case, window=window)
    # 64 heads of one KV head: items of four rows, blocks of up to eight items; on the tensor cores
    lens = [(5 * b) % 31 for b in range(min(n, 100))]
    case = Case(lens, cached[:len(lens)], 64, 1, D, seed=n)
    assert case.rows * 64 > 16 * len(lens)
    run(case, window=window)


@pytest.mark.parametrize("D,dtype", [(32, BF), (64, FP), (128, BF)])
@pytest.mark.parametrize("Hkv", [33, 40, 70])
@pytest.mark.parametrize("lens,cached", [([1, 2, 1], [300, 0, 130]), ([60, 1, 200], [300, 40, 70])])
def test_many_kv_heads(D, dtype, Hkv, lens, cached):
    run(Case(lens, cached, 2 * Hkv, Hkv, D, dtype, layout="token", seed=Hkv))


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("lens,cached", [([1], [60000]), ([1, 1, 1], [131071, 5, 40000]), ([30], [50000]), ([300, 1], [33000, 70000])])
def test_long_contexts(D, lens, cached):
    run(Case(lens, cached, 2, 1, D, page=256, seed=len(lens)))


@pytest.mark.parametrize("lens", [[1], [4], [100]])
@pytest.mark.parametrize("append", [False, True])
def test_positions_next_to_2_to_the_31(lens, append):
    """The last positions that a call takes, behind a window: every page of the table is the same one."""
    page, n, window = 1 << 20, lens[0], 300
    last = 0x7fffff00
    kp, vp = (torch.randn(1, 1, page, 32, device="cuda").to(BF) for _ in range(2))
    table = torch.zeros(1, -(-last // page), dtype=torch.int32, device="cuda")
    q, new = (torch.randn(n, h, 32, device="cuda").to(BF) for h in (4, 1))
    blocks = (torch.zeros(1, dtype=torch.int32, device="cuda"), *(torch.tensor([x], dtype=torch.int32, device="cuda") for x in (n, last - n)), table)
    cache = cs.PagedCache(kp, vp)
    at = [(last - n + r) % page for r in range(n)]
    if append:
        cache.cs_paged_append(new, -new, *blocks)
        assert torch.equal(kp[0, 0, at], new[:, 0]) and torch.equal(vp[0, 0, at], -new[:, 0])
    out, lse = cache.cs_paged_attention(q, *blocks, window=window, with_lse=True)
    assert cache.cs_paged_status() == cs.CS_OK
    for r in range(n):
        keys = torch.arange(last - n + r + 1 - window, last - n + r + 1, device="cuda") % page
        k, v = kp[0, 0, keys].double(), vp[0, 0, keys].double()
        x = q[r].double() @ k.T * 32 ** -0.5
        w = torch.softmax(x, dim=1)
        want, size = w @ v, w @ v.abs()
        u = U[BF]
        assert bool(((out[r].double() - want).abs() <= u * want.abs() * (1 + u) + (u + 1e-4) * size + 2.0 ** -24).all())
        assert float((lse[r].double() - torch.logsumexp(x, dim=1)).abs().max()) <= 1e-4


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,cached", [([200] + [1] * 150, [900] + [70] * 150), ([1] * 60 + [700], [40] * 60 + [100])])
def test_a_chunk_beside_single_tokens(D, lens, cached):
    run(Case(lens, cached, 8, 2, D, page=32, seed=7))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("lens,cached", [([1] * 40, [15] * 40), ([3] * 20, [40] * 20), ([1], [700])])
def test_few_rows_are_as_exact_as_their_scores(dtype, D, lens, cached):
    """Weights w go into the product as hi + lo, each rounded to u: what is left of w is u^2 / 4, below 2^-17.  So beside the result's own rounding there are only the scores' errors and that, together below
    1e-4 of the sum of sizes (one term would leave u / 2 of each weight).  Values of either sign, so that results are small beside that sum."""
    case = Case(lens, cached, 8, 2, D, dtype, seed=3)
    for b in range(len(lens)):
        case.v[b] = torch.where(case.v[b] > 0, 1.0, -1.0).to(dtype)
        case.put(b)
    assert case.rows * 4 <= 16 * len(lens)
    cache = cs.PagedCache(case.kp, case.vp)
    out = cache.cs_paged_attention(case.q, *case.blocks()).double()
    want, _, size = case.attention()
    u = U[dtype]
    assert bool(((out - want).abs() <= u * want.abs() * (1 + u) + 1e-4 * size + 2.0 ** -24).all())
