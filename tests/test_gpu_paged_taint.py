"""Values that are not finite in the cache, at positions that some rows of a block attend to and others of the same work item do not, behind long
contexts: rows that do not see them are right, rows that do are not finite where the formula is not, and no wait runs out."""
import math

import pytest
import torch

from paper_2502_08923_b200 import binding as cs
from paged_helpers import U, Case, check_attention

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16


def check(case, out, lse, want, want_lse, size):
    """check_attention where the definition is finite, not finite where it is not."""
    odd, odd_lse = ~torch.isfinite(want), torch.isnan(want_lse)
    assert not bool(torch.isfinite(out.float())[odd].any()) and bool(torch.isnan(lse)[odd_lse].all())
    check_attention(case, out.float().masked_fill(odd, 0.0), lse.masked_fill(odd_lse, 0.0), want.masked_fill(odd, 0.0), want_lse.masked_fill(odd_lse, 0.0),
                    size.masked_fill(odd, 0.0))


@pytest.mark.parametrize("D,dtype", [(32, BF), (64, FP), (128, BF), (128, FP)])
@pytest.mark.parametrize("mask,window", [(cs.MASK_CAUSAL, 0), (cs.MASK_CAUSAL, 60), (cs.MASK_CAUSAL, 700), (cs.MASK_PREFIX, 333), (cs.MASK_FULL, 90)])
@pytest.mark.parametrize("H,Hkv,page", [(8, 2, 16), (6, 2, 128), (3, 3, 64), (40, 2, 32)])
def test_many_bad_values(D, dtype, mask, window, H, Hkv, page):
    case = Case([150, 1, 33, 260], [1400, 700, 0, 90], H, Hkv, D, dtype, page=page, layout="token" if H == 6 else "head", seed=window + H)
    g = torch.Generator().manual_seed(window + D)
    for b, (n, c) in enumerate(zip(case.lens, case.cached)):
        for _ in range(12):                              # single elements, whole values, keys with them
            at, h, d = (int(torch.randint(0, m, (1,), generator=g)) for m in (n + c, Hkv, D))
            bad = (math.nan, math.inf, -math.inf)[int(torch.randint(0, 3, (1,), generator=g))]
            kind = int(torch.randint(0, 3, (1,), generator=g))
            case.v[b][at, h, d if kind == 0 else slice(None)] = bad
            if kind == 2 and mask != cs.MASK_FULL:
                case.k[b][max(at, c), h, d] = math.nan
        case.put(b)
    cache = cs.PagedCache(case.kp, case.vp)
    out, lse = cache.cs_paged_attention(case.q, *case.blocks(), mask=mask, window=window, with_lse=True)
    assert cache.cs_paged_status() == cs.CS_OK
    check(case, out, lse, *case.attention(mask, window))
    again = cache.cs_paged_attention(case.q, *case.blocks(), mask=mask, window=window, with_lse=True)
    assert torch.equal(out.view(torch.int16), again[0].view(torch.int16)) and torch.equal(lse.view(torch.int32), again[1].view(torch.int32))


@pytest.mark.parametrize("whole", [True, False])
@pytest.mark.parametrize("D", [64, 128])
def test_a_long_context(D, whole):
    """One value of one token of a 2,048-row chunk behind 30,720 keys, NaN in all heads.  `whole`: items that no two CTAs share - 37 chunks of 64 tokens, four KV heads, an equal run of tiles each."""
    H, Hkv, bad = 32, 8, 777
    case = Case([2048], [30720], H, Hkv, D, page=64, seed=D)
    lens, cached = case.lens, case.cached
    if whole:
        lens, cached, bad = [64] * 37, [2496] * 37, 30
        case = Case(lens, cached, 16, 4, D, page=64, seed=D)
        H, Hkv = 16, 4
    cache = cs.PagedCache(case.kp, case.vp)
    clean = cache.cs_paged_attention(case.q, *case.blocks(), with_lse=True)
    for b in range(len(lens)):
        at, slot = divmod(cached[b] + bad, 64)
        case.vp[case.table[b, at].long(), :, slot] = math.nan
    out, lse = cache.cs_paged_attention(case.q, *case.blocks(), with_lse=True)
    assert cache.cs_paged_status() == cs.CS_OK
    assert torch.equal(lse, clean[1]) or float((lse - clean[1]).abs().max()) <= 2e-4
    u, scale = U[BF], D ** -0.5
    for b in range(len(lens)):
        s = case.starts[b]
        assert bool(torch.isfinite(out[s:s + bad].float()).all()) and bool(torch.isnan(out[s + bad:s + lens[b]].float()).all())
        first = (bad // 64) * 64                         # items of 256 query rows: tokens of others are as they were
        assert torch.equal(out[s:s + first], clean[0][s:s + first])
        for r in (first, first + 1, bad - 1) if b in (0, len(lens) - 1) else ():
            n = cached[b] + r + 1
            for h in range(Hkv):
                k, v, q = case.k[b][:n, h].double(), case.v[b][:n, h].double(), case.q[s + r, h * 4:h * 4 + 4].double()
                x = (q @ k.T) * scale
                w = torch.softmax(x, dim=1)
                want, size = w @ v, w @ v.abs()
                assert bool(((out[s + r, h * 4:h * 4 + 4].double() - want).abs() <= u * want.abs() * (1 + u) + (u + 1e-4) * size + 2.0 ** -24).all())
                assert float((lse[s + r, h * 4:h * 4 + 4].double() - torch.logsumexp(x, dim=1)).abs().max()) <= 1e-4
