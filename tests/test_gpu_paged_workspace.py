"""Caches of several layers on one workspace, and two workspaces over one pair of pools."""
import pytest
import torch

from paper_2502_08923_b200 import binding as cs
from paged_helpers import Case, check_attention, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens", [[1, 2], [50, 70]])
def test_a_further_layer_keeps_what_the_first_has_to_report(lens):
    case = Case(lens, [200, 90], 8, 2, 128, seed=1)
    first = cs.PagedCache(case.kp, case.vp)
    length = i32([lens[0], -1])
    first.cs_paged_attention(case.q, case.start, length, case.kv_len, case.table)
    second = cs.PagedCache(case.kp.clone(), case.vp.clone(), workspace=first)
    assert second.cs_paged_status() == cs.CS_ERR_ARG and first.cs_paged_status() == cs.CS_OK
    check_attention(case, *second.cs_paged_attention(case.q, *case.blocks(), with_lse=True), *case.attention())
    first.close()
    check_attention(case, *second.cs_paged_attention(case.q, *case.blocks(), with_lse=True), *case.attention())
    third = cs.PagedCache(case.kp, case.vp, workspace=second)
    check_attention(case, *third.cs_paged_attention(case.q, *case.blocks(), with_lse=True), *case.attention())
    assert third.cs_paged_status() == cs.CS_OK
    with pytest.raises(cs.CsError) as e:
        cs.PagedCache(case.kp, case.vp, workspace=first)
    assert e.value.code == cs.CS_ERR_ARG                  # it has been closed


def test_heads_that_the_workspace_is_too_small_for():
    small, large = Case([1], [20], 4, 2, 64), Case([1], [20], 4, 2, 128)
    cache = cs.PagedCache(small.kp, small.vp)
    with pytest.raises(cs.CsError) as e:
        cs.PagedCache(large.kp, large.vp, workspace=cache)
    assert e.value.code == cs.CS_ERR_CAPACITY and "cs_paged_create_beside" in str(e.value)


def test_two_streams_have_a_workspace_each():
    """Prompts' chunks on one stream, single tokens of other sequences on another, over the same pools."""
    case = Case([150, 1, 90, 1, 1], [3000, 4000, 2000, 500, 2500], 8, 2, 128, seed=2)
    want = case.attention()
    lens = [i32([n if tall == (n > 1) else 0 for n in case.lens]) for tall in (True, False)]
    caches = [cs.PagedCache(case.kp, case.vp) for _ in lens]
    torch.cuda.synchronize()
    out, lse = torch.full_like(case.q, 7.0), torch.full(case.q.shape[:2], 7.0, device="cuda")
    streams = [torch.cuda.Stream() for _ in lens]
    torch.cuda.synchronize()
    for _ in range(20):
        for cache, length, stream in zip(caches, lens, streams):
            with torch.cuda.stream(stream):
                cache.cs_paged_attention(case.q, case.start, length, case.kv_len, case.table, out=out, lse=lse)
    torch.cuda.synchronize()
    assert all(c.cs_paged_status() == cs.CS_OK for c in caches)
    check_attention(case, out, lse, *want)
