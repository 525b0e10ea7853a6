"""Many softmax weights far below the largest one: by themselves next to nothing, together a share of the result that its type can hold.  One key 17.5 nats above tens of thousands, whose
values are 1 where its own is 0: the result is their share, some 10^-3."""
import pytest
import torch

from paper_2502_08923_b200 import binding as cs
from paged_helpers import Case, check_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("lens,cached", [([1], 30719), ([1], 131071), ([3, 2], 30719), ([40], 30719), ([70], 131071)])
@pytest.mark.parametrize("at", ["first", "middle", "last"])
def test_share_of_the_small_ones(dtype, D, lens, cached, at):
    case = Case(lens, [cached] * len(lens), 4, 1, D, dtype, page=128, seed=1)
    case.q.zero_()
    case.q[..., 0] = 1.0                                  # scores are the keys' first elements, exactly
    for b, n in enumerate(lens):
        case.k[b].zero_()
        case.v[b].fill_(1.0)
        where = {"first": 0, "middle": cached // 2, "last": cached - 1}[at]
        case.k[b][where, :, 0] = 17.5
        case.v[b][where] = 0.0
        case.put(b)
    cache = cs.PagedCache(case.kp, case.vp)
    out, lse = cache.cs_paged_attention(case.q, *case.blocks(), scale=1.0, with_lse=True)
    assert cache.cs_paged_status() == cs.CS_OK
    want = case.attention(scale=1.0)
    assert 5e-4 < float(want[0].min()) and float(want[0].max()) < 5e-3
    check_attention(case, out, lse, *want)
