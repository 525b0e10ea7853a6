"""Attention over the paged cache of 4 bits against a plain implementation in 64 bits over the values that the cache stands for."""
import math

import pytest
import torch

from paper_2502_08923_b200 import binding as cs
from quant_helpers import QuantCase, check_attention, i32, is_tall

pytestmark = pytest.mark.gpu


def run(case, mask=cs.MASK_CAUSAL, window=0, scale=None):
    got, lse = case.cache.cs_quant_attention(case.q, *case.blocks(), mask=mask, window=window, scale=scale, with_lse=True)
    assert case.cache.cs_quant_status() == cs.CS_OK
    check_attention(case, got, lse, *case.attention(mask, window, scale), tall=is_tall(case, window))
    return got, lse


# few query rows: every number of row tiles, heads, pages, blocks that end inside pages and tiles
@pytest.mark.parametrize("lens,cached,H,Hkv,D,page", [
    ([1], [0], 1, 1, 128, 16), ([1], [1], 4, 1, 64, 16), ([1], [511], 32, 8, 128, 16), ([1], [5000], 32, 8, 128, 64), ([1] * 5, [0, 15, 16, 129, 700], 32, 8, 64, 32), ([1] * 3, [40, 1000, 2], 8, 8, 32, 16),
    ([2], [300], 32, 8, 128, 16), ([3, 4], [100, 999], 16, 4, 64, 16), ([11], [512], 8, 8, 32, 16), ([11], [4096], 32, 8, 128, 16), ([5, 1, 0, 9], [33, 2000, 7, 0], 32, 8, 128, 128), ([21, 20], [900, 1500], 32, 8, 64, 32),
    ([6], [260], 12, 2, 128, 16), ([13], [77], 5, 5, 128, 16), ([8], [64], 64, 8, 32, 64), ([40], [200], 16, 4, 64, 16), ([70], [10], 4, 2, 128, 16), ([3], [90], 128, 1, 64, 16)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_blocks(lens, cached, H, Hkv, D, page, dtype):
    run(QuantCase(lens, cached, H, Hkv, D, dtype, page=page, seed=len(lens), gaps=1))


@pytest.mark.parametrize("mask", [cs.MASK_CAUSAL, cs.MASK_PREFIX, cs.MASK_FULL])
@pytest.mark.parametrize("window", [0, 1, 5, 40, 300])
@pytest.mark.parametrize("D,lens,cached", [(128, [1, 5, 2, 7], [0, 0, 333, 129]), (64, [9, 1, 30], [20, 515, 0]), (32, [3, 17], [0, 260])])
def test_masks(mask, window, D, lens, cached):
    """Rows that no key is left for, and ranges that begin and end inside a slice."""
    run(QuantCase(lens, cached, 8, 2, D, torch.bfloat16, seed=window), mask, window)


# tall blocks, with copies and without
@pytest.mark.parametrize("lens,cached,H,Hkv,D,page", [([200], [0], 8, 2, 128, 16), ([130, 64], [700, 129], 32, 8, 64, 32), ([257], [1000], 4, 4, 32, 64), ([500, 1, 90], [3, 2000, 130], 8, 2, 128, 128),
                                                    ([30, 25], [700, 129], 128, 1, 64, 32), ([700], [100], 4, 1, 128, 16), ([110, 1, 140], [0, 2000, 130], 64, 2, 32, 128)])      # (prompts' chunks by their rows per KV head)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("room", [True, False])
def test_tall_blocks(lens, cached, H, Hkv, D, page, dtype, room):
    wide = max(-(-(n + c) // page) for n, c in zip(lens, cached)) + 1
    need = len(lens) * wide * page
    for mask, window in ((cs.MASK_CAUSAL, 0), (cs.MASK_PREFIX, 0), (cs.MASK_CAUSAL, 100), (cs.MASK_FULL, 64)):
        case = QuantCase(lens, cached, H, Hkv, D, dtype, page=page, seed=3, tall=need if room else need - 16, gaps=3)
        assert is_tall(case)
        run(case, mask, window)


@pytest.mark.parametrize("D,page", [(128, 16), (64, 32), (32, 16), (128, 256)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_blocks_of_one_row_group(D, page, dtype):
    """Expanded by the kernel: slots that take tiles in turn and slots with rows of their own; long contexts, ends inside pages and tiles."""
    for lens, cached in (([20], [5000]), ([21, 17, 33], [130, 0, 1777]), ([64], [300]), ([17] * 9, [100 * i for i in range(9)]), ([1, 60], [4000, 10])):
        for mask, window in ((cs.MASK_CAUSAL, 0), (cs.MASK_FULL, 0), (cs.MASK_PREFIX, 0), (cs.MASK_CAUSAL, 200)):
            case = QuantCase(lens, cached, 32, 4, D, dtype, page=page, seed=5, gaps=1)
            assert is_tall(case)
            run(case, mask, window)


@pytest.mark.parametrize("D", [64, 128])
def test_between_few_and_tall(D):
    """Rows per KV head from 33 to 128: by the work, which goes by the room of the page table and by the window."""
    ways = set()
    for rows in (8, 9, 32):
        for cached in (100, 5000, 17000):
            for window in (0, 600):
                case = QuantCase([rows], [cached], 16, 4, D, torch.bfloat16, page=64, seed=rows)
                run(case, window=window)
                ways.add((rows * 4 > 32, is_tall(case, window)))
    assert ways == {(False, False), (True, False), (True, True)}


@pytest.mark.parametrize("room", [0, 1 << 12])
def test_no_rows_of_any_block(room):
    """A call of tall blocks' size in which no sequence has a row: everything stays as it was."""
    case = QuantCase([0, 0], [300, 0], 64, 2, 64, torch.bfloat16, seed=2, gaps=100, tall=room)
    assert is_tall(case)
    out, lse = torch.full_like(case.q, 9.0), torch.full((case.rows, 64), 9.0, device="cuda")
    for _ in range(2):
        case.cache.cs_quant_attention(case.q, *case.blocks(), out=out, lse=lse)
    assert case.cache.cs_quant_status() == cs.CS_OK and bool((out == 9.0).all()) and bool((lse == 9.0).all())


def test_repeated_queries():
    """Queries that repeat one row have no operand map: tall blocks of them take the way of short ones."""
    case = QuantCase([100, 60], [200, 30], 8, 2, 64, torch.bfloat16, seed=4)
    case.q = case.q[:1].expand(case.rows, 8, 64)
    assert not is_tall(case)
    run(case)
    case.q = case.q[:1, :1].expand(case.rows, 8, 64)
    run(case)


def test_values_beyond_fp16():
    """fp16 queries over values beyond 65504, which the tensor cores take for that in tall blocks, and over some so small that fp16 rounds them: each by 2^-25 at most, and so do their averages (the result's own rounding is as much)."""
    for size in (40000.0, 3e-6, 4e-8):
        case = QuantCase([30, 40], [100, 20], 8, 2, 64, torch.float16, seed=4)
        for b in range(2):
            case.v[b] = torch.randn(case.v[b].shape, device="cuda") * size
            case.k[b] = case.k[b].float()
            case.put(b)
            case.v[b] = case.v[b].clamp(-65504, 65504)
        got, lse = case.cache.cs_quant_attention(case.q, *case.blocks(), with_lse=True)
        assert is_tall(case) and case.cache.cs_quant_status() == cs.CS_OK
        check_attention(case, got, lse, *case.attention(), tall=True)


def test_scales_and_strides():
    case = QuantCase([4, 3], [100, 50], 8, 2, 64, torch.float16, seed=1)
    wide = torch.randn(case.rows, 3, 8, 64, device="cuda").to(torch.float16)
    for q in (wide[:, 1], wide[:, 2].transpose(0, 1).contiguous().transpose(0, 1), wide[:1, 0].expand(case.rows, 8, 64)):
        case.q = q
        run(case, scale=0.3)
    case.q = wide[:, 1]
    out, lse = torch.full((case.rows, 8, 64), 9.0, dtype=torch.float16, device="cuda"), torch.full((case.rows, 8), 9.0, device="cuda")
    case.cache.cs_quant_attention(case.q, case.start, i32([4, 0]), case.kv_len, case.table, out=out, lse=lse)
    assert bool((out[4:] == 9.0).all()) and bool((lse[4:] == 9.0).all()) and not bool((out[:4] == 9.0).any())


def test_sharp_and_flat_scores():
    """Scores far apart (reference points move often, and by much) and all the same."""
    for factor in (40.0, 0.0):
        case = QuantCase([1, 3, 9], [3000, 1500, 700], 32, 8, 128, torch.bfloat16, seed=2)
        case.q = (case.q.float() * factor).to(case.q.dtype)
        got, lse = case.cache.cs_quant_attention(case.q, *case.blocks(), with_lse=True)
        want, want_lse, size = case.attention()
        # (scores forty times as large are off forty times as far)
        assert float((lse.double() - want_lse)[case.live()].abs().max()) <= 1e-4 * max(1.0, factor)
        allowed = 2.0 ** -8 * want.abs() * 1.01 + (2.0 ** -16 + 2e-4 * max(1.0, factor)) * size + 2.0 ** -24
        assert bool(((got.double() - want).abs() <= allowed)[case.live()].all())


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("tall,room", [(False, 0), (True, 0), (True, 1 << 14)])
def test_what_is_not_finite(D, tall, room):
    """Keys and values that are NaN at positions that some rows see and others do not."""
    lens, cached = ([150, 140], [300, 40]) if tall else ([6, 3], [300, 40])
    case = QuantCase(lens, cached, 64 if room else 8, 2, D, torch.bfloat16, seed=5, tall=room)
    for name, rows, scales, at in (("v", case.v, case.vs, [(0, cached[0] + 2, 1, 0), (0, 7, 0, D // 32 - 1), (1, cached[1] + 1, 1, 0)]), ("k", case.k, case.ks, [(0, cached[0] + 4, 0, 0)])):
        for b, pos, head, group in at:
            scales[case.table[b, pos // case.page].long(), head, pos % case.page, group] = math.nan
            rows[b][pos, head, 32 * group:32 * group + 32] = math.nan
    got, lse = case.cache.cs_quant_attention(case.q, *case.blocks(), with_lse=True)
    want, want_lse, size = case.attention()
    nan = torch.isnan(want_lse)                   # (a key that is NaN makes all of the row NaN)
    assert torch.equal(torch.isnan(lse), nan)
    check_attention(case, got, lse, torch.where(nan[..., None], torch.full_like(want, math.nan), want), want_lse, size, tall=tall)


def test_many_sequences():
    """More than a launch's plan holds, among them such as have nothing to do."""
    lens = [(i * 7) % 4 for i in range(600)]
    cached = [(i * 37) % 200 for i in range(600)]
    run(QuantCase(lens, cached, 4, 2, 32, torch.bfloat16, seed=6))


@pytest.mark.parametrize("rows", [2, 140])
def test_pages_far_apart(rows):
    """Element offsets beyond 2^31: the sequence's pages are the last ones of a pool of 4.6 GB."""
    page, D, Hkv = 128, 128, 8
    case = QuantCase([rows], [700], 8, Hkv, D, torch.bfloat16, page=page, seed=8, first_page=72000, n_pages=72010)
    run(case)
    q, k, v = torch.randn(3, rows, Hkv, D, device="cuda").to(torch.bfloat16).unbind(0)
    case.cache.cs_quant_append(k, v, *case.blocks())
    assert torch.equal(*(x.double() for x in (case.cache.cs_quant_read(*case.blocks(), rows=rows)[0], __import__("quant_helpers").held(*__import__("quant_helpers").quantise(k)))))


def test_same_result_every_time():
    case = QuantCase([3, 9, 1], [5000, 300, 9000], 32, 8, 128, torch.float16, seed=9)
    first = case.cache.cs_quant_attention(case.q, *case.blocks(), with_lse=True)
    for _ in range(20):
        again = case.cache.cs_quant_attention(case.q, *case.blocks(), with_lse=True)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_wrong_blocks_and_pages():
    for tall, room in ((False, 0), (True, 0), (True, 1 << 14)):
        lens = [3, 4] if not tall else [150, 140]
        case = QuantCase(lens, [20, 300], 64 if room else 8, 2, 64, torch.bfloat16, seed=4, tall=room)
        want, want_lse, size = case.attention()
        out = torch.full((case.rows, case.H, 64), 9.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((case.rows, case.H), 9.0, device="cuda")
        case.cache.cs_quant_attention(case.q, case.start, case.len, i32([5000, 300]), case.table, out=out, lse=lse)
        assert case.cache.cs_quant_status() == cs.CS_ERR_CAPACITY and case.cache.cs_quant_status() == cs.CS_OK
        n = lens[0]
        assert bool((out[:n] == 9.0).all()) and bool((lse[:n] == 9.0).all())
        assert float((lse[n:].double() - want_lse[n:]).abs().max()) < 1e-4
        case.cache.cs_quant_attention(case.q, case.start, i32([-2, lens[1]]), case.kv_len, case.table, out=out, lse=lse)
        assert case.cache.cs_quant_status() == cs.CS_ERR_ARG and bool((out[:n] == 9.0).all())
        # a page that does not exist reads as zeros
        table = case.table.clone()
        table[1, 2] = -5
        got, got_lse = case.cache.cs_quant_attention(case.q, case.start, case.len, case.kv_len, table, with_lse=True)
        assert case.cache.cs_quant_status() == cs.CS_ERR_ARG
        case.k[1][32:48] = 0.0
        case.v[1][32:48] = 0.0
        check_attention(case, got, got_lse, *case.attention(), tall=tall)
