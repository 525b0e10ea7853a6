"""The three ways that attention over the cache of 4 bits takes - the kernel for few rows, tall blocks out of 4 bits, prompts' chunks from copies in 16 bits - where calls share what they work in: layers of one workspace, caches
of two streams over the same pools, captured graphs, streams that are not the default one."""
import pytest
import torch

from paper_2502_08923_b200 import binding as cs
from quant_helpers import QuantCase, check_attention, held, i32, is_tall, quantise

pytestmark = pytest.mark.gpu


def way(q, Hkv, n_seqs, table, page, tall_positions, window=0):
    """Which of them a call takes."""
    rows, room = -(-q.shape[0] * (q.shape[1] // Hkv) // n_seqs), table.shape[1] * page
    seen = min(room, window + q.shape[0] // n_seqs) if window else room
    if rows <= 32 or (rows <= 128 and rows * n_seqs * Hkv * seen <= 3 << 19):
        return "few"
    each = -(-tall_positions // 16) * 16 // n_seqs
    return "copies" if rows > 2560 and any(-(-room // size) * size <= each for size in (128, 64, 32, 16)) else "tall"


def way_of(case, window=0):
    return way(case.q, case.Hkv, len(case.lens), case.table, case.page, case.cache.tall_positions, window)


@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("ways", [("copies", "copies"), ("copies", "tall"), ("few", "copies"), ("tall", "few")])
def test_layers_of_other_values_on_one_workspace(D, dtype, ways):
    """Calls of two layers in turn, on one workspace: neither sees what the other left there."""
    shapes = {"copies": ([50, 70], 128), "tall": ([50, 70], 8), "few": ([1, 2], 8)}
    cases = [QuantCase(shapes[w][0], [200 + 31 * i, 90 + 70 * i], shapes[w][1], 2, D, dtype, seed=i, tall=1 << 12) for i, w in enumerate(ways)]
    if ways == ("few", "copies") and D == 32:             # (pages of another size as well)
        cases[0] = QuantCase([1, 2], [200, 90], 8, 2, D, dtype, page=64, seed=4, tall=1 << 12)
    assert tuple(way_of(c) for c in cases) == ways and [is_tall(c) for c in cases] == [w != "few" for w in ways]
    first = cases[0].cache
    caches = [first, cs.QuantCache(cases[1].kd, cases[1].vd, cases[1].ks, cases[1].vs, workspace=first)]
    want = [c.attention() for c in cases]
    got = [[cache.cs_quant_attention(c.q, *c.blocks(), with_lse=True) for cache, c in zip(caches, cases)] for _ in range(3)]
    assert first.cs_quant_status() == cs.CS_OK
    for turn in got:
        for c, (out, lse), w, expected in zip(cases, turn, ways, want):
            check_attention(c, out, lse, *expected, tall=w != "few")
    assert all(torch.equal(x, y) for turn in got[1:] for a, b in zip(turn, got[0]) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_chunks_from_copies_beside_single_tokens(dtype):
    """Prompts' chunks on one stream from copies, single tokens of other sequences on another by the kernel for few rows, over the same pools."""
    lens = [90, 1, 60, 1, 1]
    case = QuantCase(lens, [3000, 900, 2000, 500, 700], 128, 2, 128, dtype, seed=2)
    want, want_lse, size = case.attention()
    out, lse = torch.full_like(case.q, 7.0), torch.full(case.q.shape[:2], 7.0, device="cuda")
    calls = []
    for took in ("copies", "few"):
        pick = [b for b, n in enumerate(lens) if (n > 1) == (took == "copies")]
        cache = cs.QuantCache(case.kd, case.vd, case.ks, case.vs, tall_positions=1 << 15 if took == "copies" else 0)
        rows = torch.cat([torch.arange(case.starts[b], case.starts[b] + lens[b]) for b in pick]).cuda()
        q, table = case.q[rows].contiguous(), case.table[torch.tensor(pick).cuda()].contiguous()
        blocks = i32([sum(lens[c] for c in pick[:i]) for i in range(len(pick))]), i32([lens[b] for b in pick]), i32([case.cached[b] for b in pick]), table
        assert way(q, 2, len(pick), table, case.page, cache.tall_positions) == took
        calls.append((cache, q, blocks, rows, torch.cuda.Stream(), torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")))
    torch.cuda.synchronize()
    for _ in range(20):
        for cache, q, blocks, _, stream, o, l in calls:
            with torch.cuda.stream(stream):
                cache.cs_quant_attention(q, *blocks, out=o, lse=l)
    torch.cuda.synchronize()
    for cache, _, _, rows, _, o, l in calls:
        assert cache.cs_quant_status() == cs.CS_OK
        out[rows], lse[rows] = o, l
    check_attention(case, out, lse, want, want_lse, size, tall=True)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows,H,took", [(45, 128, "copies"), (45, 16, "tall"), (2, 8, "few")])
def test_captured_steps_of_two_layers(D, rows, H, took):
    """Two layers on one workspace, each with an append, an attention and what it appended read back, captured in one graph and replayed as the sequences grow, against the same outside of a graph."""
    B, Hkv, page, steps = 3, 2, 16, 4
    wide = -(-(200 + steps * rows) // page) + 1
    g = torch.Generator(device="cuda").manual_seed(rows)
    table = torch.randperm(B * wide, generator=torch.Generator().manual_seed(1)).to(torch.int32).view(B, wide).cuda().contiguous()
    rope = cs.cs_rope_table(wide * page, D)
    start, length = i32([b * rows for b in range(B)]), i32([rows, rows - 1, rows])
    layers = []
    for _ in range(2):                                    # of the graph, of the calls outside of it
        first = cs.QuantCache.empty(B * wide, Hkv, page, D, tall_positions=B * (wide + 8) * page)
        layers.append([first, cs.QuantCache.empty(B * wide, Hkv, page, D, workspace=first)])
    kv = [i32([100, 0, 37]) for _ in range(2)]
    qkv = torch.empty(2, B * rows, H + 2 * Hkv, D, device="cuda")
    out = torch.zeros(2, 2, B * rows, H, D, dtype=torch.bfloat16, device="cuda")
    back = torch.zeros(2, 2, 2, B * rows, Hkv, D, device="cuda")
    assert way(out[0, 0], Hkv, B, table, page, layers[0][0].tall_positions) == took

    def step(i):
        for n, cache in enumerate(layers[i]):
            q, k, v = qkv[n].split([H, Hkv, Hkv], dim=1)
            blocks = start, length, kv[i], table
            q = cache.cs_quant_append(k, v, *blocks, rope, None, q, None)
            cache.cs_quant_attention(q, *blocks, out=out[i, n])
            cache.cs_quant_read(*blocks, out=tuple(back[i, n]))
        kv[i] += length

    qkv.copy_(torch.randn(qkv.shape, generator=g, device="cuda"))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for i in range(2):
            step(i)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step(0)
    live = torch.cat([torch.arange(b * rows, b * rows + int(length[b])) for b in range(B)]).cuda()
    for _ in range(steps - 1):
        qkv.copy_(torch.randn(qkv.shape, generator=g, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        step(1)
        torch.cuda.synchronize()
        assert torch.equal(out[0], out[1]) and torch.equal(back[0], back[1]) and torch.equal(kv[0], kv[1])
        assert not torch.equal(out[0, 0], out[0, 1])
        for n in range(2):
            assert torch.equal(back[0, n, 1][live].double(), held(*quantise(qkv[n, :, H + Hkv:]))[live])
    assert all(c.cs_quant_status() == cs.CS_OK for pair in layers for c in pair)
    for n in range(2):
        assert torch.equal(layers[0][n].k_data, layers[1][n].k_data) and torch.equal(layers[0][n].v_scale.view(torch.int16), layers[1][n].v_scale.view(torch.int16))


@pytest.mark.parametrize("lens,H,took", [([50, 70], 128, "copies"), ([90, 40], 8, "tall"), ([3, 1], 8, "few")])
def test_not_the_default_stream(lens, H, took):
    """Everything on a stream that is not the default one, its inputs made there."""
    with torch.cuda.stream(torch.cuda.Stream()):
        for seed in range(3):
            case = QuantCase(lens, [100, 33], H, 2, 64, seed=seed, tall=1 << 12)
            assert way_of(case) == took
            got = case.cache.cs_quant_attention(case.q, *case.blocks(), with_lse=True)
            check_attention(case, *got, *case.attention(), tall=took != "few")
            assert case.cache.cs_quant_status() == cs.CS_OK
