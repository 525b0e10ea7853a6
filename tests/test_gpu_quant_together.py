"""The operators around the cache of 4 bits as they are used: one after the other, by several layers and streams, captured and replayed, in the example."""
import importlib.util
import os

import pytest
import torch

from paper_2502_08923_b200 import binding as cs, inputs
from paged_helpers import i32, norm_rope
from quant_helpers import QuantCase, check_attention, is_tall, held, quantise

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_decode.py")


@pytest.mark.parametrize("lens", [[1, 2], [50, 70]])
def test_further_layers_on_one_workspace(lens):
    case = QuantCase(lens, [200, 90], 8, 2, 128, seed=1, tall=1 << 12)
    first, want = case.cache, case.attention()
    tall = is_tall(case)
    pools = lambda: (case.data[0].clone(), case.data[1].clone(), case.scales[0].clone(), case.scales[1].clone())
    first.cs_quant_attention(case.q, case.start, i32([lens[0], -1]), case.kv_len, case.table)
    second = cs.QuantCache(*pools(), workspace=first)      # (made while the first is at work: nothing is cleared)
    assert second.cs_quant_status() == cs.CS_ERR_ARG and first.cs_quant_status() == cs.CS_OK
    check_attention(case, *second.cs_quant_attention(case.q, *case.blocks(), with_lse=True), *want, tall=tall)
    first.close()
    check_attention(case, *second.cs_quant_attention(case.q, *case.blocks(), with_lse=True), *want, tall=tall)
    third = cs.QuantCache(*pools(), workspace=second)
    check_attention(case, *third.cs_quant_attention(case.q, *case.blocks(), with_lse=True), *want, tall=tall)
    assert third.cs_quant_status() == cs.CS_OK
    with pytest.raises(cs.CsError) as e:
        cs.QuantCache(*pools(), workspace=first)
    assert e.value.code == cs.CS_ERR_ARG                   # it has been closed
    other = QuantCase([1], [20], 4, 2, 64)
    with pytest.raises(cs.CsError) as e:
        cs.QuantCache(other.kd, other.vd, other.ks, other.vs, workspace=second)
    assert e.value.code in (cs.CS_ERR_SHAPE, cs.CS_ERR_CAPACITY) and "cs_quant_create_beside" in str(e.value)


def test_two_streams_have_a_workspace_each():
    """Prompts' chunks on one stream, single tokens of other sequences on another, over the same pools."""
    case = QuantCase([150, 1, 90, 1, 1], [3000, 4000, 2000, 500, 2500], 8, 2, 128, seed=2)
    out_want, lse_want, size = case.attention()
    lens = [i32([n if tall == (n > 1) else 0 for n in case.lens]) for tall in (True, False)]
    caches = [cs.QuantCache(case.kd, case.vd, case.ks, case.vs, tall_positions=t) for t in (1 << 15, 0)]
    out, lse = torch.full_like(case.q, 7.0), torch.full(case.q.shape[:2], 7.0, device="cuda")
    streams = [torch.cuda.Stream() for _ in lens]
    torch.cuda.synchronize()
    for _ in range(20):
        for cache, length, stream in zip(caches, lens, streams):
            with torch.cuda.stream(stream):
                cache.cs_quant_attention(case.q, case.start, length, case.kv_len, case.table, out=out, lse=lse)
    torch.cuda.synchronize()
    assert all(c.cs_quant_status() == cs.CS_OK for c in caches)
    check_attention(case, out, lse, out_want, lse_want, size, tall=True)


@pytest.mark.parametrize("rows", [1, 11, 40])
def test_a_captured_step_follows_the_lengths(rows):
    """A step (append, attention, reading back) captured once and replayed as the sequences grow, against the same step outside of a graph."""
    B, H, Hkv, D, page, steps = 3, 8, 2, 64, 16, 5
    n_pages = B * (-(-(200 + steps * rows) // page) + 1)
    g = torch.Generator(device="cuda").manual_seed(rows)
    table = torch.randperm(n_pages, generator=torch.Generator().manual_seed(1)).to(torch.int32).view(B, -1).cuda().contiguous()
    rope = cs.cs_rope_table(table.shape[1] * page, D)
    start, length = i32([b * rows for b in range(B)]), i32([rows, max(0, rows - 1), rows])
    caches = [cs.QuantCache.empty(n_pages, Hkv, page, D, tall_positions=n_pages * page) for _ in range(2)]
    kv = [i32([100, 0, 37]) for _ in range(2)]
    qkv = torch.empty(B * rows, H + 2 * Hkv, D, device="cuda")
    out = [torch.zeros(B * rows, H, D, dtype=torch.float16, device="cuda") for _ in range(2)]
    held_rows = [tuple(torch.zeros(B * rows, Hkv, D, device="cuda") for _ in range(2)) for _ in range(2)]

    def step(i):
        q, k, v = qkv.split([H, Hkv, Hkv], dim=1)
        blocks = start, length, kv[i], table
        q = caches[i].cs_quant_append(k, v, *blocks, rope, None, q, None, dtype=torch.float16)
        caches[i].cs_quant_attention(q, *blocks, out=out[i])
        caches[i].cs_quant_read(*blocks, out=held_rows[i])
        kv[i] += length

    first = torch.randn(qkv.shape, generator=g, device="cuda")
    qkv.copy_(first)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for i in range(2):
            step(i)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step(0)
    for _ in range(steps - 1):
        qkv.copy_(torch.randn(qkv.shape, generator=g, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        step(1)
        torch.cuda.synchronize()
        assert torch.equal(out[0], out[1]) and all(torch.equal(x, y) for x, y in zip(*held_rows)) and torch.equal(kv[0], kv[1])
        n, s = quantise(qkv[:, H + Hkv:])
        live = torch.cat([torch.arange(b * rows, b * rows + int(length[b])) for b in range(B)]).cuda()
        assert torch.equal(held_rows[0][1][live].double(), held(n, s)[live])
    assert all(c.cs_quant_status() == cs.CS_OK for c in caches)
    assert torch.equal(caches[0].k_data, caches[1].k_data) and torch.equal(caches[0].v_scale.view(torch.int16), caches[1].v_scale.view(torch.int16))


def test_other_than_the_current_stream():
    """Everything on a stream that is not the default one, its inputs made there."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        for lens in ([3, 1], [90, 40]):
            case = QuantCase(lens, [100, 33], 8, 2, 64, seed=3, tall=1 << 12)
            got = case.cache.cs_quant_attention(case.q, *case.blocks(), with_lse=True)
            check_attention(case, *got, *case.attention(), tall=is_tall(case))
            assert case.cache.cs_quant_status() == cs.CS_OK


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("paged_decode", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def logits_64(cfg, w, tokens, theta, q_gain, k_gain):
    """Logits [tokens][vocab] of a whole sequence in 64 bits, keys and values as the cache holds them."""
    H, Hkv, D = cfg.n_heads, cfg.n_kv_heads, cfg.head_dim
    n = len(tokens)
    norm = lambda x, g: x / torch.sqrt((x * x).mean(dim=-1, keepdim=True) + cfg.rms_eps) * g.double()
    rope = cs.cs_rope_table(n, D, theta)
    x = w["embed"][torch.tensor(tokens, device="cuda")].double()
    pos = torch.arange(n, device="cuda")
    hidden = pos[None, :] > pos[:, None]
    for layer in w["layers"]:
        qkv = norm(x, layer["attn_norm"]) @ layer["wqkv"].double().T
        q, k, v = (t.unflatten(1, (-1, D)) for t in qkv.split([cfg.q_dim, cfg.kv_dim, cfg.kv_dim], dim=1))
        q, k = norm_rope(q, q_gain, rope, pos, cfg.rms_eps)[0], norm_rope(k, k_gain, rope, pos, cfg.rms_eps)[0]
        k, v = held(*quantise(k)), held(*quantise(v))
        s = torch.einsum("ihd,jhd->hij", q, k.repeat_interleave(H // Hkv, dim=1)) / D ** 0.5
        a = torch.einsum("hij,jhd->ihd", torch.softmax(s.masked_fill(hidden, float("-inf")), dim=-1), v.repeat_interleave(H // Hkv, dim=1))
        x = x + a.flatten(1) @ layer["wo"].double().T
        gate, up = (norm(x, layer["ffn_norm"]) @ layer["w_gate_up"].double().T).chunk(2, dim=1)
        x = x + (torch.nn.functional.silu(gate) * up) @ layer["w_down"].double().T
    return norm(x, w["final_norm"]) @ w["lm_head"].double().T


@pytest.mark.parametrize("head_dim,kv_heads", [(32, 8), (64, 2), (128, 1)])
@pytest.mark.parametrize("k,qk_norm", [(0, False), (10, True)])
def test_greedy_continuations(example, head_dim, kv_heads, k, qk_norm):
    """Queries, softmax weights of prompts and the LM head's input are rounded to bf16 in the example and not in the plain forward: with logits below 2 that is a few roundings of 2^-9 each, so a token that is not its
    choice lies within 5e-2 of it.  (A key that comes out on the other side of a border for a last bit changes one of hundreds of elements of one score by a step.)"""
    cfg = inputs.ModelConfig(n_layers=2, d_model=256, n_heads=4 if head_dim == 128 else 256 // head_dim, n_kv_heads=kv_heads, head_dim=head_dim, d_ffn=512, vocab=1000)
    w = inputs.weights_to(inputs.make_weights(cfg, seed=3, gain_jitter=0.1), "cuda")
    prompts = example.prompts_with_repeats(cfg, 3, 150, seed=2)
    model = example.PagedModel(cfg, w, 3, 150 + 24 + 11, qk_norm=qk_norm, bits=4)
    out, stats = example.generate(model, prompts, 24, k=k)
    for p, o in zip(prompts, out):
        assert len(o) == 24
        logits = logits_64(cfg, w, p + o, cfg.rope_theta, model.q_gain, model.k_gain)[len(p) - 1:-1]
        margin = logits.amax(dim=1) - logits[torch.arange(24), torch.tensor(o, device="cuda")]
        assert float(margin.max()) < 5e-2
    model.close()
