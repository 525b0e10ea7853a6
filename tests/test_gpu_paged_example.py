"""The example that decodes over a paged cache: its greedy continuations against the oracle's model, its copying against its plain
decoding's bookkeeping, and the fused append against norms and rotation by themselves."""
import importlib.util
import os

import pytest
import torch

from oracle import copyspec_oracle as O
from paper_2502_08923_b200 import inputs
from helpers import counters_for_streams, greedy_margins

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_decode.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("paged_decode", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("head_dim,kv_heads", [(32, 8), (64, 2), (128, 1)])
@pytest.mark.parametrize("k", [0, 10])
def test_greedy_continuations(example, head_dim, kv_heads, k):
    """Queries, weights and the LM head's input are rounded to bf16 here and not in the oracle: with logits below 2 that is a few roundings of 2^-9 each, so a
    token that is not the oracle's choice lies within 5e-2 of it."""
    cfg = inputs.ModelConfig(n_layers=2, d_model=256, n_heads=256 // head_dim * 2 if head_dim == 128 else 256 // head_dim, n_kv_heads=kv_heads, head_dim=head_dim, d_ffn=512, vocab=1000)
    w = inputs.make_weights(cfg, seed=3, gain_jitter=0.1)
    prompts = example.prompts_with_repeats(cfg, 3, 150, seed=2)
    model = example.PagedModel(cfg, inputs.weights_to(w, "cuda"), 3, 150 + 24 + 11)
    out, stats = example.generate(model, prompts, 24, k=k)
    model.close()
    oracle = O.Model(cfg, w, contract=True)
    for p, o in zip(prompts, out):
        assert len(o) == 24 and max(greedy_margins(oracle, cfg, p, o)) < 5e-2
    want = counters_for_streams(prompts, out, 3, k)
    assert {n: stats[n] for n in ("steps", "accepted", "emitted")} == {n: want[n] for n in ("steps", "accepted", "emitted")}


@pytest.mark.parametrize("qk_norm", [False, True])
def test_norms_and_rotation_apart_are_the_same(example, qk_norm):
    cfg = inputs.TINY
    w = inputs.weights_to(inputs.make_weights(cfg, seed=5), "cuda")
    prompts = example.prompts_with_repeats(cfg, 4, 200, seed=6)
    got = []
    for fused in (True, False):
        model = example.PagedModel(cfg, w, 4, 200 + 32 + 11, qk_norm=qk_norm, fused=fused)
        got.append((example.generate(model, prompts, 32), torch.stack([c.k_pages for c in model.caches]), torch.stack([c.v_pages for c in model.caches])))
        model.close()
    assert got[0][0] == got[1][0] and torch.equal(got[0][1], got[1][1]) and torch.equal(got[0][2], got[1][2])
