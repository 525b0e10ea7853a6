"""Copy-and-verify decoding of a batch of sequences over a paged KV cache (Sec. 3.1, 3.2; App. B.3), with the library's operators
and torch for what lies between them.

    python examples/paged_decode.py [--batch 4] [--prompt 300] [--new 64] [--k 10] [--qk-norm]

Every step looks the last tokens of each history up (cs_find_match), runs the blocks [last token, copied draft] of all
sequences side by side - blocks of different heights, no padding - and keeps the longest agreeing prefix and one token more.  Rows of rejected tokens stay in
their pages behind kv_len and are overwritten by the next block.  Prompts go through the same path in chunks.  Per layer:

    cs_paged_append      the block's keys and values into the pages, normed and rotated, and its queries with them
    cs_paged_attention   the block's rows over the pages

(or, with fused=False, cs_qk_norm_rope for queries and keys and an append of what it returns: the same bits).
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2502_08923_b200 import binding as cs, inputs  # noqa: E402


class PagedModel:
    """A pre-norm decoder (RMSNorm, rotation, grouped heads, SwiGLU) whose keys and values live in pages, handed out as sequences grow."""

    def __init__(self, cfg, weights, batch, max_tokens, page_size=16, qk_norm=False, fused=True, seed=0):
        self.cfg, self.w, self.fused = cfg, weights, fused
        self.wide = -(-max_tokens // page_size)
        n_pages = batch * self.wide
        pools = torch.zeros(cfg.n_layers, 2, n_pages, cfg.n_kv_heads, page_size, cfg.head_dim, dtype=torch.bfloat16, device="cuda")
        self.caches = []
        for l in range(cfg.n_layers):      # one workspace for all layers: their work is on one stream
            self.caches.append(cs.PagedCache(pools[l, 0], pools[l, 1], workspace=self.caches[0] if self.caches else None))
        # a server hands pages out as it gets them back: in any order
        self.free = np.random.default_rng(seed).permutation(n_pages).tolist()
        self.page_size = page_size
        self.table_host = np.full((batch, self.wide), -1, dtype=np.int32)
        self.owned = [0] * batch
        self.table = torch.from_numpy(self.table_host).cuda()
        self.kv_len = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.rope = cs.cs_rope_table(max_tokens, cfg.head_dim, cfg.rope_theta)
        gain = lambda: (1 + 0.1 * torch.randn(cfg.head_dim, generator=torch.Generator().manual_seed(seed + 1))).to(torch.bfloat16).cuda()
        self.q_gain, self.k_gain = (gain(), gain()) if qk_norm else (None, None)
        self.fp32 = [{n: t.float() for n, t in layer.items()} for layer in weights["layers"]]

    def reserve(self, b, tokens):
        """Pages for `tokens` positions of sequence b."""
        need = -(-tokens // self.page_size)
        if need > self.owned[b]:
            for i in range(self.owned[b], need):
                self.table_host[b, i] = self.free.pop()
            self.owned[b] = need
            self.table[b].copy_(torch.from_numpy(self.table_host[b]))

    def _norm(self, x, gain):
        return x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + self.cfg.rms_eps) * gain.float()

    def forward(self, tokens, start, length):
        """Final normed activations [rows][d] of the blocks' tokens [rows]; their keys and values are in the pages afterwards."""
        c = self.cfg
        x = self.w["embed"][tokens.long()].float()
        for l, w in enumerate(self.fp32):
            qkv = self._norm(x, w["attn_norm"]) @ w["wqkv"].T
            q, k, v = (t.unflatten(1, (-1, c.head_dim)) for t in qkv.split([c.q_dim, c.kv_dim, c.kv_dim], dim=1))
            cache, blocks = self.caches[l], (start, length, self.kv_len, self.table)
            if self.fused:
                q = cache.cs_paged_append(k, v, *blocks, self.rope, self.k_gain, q, self.q_gain, eps=c.rms_eps)
            else:
                # rows of a block sit at kv_len + r; rows of none (there are none here) could have any position
                pos = (self.kv_len - start).repeat_interleave(length.long()) + torch.arange(len(tokens), device="cuda", dtype=torch.int32)
                q, k = cs.cs_qk_norm_rope(q, k, pos, self.rope, self.q_gain, self.k_gain, eps=c.rms_eps, dtype=torch.bfloat16)
                cache.cs_paged_append(k, v.to(torch.bfloat16), *blocks)
            a = cache.cs_paged_attention(q, *blocks)
            x = x + a.flatten(1).float() @ w["wo"].T
            gate, up = (self._norm(x, w["ffn_norm"]) @ w["w_gate_up"].T).chunk(2, dim=1)
            x = x + (torch.nn.functional.silu(gate) * up) @ w["w_down"].T
        return self._norm(x, self.w["final_norm"])

    def greedy(self, x):
        rows = x.shape[0]
        padded = torch.zeros(-(-rows // 16) * 16, x.shape[1], dtype=torch.bfloat16, device="cuda")      # (the call reads whole groups of 16 rows)
        padded[:rows] = x.to(torch.bfloat16)
        ids = torch.empty(rows, dtype=torch.int32, device="cuda")
        return cs.cs_lm_head_static(padded, self.w["lm_head"], ids, rows)

    def prefill(self, prompts, chunk=256):
        """Prompts but their last tokens into the pages, `chunk` tokens of every sequence at a time."""
        todo = [np.asarray(p[:-1], dtype=np.int32) for p in prompts]
        for b, t in enumerate(todo):
            self.reserve(b, len(t))
        for at in range(0, max(map(len, todo)), chunk):
            parts = [t[at:at + chunk] for t in todo]
            start, length = _blocks([len(p) for p in parts])
            self.forward(torch.from_numpy(np.concatenate(parts)).cuda(), start, length)
            self.kv_len += length
        return self

    def close(self):
        for c in self.caches:
            c.close()


def _blocks(lengths):
    start = np.concatenate([[0], np.cumsum(lengths)[:-1]])
    both = torch.from_numpy(np.stack([start, lengths]).astype(np.int32)).cuda()
    return both[0], both[1]


def generate(model, prompts, max_new, gamma=3, k=10, policy=cs.LATEST):
    """Greedy continuation of every prompt (max_new tokens each) by copying and verifying; (token lists, statistics)."""
    B, longest = len(prompts), max(map(len, prompts)) + max_new + k + 1
    if B * (k + 1) > 64:
        raise ValueError("the LM-head call takes 64 rows")
    hist = np.zeros((B, longest), dtype=np.int32)
    n = np.array([len(p) for p in prompts], dtype=np.int32)
    for b, p in enumerate(prompts):
        hist[b, :n[b]] = p
    model.prefill(prompts)
    hist_dev, out = torch.from_numpy(hist).cuda(), [[] for _ in prompts]
    stats = {"steps": 0, "attempts": 0, "accepted": 0, "emitted": 0}
    while any(len(o) < max_new for o in out):
        open_ = [b for b in range(B) if len(out[b]) < max_new]
        _, draft, draft_len = cs.cs_find_match(hist_dev, torch.from_numpy(n).cuda(), gamma, k, policy)
        draft, draft_len = draft.cpu().numpy(), draft_len.cpu().numpy()
        rows = [1 + min(int(draft_len[b]), max_new - len(out[b]) - 1) if b in open_ else 0 for b in range(B)]
        blocks = [np.concatenate([hist[b, n[b] - 1:n[b]], draft[b, :rows[b] - 1]]) if rows[b] else np.zeros(0, np.int32) for b in range(B)]
        for b in open_:
            model.reserve(b, int(n[b]) - 1 + rows[b])
        start, length = _blocks(rows)
        ids = model.greedy(model.forward(torch.from_numpy(np.concatenate(blocks).astype(np.int32)).cuda(), start, length)).cpu().numpy()
        keep, at = np.zeros(B, dtype=np.int32), 0
        for b in range(B):
            target, at = ids[at:at + rows[b]], at + rows[b]
            if not rows[b]:
                continue
            tau = 0
            while tau < rows[b] - 1 and draft[b, tau] == target[tau]:
                tau += 1
            new = target[:tau + 1]
            hist[b, n[b]:n[b] + len(new)] = new
            n[b] += len(new)
            out[b] += new.tolist()
            keep[b] = len(new)                                    # the last token's rows come with the next block
            stats["steps"] += 1
            stats["attempts"] += int(rows[b] > 1)
            stats["accepted"] += tau
            stats["emitted"] += len(new)
        model.kv_len += torch.from_numpy(keep).cuda()
        hist_dev.copy_(torch.from_numpy(hist))
    for c in model.caches[:1]:
        if c.cs_paged_status() != cs.CS_OK:
            raise RuntimeError("the paged cache reports an error")
    return out, stats


def prompts_with_repeats(cfg, batch, length, seed):
    """Random prompts that end in the middle of a stretch they have had before."""
    rng = np.random.default_rng(seed)
    prompts = []
    for b in range(batch):
        n = max(24, length - 37 * b)
        p = rng.integers(0, cfg.vocab, size=n)
        p[-8:] = p[n // 3:n // 3 + 8]
        prompts.append(p.astype(np.int32).tolist())
    return prompts


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--batch", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=300)
    ap.add_argument("--new", type=int, default=64)
    ap.add_argument("--k", type=int, default=10)
    ap.add_argument("--qk-norm", action="store_true")
    a = ap.parse_args()
    cfg = inputs.TINY
    w = inputs.weights_to(inputs.make_weights(cfg, seed=0), "cuda")
    prompts = prompts_with_repeats(cfg, a.batch, a.prompt, seed=1)
    results = {}
    for k in (0, a.k):
        model = PagedModel(cfg, w, a.batch, a.prompt + a.new + a.k + 1, qk_norm=a.qk_norm)
        results[k], stats = generate(model, prompts, a.new, k=k)
        model.close()
        print(f"k = {k}: {stats['emitted']} tokens in {stats['steps']} blocks, {stats['accepted']} copied tokens accepted in {stats['attempts']} attempts")
    same = sum(x == y for p, q in zip(results[0], results[a.k]) for x, y in zip(p, q))
    print(f"{same} of {a.batch * a.new} tokens equal those of plain decoding")


if __name__ == "__main__":
    main()
