"""The operators around a paged key/value cache, as a server of copy-and-verify decoding calls them: what is measured, their plain
forms, and their definitions in 64 bits.

Three operators (`op`):
  norm_rope   per-head RMS norms of queries and keys and the position rotation, for caches of the caller's own
  append      a block's keys and values into the pages of their sequences, keys normed and rotated on the way, the block's queries with them
  attention   blocks of new rows, from single tokens to a prompt's chunk, over the pages

Conventions are the package's: row r of sequence b's block sits at position kv_len[b] + r, where kv_len counts what was cached before the
block; the rows of all blocks lie one after the other in the tensors.  Head layouts are those of the 8B-class shape (32 query heads over 8
of 128), of the 1B-class draft model (32 over 8 of 64) and of the small model (8 over 8 of 32).
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEVICE = "cuda" if torch.cuda.is_available() else "cpu"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-5
SHAPES = {"8b": (32, 8, 128, 500000.0), "1b": (32, 8, 64, 500000.0), "tiny": (8, 8, 32, 10000.0)}   # heads, KV heads, head size, theta


def listed():
    att = {"op": "attention", "dtype": "bf16", "page": 16, "layout": "head", "ragged": False, "mask": "causal", "window": 0}
    app = {"op": "append", "dtype": "bf16", "source": "bf16", "page": 16, "layout": "head", "ragged": False, "norm": True}
    nrm = {"op": "norm_rope", "dtype": "bf16", "source": "bf16", "norm": True}
    return [
        # the smallest call: the small model verifies ten copied tokens behind 512, launch latency counts
        att | {"name": "attn_tiny_b1_512_k10", "shape": "tiny", "batch": 1, "rows": 11, "keys": 512},
        # the usual verification: one sequence, 4k context, ten copied tokens
        att | {"name": "attn_8b_b1_4k_k10", "shape": "8b", "batch": 1, "rows": 11, "keys": 4096},
        # one token over a long document
        att | {"name": "attn_8b_b1_30k_decode", "shape": "8b", "batch": 1, "rows": 1, "keys": 30720},
        # a server's batch of single tokens, sequences of all lengths
        att | {"name": "attn_8b_b64_4k_decode", "shape": "8b", "dtype": "fp16", "page": 64, "batch": 64, "rows": 1, "keys": 4097, "ragged": True},
        # a draft model's blocks behind long contexts, twenty copied tokens, pages with the heads inside
        att | {"name": "attn_1b_b8_16k_k20", "shape": "1b", "page": 32, "layout": "token", "batch": 8, "rows": 21, "keys": 16384},
        # chunks of several prompts with a sliding window, odd sizes
        att | {"name": "attn_8b_b3_chunk_1531_window", "shape": "8b", "dtype": "fp16", "page": 64, "batch": 3, "rows": 1531, "keys": 3001, "ragged": True, "window": 1000},
        # the largest: a prompt's chunk behind a long context
        att | {"name": "attn_8b_b1_30k_chunk_2048", "shape": "8b", "page": 64, "batch": 1, "rows": 2048, "keys": 30720},
        # a verification block's rows into the cache, straight out of a projection in 32 bits
        app | {"name": "append_8b_b1_k10", "shape": "8b", "source": "fp32", "batch": 1, "rows": 11, "keys": 4096},
        # a server's batch of single tokens of the draft model, rotation only
        app | {"name": "append_1b_b64_decode", "shape": "1b", "dtype": "fp16", "source": "fp16", "page": 32, "layout": "token", "batch": 64, "rows": 1, "keys": 1531, "ragged": True, "norm": False},
        # chunks of four prompts
        app | {"name": "append_8b_b4_chunk_2048", "shape": "8b", "page": 64, "batch": 4, "rows": 2048, "keys": 1024, "ragged": True},
        # one block of a caller with a cache of its own
        nrm | {"name": "norm_rope_1b_k20", "shape": "1b", "dtype": "fp16", "source": "fp16", "rows": 21, "positions": 16384},
        # a whole prompt
        nrm | {"name": "norm_rope_8b_8k", "shape": "8b", "rows": 8192, "positions": 8192},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attention", "attention", "attention", "append", "norm_rope"])
    shape = rng.choice(["8b", "8b", "8b", "1b", "1b", "tiny"])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    source = rng.choice([dtype, dtype, "fp32"])
    if op == "norm_rope":
        return {"op": op, "shape": shape, "dtype": dtype, "source": source, "norm": rng.random() < 0.7, "rows": _log_int(rng, 1, 8192), "positions": _log_int(rng, 8192, 131072)}
    page, layout = rng.choice([16, 16, 32, 64, 128]), rng.choice(["head", "head", "token"])
    if op == "append":
        rows = _log_int(rng, 1, 8192)
        batch = min(rows, _log_int(rng, 1, 64))
        return {"op": op, "shape": shape, "dtype": dtype, "source": source, "page": page, "layout": layout, "batch": batch, "rows": rows // batch,
                "keys": _log_int(rng, 1, 65536 // batch), "ragged": rng.random() < 0.6, "norm": rng.random() < 0.6}
    kind = rng.choice(["decode", "verify", "chunk"])
    if kind == "chunk":
        batch, rows = rng.randint(1, 4), _log_int(rng, 100, 2048)
        rows = max(25, rows // batch)
        keys = _log_int(rng, 1, 30720 // batch)
    else:
        batch = _log_int(rng, 1, 64)
        rows = 1 if kind == "decode" else rng.randint(2, max(2, min(21, 256 // batch)))
        keys = _log_int(rng, 30, min(30720, 262144 // batch))
    return {"op": op, "shape": shape, "dtype": dtype, "page": page, "layout": layout, "batch": batch, "rows": rows, "keys": keys, "ragged": rng.random() < 0.6,
            "mask": rng.choice(["causal", "causal", "causal", "prefix"]), "window": rng.choice([0, 0, 0, _log_int(rng, 20, 4096)])}


def _lengths(case):
    """Rows of each sequence's block and what it has cached, by the case alone (a case's work is the same whatever the seed)."""
    B, rows, keys = case["batch"], case["rows"], case["keys"]
    if not case["ragged"]:
        return [rows] * B, [keys] * B
    rng = random.Random(1000003 * B + 1009 * rows + keys)
    return [rng.randint((rows + 1) // 2, rows) for _ in range(B)], [_log_int(rng, max(1, keys // 8), keys) for _ in range(B)]


def _range(case, n, c, r):
    """Keys [lo, hi) that row r of a block of n rows behind c cached keys attends to."""
    hi = c + r + 1 if case["mask"] == "causal" else c
    return (max(0, c + r + 1 - case["window"]) if case["window"] else 0), hi


def _rope(positions, dim, theta):
    inv = theta ** (-torch.arange(0, dim, 2, dtype=torch.float64, device=DEVICE) / dim)
    angle = torch.arange(positions, dtype=torch.float64, device=DEVICE)[:, None] * inv
    return torch.cat([angle.cos(), angle.sin()], dim=1).float()


def prepare(case, seed):
    H, Hkv, D, theta = SHAPES[case["shape"]]
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0, to=dtype):
        return (torch.randn(*shape, generator=g, device=DEVICE) * scale).to(to)

    def gain(n):
        return normal(n, scale=0.1, to=torch.float32).add_(1.0).to(dtype)

    s = {"case": case}
    if case["op"] == "norm_rope":
        T, source = case["rows"], DTYPES[case["source"]]
        qkv = normal(T, (H + 2 * Hkv) * D, to=source)                 # a projection's output; queries and keys are views of it
        s |= {"q": qkv[:, :H * D].unflatten(1, (H, D)), "k": qkv[:, H * D:(H + Hkv) * D].unflatten(1, (Hkv, D)),
              "pos": torch.randint(0, case["positions"], (T,), generator=g, device=DEVICE, dtype=torch.int32),
              "rope": _rope(case["positions"], D, theta), "q_gain": gain(D) if case["norm"] else None, "k_gain": gain(D) if case["norm"] else None}
        return s
    lens, cached = _lengths(case)
    B, T, page = case["batch"], sum(lens), case["page"]
    total = [n + c for n, c in zip(lens, cached)]
    wide = max(-(-t // page) for t in total)
    used = sum(-(-t // page) for t in total)
    n_pages = used + 3
    shape = (n_pages, Hkv, page, D) if case["layout"] == "head" else (n_pages, page, Hkv, D)
    pools = normal(2, *shape)
    if case["layout"] == "token":
        pools = pools.transpose(2, 3)
    # pages in the order a server hands them out after a while: any; entries behind a sequence's last page are -1
    order = torch.randperm(n_pages, generator=g, device=DEVICE).to(torch.int32)
    table = torch.full((B, wide), -1, dtype=torch.int32, device=DEVICE)
    at = 0
    for b, t in enumerate(total):
        n = -(-t // page)
        table[b, :n] = order[at:at + n]
        at += n
    starts = [sum(lens[:b]) for b in range(B)]
    ints = torch.tensor([starts, lens, cached], dtype=torch.int32, device=DEVICE)
    s |= {"k_pages": pools[0], "v_pages": pools[1], "table": table, "start": ints[0], "len": ints[1], "kv_len": ints[2]}
    if case["op"] == "attention":
        # heads differ in how sharply they look
        s["q"] = (torch.randn(T, H, D, generator=g, device=DEVICE) * torch.linspace(0.5, 2.5, H, device=DEVICE)[:, None]).to(dtype)
    else:
        qkv = normal(T, (H + 2 * Hkv) * D, to=DTYPES[case["source"]])
        s |= {"q": qkv[:, :H * D].unflatten(1, (H, D)), "k": qkv[:, H * D:(H + Hkv) * D].unflatten(1, (Hkv, D)), "v": qkv[:, (H + Hkv) * D:].unflatten(1, (Hkv, D)),
              "rope": _rope(max(total), D, theta), "q_gain": gain(D) if case["norm"] else None, "k_gain": gain(D) if case["norm"] else None}
    if own:
        from paper_2502_08923_b200 import binding as cs
        s["cache"] = cs.PagedCache(s["k_pages"], s["v_pages"])
    return s


# ------------------------------------------------------------------------------------------ plain forms
def _norm_rope(x, gain, rope, pos):
    x = x.float()
    if gain is not None:
        x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * gain.float()
    h = x.shape[-1] // 2
    cs = rope[pos.long()][:, None, :]
    c, sn = cs[..., :h], cs[..., h:]
    a, b = x[..., :h], x[..., h:]
    return torch.cat([a * c - b * sn, b * c + a * sn], dim=-1)


def _plain_append(s):
    T, page = s["k"].shape[0], s["k_pages"].shape[2]
    t = torch.arange(T, device=DEVICE)
    b = (t[:, None] >= s["start"][None, :]).sum(dim=1) - 1
    pos = s["kv_len"][b].long() + t - s["start"][b].long()
    at = s["table"][b, pos // page].long()
    dtype = s["k_pages"].dtype
    s["k_pages"][at, :, pos % page] = _norm_rope(s["k"], s["k_gain"], s["rope"], pos).to(dtype)
    s["v_pages"][at, :, pos % page] = s["v"].to(dtype)
    return _norm_rope(s["q"], s["q_gain"], s["rope"], pos).to(dtype), s["k_pages"], s["v_pages"]


def _plain_attention(s):
    case, q = s["case"], s["q"]
    H, Hkv, D, _ = SHAPES[case["shape"]]
    (T, page), B = (q.shape[0], s["k_pages"].shape[2]), s["table"].shape[0]
    R, N = case["rows"], s["table"].shape[1] * page
    # every sequence's rows and keys side by side, as wide as the longest has them
    r, j = torch.arange(R, device=DEVICE), torch.arange(N, device=DEVICE)
    row = (s["start"][:, None] + r).clamp(max=T - 1).long()
    live = r[None, :] < s["len"][:, None]
    at = s["table"].long().clamp(min=0)
    k = s["k_pages"][at].float().transpose(1, 2).reshape(B, Hkv, 1, N, D)
    v = s["v_pages"][at].float().transpose(1, 2).reshape(B, Hkv, 1, N, D)
    x = q[row].float().reshape(B, R, Hkv, H // Hkv, D).permute(0, 2, 3, 1, 4)
    scores = (x @ k.transpose(-1, -2)).mul_(1.0 / math.sqrt(D))
    pos = s["kv_len"][:, None] + r
    hi = pos + 1 if case["mask"] == "causal" else s["kv_len"][:, None].expand(B, R)
    seen = j < hi[..., None]
    if case["window"]:
        seen &= j > pos[..., None] - case["window"]
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    m = scores.amax(dim=-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    w = scores.sub_(m).exp_()
    total = w.sum(dim=-1, keepdim=True)
    out = (w @ v) / torch.where(total > 0, total, torch.ones_like(total))
    lse = (m + total.log()).squeeze(-1)
    out = out.permute(0, 3, 1, 2, 4).reshape(B, R, H, D)[live]
    lse = lse.permute(0, 3, 1, 2).reshape(B, R, H)[live]
    return out.to(q.dtype), lse


def run(s):
    case = s["case"]
    if own:
        from paper_2502_08923_b200 import binding as cs
        if case["op"] == "norm_rope":
            return cs.cs_qk_norm_rope(s["q"], s["k"], s["pos"], s["rope"], q_gain=s["q_gain"], k_gain=s["k_gain"], eps=EPS, dtype=DTYPES[case["dtype"]])
        if case["op"] == "append":
            q = s["cache"].cs_paged_append(s["k"], s["v"], s["start"], s["len"], s["kv_len"], s["table"], s["rope"], k_gain=s["k_gain"],
                                           q=s["q"], q_gain=s["q_gain"], eps=EPS)
            return q, s["k_pages"], s["v_pages"]
        return s["cache"].cs_paged_attention(s["q"], s["start"], s["len"], s["kv_len"], s["table"], window=case["window"],
                                             mask=cs.MASK_CAUSAL if case["mask"] == "causal" else cs.MASK_PREFIX, with_lse=True)
    if case["op"] == "norm_rope":
        dtype = DTYPES[case["dtype"]]
        return _norm_rope(s["q"], s["q_gain"], s["rope"], s["pos"]).to(dtype), _norm_rope(s["k"], s["k_gain"], s["rope"], s["pos"]).to(dtype)
    return _plain_append(s) if case["op"] == "append" else _plain_attention(s)


def work(case):
    H, Hkv, D, _ = SHAPES[case["shape"]]
    size = {"bf16": 2, "fp16": 2, "fp32": 4}
    e = size[case["dtype"]]
    if case["op"] == "norm_rope":
        n = case["rows"] * (H + Hkv) * D
        # the rotation's rows: each position once at most
        return {"bytes": n * (size[case["source"]] + e) + 4 * case["rows"] + 4 * D * min(case["rows"], case["positions"]), "flops": 10 * n}
    lens, cached = _lengths(case)
    T = sum(lens)
    if case["op"] == "append":
        n, nv = T * (H + Hkv) * D, T * Hkv * D
        return {"bytes": (n + nv) * (size[case["source"]] + e) + 4 * D * min(T, max(a + c for a, c in zip(lens, cached))), "flops": 10 * n}
    pairs = keys = 0
    for n, c in zip(lens, cached):
        ends = [_range(case, n, c, r) for r in range(n)]
        pairs += sum(max(0, hi - lo) for lo, hi in ends)
        keys += max(0, max(hi for _, hi in ends) - min(lo for lo, _ in ends))
    return {"bytes": keys * 2 * Hkv * D * e + T * H * (2 * D * e + 4), "flops": 4 * D * H * pairs}


# ------------------------------------------------------------------------------------------ definitions in 64 bits
def _exact_row_heads(x, gain, rope, pos):
    y = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    h = x.shape[-1] // 2
    x = x.double()
    if gain is not None:
        x = x / torch.sqrt(torch.einsum("thd,thd->th", x, x)[..., None] / x.shape[-1] + EPS) * gain.double()
    cos, sin = rope.double()[pos.long()].split(h, dim=1)
    y[..., :h] = torch.einsum("thd,td->thd", x[..., :h], cos) - torch.einsum("thd,td->thd", x[..., h:], sin)
    y[..., h:] = torch.einsum("thd,td->thd", x[..., h:], cos) + torch.einsum("thd,td->thd", x[..., :h], sin)
    return y


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm_rope":
        return _exact_row_heads(s["q"], s["q_gain"], s["rope"], s["pos"]), _exact_row_heads(s["k"], s["k_gain"], s["rope"], s["pos"])
    H, Hkv, D, _ = SHAPES[case["shape"]]
    G, page = H // Hkv, case["page"]
    lens, cached = _lengths(case)
    if case["op"] == "append":
        pos = torch.cat([torch.arange(c, c + n) for n, c in zip(lens, cached)]).to(DEVICE)
        q, k = _exact_row_heads(s["q"], s["q_gain"], s["rope"], pos), _exact_row_heads(s["k"], s["k_gain"], s["rope"], pos)
        kp, vp, t = s["k_pages"].double(), s["v_pages"].double(), 0
        for b, (n, c) in enumerate(zip(lens, cached)):
            for first in range(c // page * page, c + n, page):
                at, lo, hi = int(s["table"][b, first // page]), max(first, c), min(first + page, c + n)
                kp[at, :, lo - first:hi - first] = k[t + lo - c:t + hi - c].transpose(0, 1)
                vp[at, :, lo - first:hi - first] = s["v"][t + lo - c:t + hi - c].double().transpose(0, 1)
            t += n
        return q, kp, vp
    out, lse, t = torch.empty(sum(lens), H, D, dtype=torch.float64, device=DEVICE), torch.empty(sum(lens), H, dtype=torch.float64, device=DEVICE), 0
    for b, (n, c) in enumerate(zip(lens, cached)):
        pages = s["table"][b, :-(-(n + c) // page)].long()
        ends = torch.tensor([_range(case, n, c, r) for r in range(n)], device=DEVICE)
        j = torch.arange(n + c, device=DEVICE)
        hidden = (j < ends[:, :1]) | (j >= ends[:, 1:])
        for h in range(Hkv):
            k, v = (p[pages, h].reshape(-1, D)[:n + c].double() for p in (s["k_pages"], s["v_pages"]))
            for i in range(h * G, (h + 1) * G):
                x = s["q"][t:t + n, i].double() @ k.T / math.sqrt(D)
                x[hidden] = -math.inf
                lse[t:t + n, i] = torch.logsumexp(x, dim=1)
                w = torch.exp(x - lse[t:t + n, i, None])
                w[hidden] = 0.0
                out[t:t + n, i] = w @ v
        t += n
    return out, lse
