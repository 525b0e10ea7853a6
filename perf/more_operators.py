"""The operators around a paged key/value cache held in 4 bits, as a server of copy-and-verify decoding calls them: what is measured, their plain
forms, and their definitions in 64 bits.

Three operators (`op`):
  append      a block's keys (normed, rotated) and values quantised into the pages of their sequences, the block's queries normed and rotated with
              them; what the pages hold of the block is read back, so a pass is a write and a read
  read        whole sequences read back in 16 bits
  attention   blocks of new rows, from single tokens to a prompt's chunk, over the pages

The cache: a row (one position, one KV head) is cut into groups of 32 neighbouring elements.  With a = max |x| of a group, s = a / 7 rounded to five
significant bits (nearest, halves to even) and n = x / s rounded to the nearest whole number (halves to even), at most 7 either way, the group is held as s (bf16) and 4-bit numbers
n + 8, and stands for s n.  Eight elements make a word of 32 bits: elements 2i and 2i + 1 are its fields i and i + 4, and field f begins at bit 4f.  A page holds [KV head][slot] rows of words, and of scales.

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
GROUP = 32


def listed():
    att = {"op": "attention", "dtype": "bf16", "page": 16, "ragged": False, "mask": "causal", "window": 0}
    app = {"op": "append", "dtype": "bf16", "source": "bf16", "page": 16, "ragged": False, "norm": True}
    red = {"op": "read", "dtype": "bf16", "page": 16, "ragged": False}
    return [
        # the smallest call: the small model verifies ten copied tokens behind 512, launch latency counts
        att | {"name": "attn4_tiny_b1_512_k10", "shape": "tiny", "batch": 1, "rows": 11, "keys": 512},
        # the usual verification: one sequence, 4k context, ten copied tokens
        att | {"name": "attn4_8b_b1_4k_k10", "shape": "8b", "batch": 1, "rows": 11, "keys": 4096},
        # one token over a long document
        att | {"name": "attn4_8b_b1_30k_decode", "shape": "8b", "batch": 1, "rows": 1, "keys": 30720},
        # a server's batch of single tokens, sequences of all lengths
        att | {"name": "attn4_8b_b64_4k_decode", "shape": "8b", "dtype": "fp16", "page": 64, "batch": 64, "rows": 1, "keys": 4097, "ragged": True},
        # a draft model's blocks behind long contexts, twenty copied tokens
        att | {"name": "attn4_1b_b8_16k_k20", "shape": "1b", "page": 32, "batch": 8, "rows": 21, "keys": 16384},
        # chunks of several prompts with a sliding window, odd sizes
        att | {"name": "attn4_8b_b3_chunk_1531_window", "shape": "8b", "dtype": "fp16", "page": 64, "batch": 3, "rows": 1531, "keys": 3001, "ragged": True, "window": 1000},
        # the largest: a prompt's chunk behind a long context
        att | {"name": "attn4_8b_b1_30k_chunk_2048", "shape": "8b", "page": 64, "batch": 1, "rows": 2048, "keys": 30720},
        # a verification block's rows into the cache, straight out of a projection in 32 bits
        app | {"name": "append4_8b_b1_k10", "shape": "8b", "source": "fp32", "batch": 1, "rows": 11, "keys": 4096},
        # a server's batch of single tokens of the draft model, rotation only
        app | {"name": "append4_1b_b64_decode", "shape": "1b", "dtype": "fp16", "source": "fp16", "page": 32, "batch": 64, "rows": 1, "keys": 1531, "ragged": True, "norm": False},
        # chunks of four prompts
        app | {"name": "append4_8b_b4_chunk_2048", "shape": "8b", "page": 64, "batch": 4, "rows": 2048, "keys": 1024, "ragged": True},
        # the last block of the draft model's sequences, for a check
        red | {"name": "read4_1b_b3_k20", "shape": "1b", "dtype": "fp16", "batch": 3, "rows": 21, "keys": 1000, "ragged": True},
        # two long sequences, on their way into a cache of 16 bits
        red | {"name": "read4_8b_b2_16k", "shape": "8b", "page": 64, "batch": 2, "rows": 16384, "keys": 0},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attention", "attention", "attention", "append", "append", "read"])
    shape = rng.choice(["8b", "8b", "8b", "1b", "1b", "tiny"])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    page = rng.choice([16, 16, 32, 64, 128])
    if op == "read":
        rows = _log_int(rng, 1, 32768)
        batch = min(rows, _log_int(rng, 1, 64))
        return {"op": op, "shape": shape, "dtype": dtype, "page": page, "batch": batch, "rows": rows // batch, "keys": rng.choice([0, _log_int(rng, 1, 32768 // batch)]), "ragged": rng.random() < 0.6}
    if op == "append":
        rows = _log_int(rng, 1, 8192)
        batch = min(rows, _log_int(rng, 1, 64))
        return {"op": op, "shape": shape, "dtype": dtype, "source": rng.choice([dtype, dtype, "fp32"]), "page": page, "batch": batch, "rows": rows // batch,
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
    return {"op": op, "shape": shape, "dtype": dtype, "page": page, "batch": batch, "rows": rows, "keys": keys, "ragged": rng.random() < 0.6,
            "mask": rng.choice(["causal", "causal", "causal", "prefix"]), "window": rng.choice([0, 0, 0, _log_int(rng, 20, 4096)])}


def _lengths(case):
    """Rows of each sequence's block and what it has cached, by the case alone (a case's work is the same whatever the seed)."""
    B, rows, keys = case["batch"], case["rows"], case["keys"]
    if not case["ragged"]:
        return [rows] * B, [keys] * B
    rng = random.Random(1000003 * B + 1009 * rows + keys)
    return [rng.randint((rows + 1) // 2, rows) for _ in range(B)], [_log_int(rng, max(1, keys // 8), keys) if keys else 0 for _ in range(B)]


def _range(case, n, c, r):
    """Keys [lo, hi) that row r of a block of n rows behind c cached keys attends to."""
    hi = c + r + 1 if case["mask"] == "causal" else c
    return (max(0, c + r + 1 - case["window"]) if case["window"] else 0), hi


def _rope(positions, dim, theta):
    inv = theta ** (-torch.arange(0, dim, 2, dtype=torch.float64, device=DEVICE) / dim)
    angle = torch.arange(positions, dtype=torch.float64, device=DEVICE)[:, None] * inv
    return torch.cat([angle.cos(), angle.sin()], dim=1).float()


# ------------------------------------------------------------------------------------------ the format, in elementary operations
def _round5(x):
    """Nearest number of five significant bits, halves to even (x in 64 bits, 0 or more)."""
    b = x.contiguous().view(torch.int64)
    return ((b + ((1 << 47) - 1) + ((b >> 48) & 1)) >> 48 << 48).view(torch.float64)


def _quantise(x):
    """Rows of 32- or 64-bit values -> (whole numbers -7 .. 7, scales in 64 bits for every 32)."""
    g = x.double().unflatten(-1, (-1, GROUP))
    s = _round5(g.abs().amax(dim=-1) / 7)
    n = torch.round(g / torch.where(s > 0, s, torch.ones_like(s))[..., None]).clamp_(-7, 7)
    return n.flatten(-2), s


def _pack(n):
    """Whole numbers [..., D] -> bytes [..., D / 2]."""
    u = (n.to(torch.int64) + 8).unflatten(-1, (-1, 4, 2)).transpose(-1, -2).flatten(-2)               # fields 0 .. 7 of every word
    w = (u << (4 * torch.arange(8, device=u.device))).sum(dim=-1)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32).contiguous().view(torch.uint8)


def _unpack(data):
    """Bytes [..., D / 2] -> whole numbers -8 .. 7 [..., D], 32 bits."""
    w = data.contiguous().view(torch.int32)
    u = (w[..., None] >> (4 * torch.arange(8, device=w.device, dtype=torch.int32))) & 15
    return (u - 8).unflatten(-1, (2, 4)).transpose(-1, -2).flatten(-3).float()


def _values(data, scale):
    return (_unpack(data).unflatten(-1, (-1, GROUP)) * scale.float()[..., None]).flatten(-2)


def prepare(case, seed):
    H, Hkv, D, theta = SHAPES[case["shape"]]
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0, to=dtype):
        return (torch.randn(*shape, generator=g, device=DEVICE) * scale).to(to)

    def gain(n):
        return normal(n, scale=0.1, to=torch.float32).add_(1.0).to(dtype)

    lens, cached = _lengths(case)
    B, T, page = case["batch"], sum(lens), case["page"]
    total = [n + c for n, c in zip(lens, cached)]
    wide = max(-(-t // page) for t in total)
    used = sum(-(-t // page) for t in total)
    n_pages = used + 3
    # what earlier blocks left in the pages: rows of normal values, some channels of the keys larger than others
    data = torch.empty(2, n_pages, Hkv, page, D // 2, dtype=torch.uint8, device=DEVICE)
    scale = torch.empty(2, n_pages, Hkv, page, D // GROUP, dtype=torch.bfloat16, device=DEVICE)
    channels = torch.exp(0.3 * torch.randn(Hkv, 1, D, generator=g, device=DEVICE))
    step = max(1, 4_000_000 // (Hkv * page * D))
    for which in range(2):
        for at in range(0, n_pages, step):
            rows = torch.randn(min(step, n_pages - at), Hkv, page, D, generator=g, device=DEVICE)
            n, sc = _quantise(rows * channels if which == 0 else rows)
            data[which, at:at + step], scale[which, at:at + step] = _pack(n), sc.to(torch.bfloat16)
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
    s = {"case": case, "k_data": data[0], "v_data": data[1], "k_scale": scale[0], "v_scale": scale[1], "table": table, "start": ints[0], "len": ints[1], "kv_len": ints[2], "rows": T}
    if case["op"] == "attention":
        # heads differ in how sharply they look
        s["q"] = (torch.randn(T, H, D, generator=g, device=DEVICE) * torch.linspace(0.5, 2.5, H, device=DEVICE)[:, None]).to(dtype)
    elif case["op"] == "append":
        qkv = normal(T, (H + 2 * Hkv) * D, to=DTYPES[case["source"]])                 # a projection's output; queries, keys and values are views of it
        s |= {"q": qkv[:, :H * D].unflatten(1, (H, D)), "k": qkv[:, H * D:(H + Hkv) * D].unflatten(1, (Hkv, D)), "v": qkv[:, (H + Hkv) * D:].unflatten(1, (Hkv, D)),
              "rope": _rope(max(total), D, theta), "q_gain": gain(D) if case["norm"] else None, "k_gain": gain(D) if case["norm"] else None}
    if own:
        from paper_2502_08923_b200 import binding as cs
        # room for prompts' chunks: as many positions as the batch's page table has
        s["cache"] = cs.QuantCache(s["k_data"], s["v_data"], s["k_scale"], s["v_scale"], tall_positions=B * wide * page if case["op"] == "attention" else 0)
    return s


# ------------------------------------------------------------------------------------------ plain forms
def _norm_rope(x, gain, rope, pos, to):
    x = x.to(to)
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * gain.to(to)
    h = x.shape[-1] // 2
    cs = rope[pos.long()][:, None, :].to(to)
    c, sn = cs[..., :h], cs[..., h:]
    a, b = x[..., :h], x[..., h:]
    return torch.cat([a * c - b * sn, b * c + a * sn], dim=-1)


def _places(s):
    """Page, slot and position of every row."""
    page = s["k_data"].shape[2]
    t = torch.arange(s["rows"], device=DEVICE)
    b = (t[:, None] >= s["start"][None, :]).sum(dim=1) - 1
    pos = s["kv_len"][b].long() + t - s["start"][b].long()
    return s["table"][b, pos // page].long(), pos % page, pos


def _plain_read(s, at, slot, dtype):
    return _values(s["k_data"][at, :, slot], s["k_scale"][at, :, slot]).to(dtype), _values(s["v_data"][at, :, slot], s["v_scale"][at, :, slot]).to(dtype)


def _plain_append(s):
    at, slot, pos = _places(s)
    # (64 bits: which level a key goes to is decided at the border of two)
    for name, x in (("k", _norm_rope(s["k"], s["k_gain"], s["rope"], pos, torch.float64)), ("v", s["v"])):
        n, scale = _quantise(x)
        s[name + "_data"][at, :, slot] = _pack(n)
        s[name + "_scale"][at, :, slot] = scale.to(torch.bfloat16)
    dtype = DTYPES[s["case"]["dtype"]]
    return _norm_rope(s["q"], s["q_gain"], s["rope"], pos, torch.float32).to(dtype), *_plain_read(s, at, slot, dtype)


def _plain_attention(s):
    case, q = s["case"], s["q"]
    H, Hkv, D, _ = SHAPES[case["shape"]]
    (T, page), B = (q.shape[0], s["k_data"].shape[2]), s["table"].shape[0]
    R, N = case["rows"], s["table"].shape[1] * page
    # every sequence's rows and keys side by side, as wide as the longest has them
    r, j = torch.arange(R, device=DEVICE), torch.arange(N, device=DEVICE)
    row = (s["start"][:, None] + r).clamp(max=T - 1).long()
    live = r[None, :] < s["len"][:, None]
    at = s["table"].long().clamp(min=0)
    k = _values(s["k_data"][at], s["k_scale"][at]).transpose(1, 2).reshape(B, Hkv, 1, N, D)
    v = _values(s["v_data"][at], s["v_scale"][at]).transpose(1, 2).reshape(B, Hkv, 1, N, D)
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
    dtype = DTYPES[case["dtype"]]
    if own:
        blocks = s["start"], s["len"], s["kv_len"], s["table"]
        if case["op"] == "read":
            return s["cache"].cs_quant_read(*blocks, rows=s["rows"], dtype=dtype)
        if case["op"] == "append":
            q = s["cache"].cs_quant_append(s["k"], s["v"], *blocks, s["rope"], k_gain=s["k_gain"], q=s["q"], q_gain=s["q_gain"], eps=EPS, dtype=dtype)
            return q, *s["cache"].cs_quant_read(*blocks, rows=s["rows"], dtype=dtype)
        from paper_2502_08923_b200 import binding as cs
        return s["cache"].cs_quant_attention(s["q"], *blocks, window=case["window"], mask=cs.MASK_CAUSAL if case["mask"] == "causal" else cs.MASK_PREFIX, with_lse=True)
    if case["op"] == "read":
        at, slot, _ = _places(s)
        return _plain_read(s, at, slot, dtype)
    return _plain_append(s) if case["op"] == "append" else _plain_attention(s)


def work(case):
    H, Hkv, D, _ = SHAPES[case["shape"]]
    size = {"bf16": 2, "fp16": 2, "fp32": 4}
    e, held = size[case["dtype"]], 0.5 + 2 / GROUP               # bytes of a value
    lens, cached = _lengths(case)
    T = sum(lens)
    if case["op"] == "read":
        return {"bytes": int(T * 2 * Hkv * D * (held + e)), "flops": T * 2 * Hkv * D}
    if case["op"] == "append":
        # rows in, queries out, keys and values into the pages, out of them again and to their readers; the rotation's rows: each position once at most
        n = T * 2 * Hkv * D
        return {"bytes": int((T * H * D + n) * size[case["source"]] + T * H * D * e + n * (2 * held + e) + 4 * D * min(T, max(a + c for a, c in zip(lens, cached)))), "flops": 12 * (T * H * D + n)}
    pairs = keys = 0
    for n, c in zip(lens, cached):
        ends = [_range(case, n, c, r) for r in range(n)]
        pairs += sum(max(0, hi - lo) for lo, hi in ends)
        keys += max(0, max(hi for _, hi in ends) - min(lo for lo, _ in ends))
    return {"bytes": int(keys * 2 * Hkv * D * held + T * H * (2 * D * e + 4)), "flops": 4 * D * H * pairs}


# ------------------------------------------------------------------------------------------ definitions in 64 bits
def _exact_held(x):
    """What the cache stands for where it was given x (64 bits): each group's scale by its exponent, each element by the nearest multiple of it."""
    g = x.unflatten(-1, (-1, GROUP))
    seventh = g.abs().amax(dim=-1, keepdim=True) / 7
    unit = torch.exp2(torch.floor(torch.log2(torch.where(seventh > 0, seventh, torch.ones_like(seventh)))) - 4)
    # (log2 may end up on the wrong side of a power of two, where either unit gives the same five bits)
    s = torch.round(seventh / unit) * unit
    y = torch.where(s > 0, torch.clamp(torch.round(g / torch.where(s > 0, s, unit)), -7, 7) * s, torch.zeros_like(g))
    return y.flatten(-2)


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


def _exact_pages(data, scale, pages, n):
    """Values [heads][n][D] in 64 bits of the first n positions of some pages, nibble by nibble."""
    b = data[pages].transpose(0, 1).flatten(1, 2)[:, :n].to(torch.int64).unflatten(-1, (-1, 4))
    w = b[..., 0] + b[..., 1] * 256 + b[..., 2] * 65536 + b[..., 3] * 16777216
    out = torch.empty(*w.shape, 8, dtype=torch.float64, device=w.device)
    for f in range(8):
        out[..., 2 * (f % 4) + f // 4] = (w // 16 ** f % 16 - 8).double()
    s = scale[pages].transpose(0, 1).flatten(1, 2)[:, :n].double()
    return out.flatten(-2) * s.repeat_interleave(GROUP, dim=-1)


def exact(case, seed):
    s = prepare(case, seed)
    H, Hkv, D, _ = SHAPES[case["shape"]]
    G, page = H // Hkv, case["page"]
    lens, cached = _lengths(case)
    if case["op"] == "append":
        pos = torch.cat([torch.arange(c, c + n) for n, c in zip(lens, cached)]).to(DEVICE)
        q, k = _exact_row_heads(s["q"], s["q_gain"], s["rope"], pos), _exact_row_heads(s["k"], s["k_gain"], s["rope"], pos)
        return q, _exact_held(k), _exact_held(s["v"].double())
    keys = []
    for b, (n, c) in enumerate(zip(lens, cached)):
        pages = s["table"][b, :-(-(n + c) // page)].long()
        keys.append([_exact_pages(s[x + "_data"], s[x + "_scale"], pages, n + c) for x in "kv"])
    if case["op"] == "read":
        return tuple(torch.cat([kv[i][:, c:].transpose(0, 1) for kv, c in zip(keys, cached)]) for i in range(2))
    out, lse, t = torch.empty(sum(lens), H, D, dtype=torch.float64, device=DEVICE), torch.empty(sum(lens), H, dtype=torch.float64, device=DEVICE), 0
    for (k, v), n, c in zip(keys, lens, cached):
        ends = torch.tensor([_range(case, n, c, r) for r in range(n)], device=DEVICE)
        j = torch.arange(n + c, device=DEVICE)
        hidden = (j < ends[:, :1]) | (j >= ends[:, 1:])
        for h in range(H):
            x = s["q"][t:t + n, h].double() @ k[h // G].T / math.sqrt(D)
            x[hidden] = -math.inf
            total = torch.logsumexp(x, dim=1)
            lse[t:t + n, h] = total
            w = torch.exp(x - total[:, None])
            w[hidden] = 0.0
            out[t:t + n, h] = w @ v[h // G]
        t += n
    return out, lse
