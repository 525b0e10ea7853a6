"""Plain implementations in 64 bits of the operators around the paged KV cache, and caches filled for their tests: everything
that a call has no business to look at (slots nobody wrote, pages of nobody, page-table entries behind the last position) holds
NaN or nonsense."""
import math

import torch

from paper_2502_08923_b200 import binding as cs

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}   # unit roundoff of a stored value


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Case:
    """Blocks of `lens` rows behind `cached` positions in a paged cache of the given shape; K and V of all kv + len positions are in `k`, `v`
    (lists of [n][Hkv][D])."""

    def __init__(self, lens, cached, H, Hkv, D, dtype=torch.bfloat16, page=16, layout="head", seed=0, spare=2, v_mean=0.0, gaps=0, first_page=0, n_pages=None):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.lens, self.cached, self.H, self.Hkv, self.D, self.page, self.dtype = lens, cached, H, Hkv, D, page, dtype
        total = [n + c for n, c in zip(lens, cached)]
        used = sum(-(-t // page) for t in total)
        n_pages = n_pages or used + spare
        shape = (n_pages, Hkv, page, D) if layout == "head" else (n_pages, page, Hkv, D)
        self.kp, self.vp = (torch.empty(shape, dtype=dtype, device="cuda") for _ in range(2))
        for p in (self.kp, self.vp):
            (p[first_page:] if first_page else p).fill_(float("nan"))
        if layout == "token":
            self.kp, self.vp = self.kp.transpose(1, 2), self.vp.transpose(1, 2)
        wide = max([-(-t // page) for t in total] + [1]) + 1
        order = (torch.randperm(n_pages - first_page, generator=torch.Generator().manual_seed(seed)) + first_page).tolist()
        table = torch.full((len(lens), wide), -1, dtype=torch.int32)
        at = 0
        self.k, self.v = [], []
        for b, t in enumerate(total):
            n = -(-t // page)
            table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
            at += n
            k = torch.randn(t, Hkv, D, generator=g, device="cuda").to(dtype)
            v = (torch.randn(t, Hkv, D, generator=g, device="cuda") + v_mean).to(dtype)
            self.k.append(k)
            self.v.append(v)
        self.table = table.cuda()
        for b in range(len(lens)):
            self.put(b)
        starts, rows = [], 0
        for n in lens:
            starts.append(rows)
            rows += n + gaps
        self.starts, self.rows = starts, rows
        self.start, self.len, self.kv_len = i32(starts), i32(lens), i32(cached)
        self.q = torch.randn(rows, H, D, generator=g, device="cuda").to(dtype)

    def put(self, b):
        """self.k[b], self.v[b] into the pages."""
        t = self.k[b].shape[0]
        if t:
            pos = torch.arange(t, device="cuda")
            at = self.table[b].long()[pos // self.page]
            self.kp[at, :, pos % self.page] = self.k[b]
            self.vp[at, :, pos % self.page] = self.v[b]

    def blocks(self):
        return self.start, self.len, self.kv_len, self.table

    def attention(self, mask=cs.MASK_CAUSAL, window=0, scale=None):
        """(out, lse, sum of weight x |value|) of the blocks' rows in 64 bits; rows of no block are NaN."""
        H, Hkv, D = self.H, self.Hkv, self.D
        scale = scale or 1.0 / math.sqrt(D)
        out, size = (torch.full((self.rows, H, D), float("nan"), dtype=torch.float64, device="cuda") for _ in range(2))
        lse = torch.full((self.rows, H), float("nan"), dtype=torch.float64, device="cuda")
        for b, (n, c) in enumerate(zip(self.lens, self.cached)):
            for r in range(n):
                p, row = c + r, self.starts[b] + r
                hi = {cs.MASK_CAUSAL: p + 1, cs.MASK_PREFIX: c, cs.MASK_FULL: c + n}[mask]
                lo = max(0, p + 1 - window) if window else 0
                if hi <= lo:
                    out[row], size[row], lse[row] = 0.0, 0.0, -math.inf
                    continue
                k = self.k[b][lo:hi].double().repeat_interleave(H // Hkv, dim=1)
                v = self.v[b][lo:hi].double().repeat_interleave(H // Hkv, dim=1)
                s = torch.einsum("hd,jhd->hj", self.q[row].double(), k) * scale
                lse[row] = torch.logsumexp(s, dim=1)
                w = torch.exp(s - lse[row][:, None])
                out[row] = torch.einsum("hj,jhd->hd", w, v)
                size[row] = torch.einsum("hj,jhd->hd", w, v.abs())
        return out, lse, size


def check_attention(case, got, lse, want, want_lse, size):
    """Rounding when stored, weights in 16 bits (u of the type each), scores in 32 bits: a score of D products is off by at most about
    D 2^-24 times the sum of their sizes, which for these inputs is below 1e-4, and so are a weight and the log of the sum."""
    u = U[case.dtype]
    live = torch.zeros(case.rows, dtype=torch.bool, device="cuda")
    for s, n in zip(case.starts, case.lens):
        live[s:s + n] = True
    d = (got.double() - want)[live].abs()
    allowed = (u * want.abs() * (1 + u) + (u + 1e-4) * size + 2.0 ** -24)[live]
    bad = ~(d <= allowed)
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} off, first {torch.nonzero(bad)[0].tolist()}, worst {float((d / allowed).nan_to_num(1e9).max()):.2f} of what rounding allows"
    a, b = lse[live].double(), want_lse[live]
    assert torch.equal(a == -math.inf, b == -math.inf)
    finite = b > -math.inf
    assert float((a - b)[finite].abs().max() if finite.any() else 0.0) <= 1e-4


def norm_rope(x, gain, rope, pos, eps=1e-5):
    """(y, what its roundings in 32 bits are relative to), 64 bits."""
    u = x.double()
    if gain is not None:
        u = u / torch.sqrt((u * u).mean(dim=-1, keepdim=True) + eps) * gain.double()
    y, size = u.clone(), u.abs()
    if rope is not None and rope.shape[1]:
        h = rope.shape[1] // 2
        c, s = rope.double()[pos.long()][:, None, :h], rope.double()[pos.long()][:, None, h:]
        a, b = u[..., :h], u[..., h:2 * h]
        y[..., :h], y[..., h:2 * h] = a * c - b * s, b * c + a * s
        size = size.clone()
        size[..., :h] = size[..., h:2 * h] = a.abs() + b.abs()
    return y, size


def check_rows(got, want, size, dtype):
    """One rounding to the stored type, and sums, a root, quotients and products in 32 bits (32 roundings are more than any value sees)."""
    allowed = U[dtype] * want.abs() * (1 + U[dtype]) + 32 * 2.0 ** -24 * size + (2.0 ** -25 if dtype is torch.float16 else 0.0)
    d = (got.double() - want).abs()
    assert bool((d <= allowed).all()), f"worst {float((d / allowed.clamp(min=1e-30)).max()):.2f} of what rounding allows"
