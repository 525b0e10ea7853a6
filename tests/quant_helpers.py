"""Plain implementations in 64 bits of the operators around the paged KV cache held in 4 bits, and caches filled for their tests: everything
that a call has no business to look at (slots nobody wrote, pages of nobody, page-table entries behind the last position) holds scales of NaN or nonsense."""
import math

import torch

from paged_helpers import U, i32, norm_rope          # noqa: F401  (tests take them from here)
from paper_2502_08923_b200 import binding as cs

GROUP = 32


def round5(x):
    """x >= 0 in 64 bits to five significant bits, halves to even."""
    e = torch.floor(torch.log2(torch.where(x > 0, x, torch.ones_like(x))))
    # (log2 may be off by one beside powers of two, where both units give the same)
    unit = torch.ldexp(torch.ones_like(x), (e - 4).to(torch.int32).double())
    return torch.where(x > 0, torch.round(x / unit) * unit, x)


def quantise(x):
    """Rows [..., D] -> (whole numbers [..., D], scales [..., D / 32]) in 64 bits; groups with a value that is not finite: 0 and NaN."""
    g = x.double().unflatten(-1, (-1, GROUP))
    odd = ~torch.isfinite(g).all(dim=-1)
    g = torch.where(odd[..., None], torch.zeros_like(g), g)
    s = torch.clamp(round5(g.abs().amax(dim=-1) / 7), max=2.0 ** 123)
    n = torch.round(g / torch.where(s > 0, s, torch.ones_like(s))[..., None]).clamp(-7, 7)
    return n.flatten(-2), torch.where(odd, torch.full_like(s, math.nan), s)


def held(n, s):
    """What numbers and scales stand for."""
    return (n.unflatten(-1, (-1, GROUP)) * s[..., None]).flatten(-2)


def pack(n):
    """Numbers -8 .. 7 [..., D] -> bytes [..., D / 2], byte by byte: elements 0, 2, 4, 6 of eight fill a word's low half from bit 0 on, 1, 3, 5, 7 its high half."""
    u = (n + 8).to(torch.uint8).unflatten(-1, (-1, 8))
    return torch.stack([u[..., a] | (u[..., b] << 4) for a, b in ((0, 2), (4, 6), (1, 3), (5, 7))], dim=-1).flatten(-2)


def unpack(data):
    b = data.unflatten(-1, (-1, 4)).to(torch.int16)
    n = torch.empty(*b.shape[:-1], 8, dtype=torch.float64, device=data.device)
    for i, (lo, hi) in enumerate(((0, 2), (4, 6), (1, 3), (5, 7))):
        n[..., lo], n[..., hi] = (b[..., i] & 15).double() - 8, (b[..., i] >> 4).double() - 8
    return n.flatten(-2)


class QuantCase:
    """Blocks of `lens` rows behind `cached` positions in a paged cache of 4 bits; what the cache stands for at all kv + len positions is in `k`, `v` (lists of [n][Hkv][D], 64 bits)."""

    def __init__(self, lens, cached, H, Hkv, D, dtype=torch.bfloat16, page=16, seed=0, spare=2, v_mean=0.0, gaps=0, first_page=0, n_pages=None, tall=0, apart=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.lens, self.cached, self.H, self.Hkv, self.D, self.page, self.dtype = lens, cached, H, Hkv, D, page, dtype
        total = [n + c for n, c in zip(lens, cached)]
        used = sum(-(-t // page) for t in total)
        n_pages = n_pages or used + spare
        # `apart`: pages that lie that many heads' rows apart
        self.data = torch.empty(2, n_pages, Hkv + apart, page, D // 2, dtype=torch.uint8, device="cuda")
        self.scales = torch.empty(2, n_pages, Hkv + apart, page, D // GROUP, dtype=torch.bfloat16, device="cuda")
        for x, y in zip(self.data, self.scales):
            (x[first_page:] if first_page else x).fill_(0x3F)
            (y[first_page:] if first_page else y).fill_(float("nan"))
        self.kd, self.vd = self.data[0, :, :Hkv], self.data[1, :, :Hkv]
        self.ks, self.vs = self.scales[0, :, :Hkv], self.scales[1, :, :Hkv]
        wide = max([-(-t // page) for t in total] + [1]) + 1
        order = (torch.randperm(n_pages - first_page, generator=torch.Generator().manual_seed(seed)) + first_page).tolist()
        table = torch.full((len(lens), wide), -1, dtype=torch.int32)
        at = 0
        self.k, self.v = [], []
        for b, t in enumerate(total):
            n = -(-t // page)
            table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
            at += n
            self.k.append(torch.randn(t, Hkv, D, generator=g, device="cuda"))
            self.v.append(torch.randn(t, Hkv, D, generator=g, device="cuda") + v_mean)
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
        self.cache = cs.QuantCache(self.kd, self.vd, self.ks, self.vs, tall_positions=tall)

    def put(self, b):
        """self.k[b], self.v[b] into the pages, quantised; they become what the pages stand for."""
        t = self.k[b].shape[0]
        if not t:
            self.k[b], self.v[b] = self.k[b].double(), self.v[b].double()
            return
        pos = torch.arange(t, device="cuda")
        at = self.table[b].long()[pos // self.page]
        for rows, data, scales in ((self.k, self.kd, self.ks), (self.v, self.vd, self.vs)):
            n, s = quantise(rows[b])
            data[at, :, pos % self.page] = pack(n)
            scales[at, :, pos % self.page] = s.to(torch.bfloat16)
            rows[b] = held(n, s)

    def blocks(self):
        return self.start, self.len, self.kv_len, self.table

    def live(self):
        x = torch.zeros(self.rows, dtype=torch.bool, device="cuda")
        for s, n in zip(self.starts, self.lens):
            x[s:s + n] = True
        return x

    def attention(self, mask=cs.MASK_CAUSAL, window=0, scale=None):
        """(out, lse, sum of weight x |value|) of the blocks' rows in 64 bits; rows of no block are NaN."""
        H, Hkv, D = self.H, self.Hkv, self.D
        scale = scale or 1.0 / math.sqrt(D)
        out, size = (torch.full((self.rows, H, D), float("nan"), dtype=torch.float64, device="cuda") for _ in range(2))
        lse = torch.full((self.rows, H), float("nan"), dtype=torch.float64, device="cuda")
        for b, (n, c) in enumerate(zip(self.lens, self.cached)):
            if not n:
                continue
            r = torch.arange(n, device="cuda")
            p = c + r
            hi = {cs.MASK_CAUSAL: p + 1, cs.MASK_PREFIX: torch.full_like(p, c), cs.MASK_FULL: torch.full_like(p, c + n)}[mask]
            lo = (p + 1 - window).clamp(min=0) if window else torch.zeros_like(p)
            j = torch.arange(n + c, device="cuda")
            seen = (j >= lo[:, None]) & (j < hi[:, None])
            rows = slice(self.starts[b], self.starts[b] + n)
            for h in range(H):
                k, v = self.k[b][:, h * Hkv // H], self.v[b][:, h * Hkv // H]
                s = (self.q[rows, h].double() @ k.T * scale).masked_fill(~seen, -math.inf)
                m = s.amax(dim=1, keepdim=True) if n + c else torch.full((n, 1), -math.inf, dtype=torch.float64, device="cuda")
                w = torch.exp(s - torch.where(m == -math.inf, torch.zeros_like(m), m)).masked_fill(~seen, 0.0)
                total = w.sum(dim=1, keepdim=True)
                lse[rows, h] = (m + total.log()).squeeze(1)
                w = w / torch.where(total == 0, torch.ones_like(total), total)
                # (values that are not finite reach the rows that see them, and no others)
                odd = ~torch.isfinite(v)
                clean = torch.where(odd, torch.zeros_like(v), v)
                out[rows, h] = torch.where((seen.double() @ odd.double()) > 0, torch.full_like(w @ clean, math.nan), w @ clean)
                size[rows, h] = w @ clean.abs()
        return out, lse, size


def is_tall(case, window=0):
    """Worked out on the 5th-generation tensor cores, with one 16-bit term of every weight (queries that repeat one row are not)."""
    B = len(case.lens)
    rows, room = -(-case.q.shape[0] * (case.H // case.Hkv) // B), case.table.shape[1] * case.page
    seen = min(room, window + case.q.shape[0] // B) if window else room
    return rows > 32 and (rows > 128 or rows * B * case.Hkv * seen > 3 << 19) and case.q.stride(0) > 0 and case.q.stride(1) > 0


def check_attention(case, got, lse, want, want_lse, size, tall=False):
    """Rounding when stored (u of the type); weights as two bf16 terms, 16 bits of them, or in tall blocks as one term (u of the type); scores in 32 bits: a score of D products is off by at most about
    D 2^-24 times the sum of their sizes, which for these inputs is below 1e-4, and so are a weight and the log of the sum.  Values are exact."""
    u = U[case.dtype]
    live = case.live()
    odd = torch.isnan(want) | torch.isnan(want_lse)[..., None]
    assert torch.equal(torch.isnan(got)[live], odd[live])
    fine = live[:, None, None] & ~odd
    d = (got.double() - want)[fine].abs()
    allowed = (u * want.abs() * (1 + u) + ((u if tall else 2.0 ** -16) + 1e-4) * size + 2.0 ** -24)[fine]
    bad = ~(d <= allowed)
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} off, first {torch.nonzero((got.double() - want).abs().nan_to_num(0.0) > (u * want.abs() * (1 + u) + ((u if tall else 2.0 ** -16) + 1e-4) * size + 2.0 ** -24).nan_to_num(9.9))[:3].tolist()}, worst {float((d / allowed).max()):.2f} of what rounding allows"
    a, b = lse[live].double(), want_lse[live]
    assert torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(a == -math.inf, b == -math.inf)
    finite = torch.isfinite(b)
    assert float((a - b)[finite].abs().max() if finite.any() else 0.0) <= 1e-4
